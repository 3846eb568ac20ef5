"""The int8 layers with a scale per token on the GPU against 64-bit references, at the sizes, types, strides and values where they can go wrong."""
import numpy as np
import pytest
import torch

import token_forms as S
import token_ref as R

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2507_19131_amd import binding as M

FILL = 0x5A                                                     # what unwritten bytes hold
NAN = float("nan")


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def values(seed, rows, cols):
    return normal(seed, rows, cols) * torch.exp(0.5 * normal(seed + 1, cols)) * torch.where(torch.arange(cols, device="cuda") % 37 == 5, 12.0, 1.0)


class Room:
    """A matrix inside a larger buffer: `before` columns in front of it, `after` columns and a row behind it, all filled with a pattern."""

    def __init__(self, rows, cols, kind, before=0, after=0):
        dtype = R.TYPES[kind]
        es, width = dtype.itemsize, before + cols + after
        if kind == "i8":
            width = -(-width // 16) * 16
        self.buffer = torch.full((rows + 1, width * es), FILL, dtype=torch.uint8, device="cuda")
        self.t = self.buffer.view(dtype)[:rows, before:before + cols]
        self.columns = (before * es, (before + cols) * es)
        self.scales = torch.full((rows,), -1.0, device="cuda") if kind == "i8" else None

    def untouched(self):
        rows = self.t.shape[0]
        return bool((self.buffer[rows:] == FILL).all() and (self.buffer[:, :self.columns[0]] == FILL).all() and (self.buffer[:, self.columns[1]:] == FILL).all())


def placed(v, kind, before=0, after=0):
    room = Room(v.shape[0], v.shape[1], kind, before, after)
    if kind == "i8":
        codes, scales = R.quantize(v)
        room.t.copy_(codes)
        room.scales.copy_(scales)
    else:
        room.t.copy_(v.to(R.TYPES[kind]))
    return room


class Layer:
    """`experts` matrices drawn from a seed, and their handle."""

    def __init__(self, seed, N, K, experts=1, act="none", bias=True):
        self.w = placed(normal(seed, experts * N, K) / K ** 0.5, "i8")
        self.bias = 0.3 * normal(seed + 1, experts * N) if bias else None
        self.N, self.K, self.experts, self.act = N, K, experts, act
        self.h = M.mixaq_token_linear_create(self.w.t, self.w.scales, self.bias, act, experts)

    def __enter__(self):
        return self

    def __exit__(self, *_):
        torch.cuda.synchronize()
        M.mixaq_token_linear_destroy(self.h)

    def matrix(self, e=0):
        mine = slice(e * self.N, (e + 1) * self.N)
        return self.w.t[mine], self.w.scales[mine], None if self.bias is None else self.bias[mine]

    def reference(self, codes, scales, e=0, weights=None):
        return R.linear(codes, scales, *self.matrix(e), self.act, weights)

    def forward(self, x, y, scales=None):
        return M.mixaq_token_linear_forward(self.h, x, y, x_scales=scales, workspace=M.alloc_token_linear_workspace(self.h, x.shape[0], x.dtype))

    def grouped(self, x, offsets, y, scales=None, **kw):
        return M.mixaq_token_linear_forward_grouped(self.h, x, offsets, y, x_scales=scales, workspace=M.alloc_token_linear_workspace(self.h, x.shape[0], x.dtype), **kw)


# ---------------------------------------------------------------- quantizer
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,before,after", [
    (1, 1, 0, 0), (1, 7, 0, 0), (3, 8, 1, 0), (49, 96, 0, 0), (17, 129, 1, 2), (130, 257, 3, 5), (33, 384, 0, 8), (18, 500, 0, 0), (5, 1000, 7, 0), (9, 1500, 0, 1), (6, 2047, 0, 0),
    (5, 4096, 0, 0), (4, 8191, 3, 0), (3, 8193, 0, 0), (2, 30001, 5, 0)])
def test_codes_are_the_references(kind, rows, cols, before, after):
    x = placed(values(rows + cols, rows, cols), kind, before, after)
    q = Room(rows, cols, "i8", 16, 16 + before)
    M.mixaq_token_quantize(x.t, q.t, q.scales)
    codes, scales = R.quantize(x.t)
    R.same(q.scales, scales)
    R.same(q.t, codes)
    assert q.untouched()


@pytest.mark.parametrize("cols", [5, 100, 300, 1100, 5000, 9000])
def test_rows_of_special_values(cols):
    inf = float("inf")
    x = values(7, 12, cols)
    x[0] = 0.0
    x[1] *= 1e-42                                               # below the normal numbers
    x[2, 3] = -0.0
    x[3, cols - 1] = inf
    x[4, 0], x[4, 1] = NAN, -inf
    x[5] = 3.4028234e38
    x[6] = 2.0 ** -126
    x[7] = torch.arange(cols, device="cuda") % 255 - 127.0      # every code, from whole numbers
    x[8] = (torch.arange(cols, device="cuda") % 253 - 126.0) + 0.5
    x[8, 0] = 127.0                                             # ties, to the even code
    x[9, cols // 2] = -inf
    q = Room(12, cols, "i8")
    M.mixaq_token_quantize(x, q.t, q.scales)
    codes, scales = R.quantize(x)
    R.same(q.scales.view(torch.int32), scales.view(torch.int32))
    R.same(q.t, codes)
    assert bool((q.t[[0, 3, 4, 9]] == 0).all())


# ---------------------------------------------------------------- layers
@pytest.mark.parametrize("y_kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lines", [False, True])
@pytest.mark.parametrize("rows,K,N", S.SIZES)
def test_layer_to_the_last_bit(rows, K, N, lines, y_kind):
    """Without an activation every step has one nearest result.  Behind a row's columns x holds a pattern, and y keeps one.  lines: y's rows start at multiples of
    16 bytes."""
    with Layer(rows + K, N, K, bias=N % 2 == 0) as layer:
        x, y = placed(values(rows, rows, K), "i8", 16, 16), Room(rows, N, y_kind, 8, 8 + -N % 8) if lines else Room(rows, N, y_kind, 3, 2)
        layer.forward(x.t, y.t, x.scales)
        want = R.linear_bits(x.t, x.scales, *layer.matrix(), y_kind)
        R.same(y.t, want)
        assert y.untouched()


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
@pytest.mark.parametrize("rows,K,N", [(1, 1000, 333), (40, 1024, 512), (700, 1500, 200), (2100, 384, 1500), (9000, 790, 1300)])
def test_activations(rows, K, N, act):
    for kind in ("f32", "bf16"):
        with Layer(rows + K, N, K, act=act) as layer:
            x, y = placed(values(rows, rows, K), "i8"), Room(rows, N, kind)
            layer.forward(x.t, y.t, x.scales)
            R.check(y.t, *layer.reference(x.t, x.scales), kind)


@pytest.mark.parametrize("x_kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,K,N", [(1, 1, 1), (1, 1000, 333), (2, 5000, 70), (16, 1024, 512), (17, 127, 129), (130, 1000, 333), (2100, 384, 1500), (4800, 96, 400)])
def test_values_and_codes_are_two_forms_of_one_call(rows, K, N, x_kind):
    with Layer(rows + K, N, K, act="gelu") as layer:
        x = placed(values(rows, rows, K), x_kind, 3, 0)
        codes, scales = R.quantize(x.t)
        q = placed(values(rows, rows, K), "i8")
        q.t.copy_(codes)
        a, b = Room(rows, N, "f32"), Room(rows, N, "f32")
        layer.forward(x.t, a.t)
        layer.forward(q.t, b.t, scales)
        R.same(a.t, b.t)
        assert x.untouched()


def test_a_row_depends_on_nothing_but_itself():
    """The same bits whatever stands beside a row and however many there are: sums are whole numbers."""
    K, N, rows = 500, 600, 9000
    with Layer(11, N, K, act="gelu") as layer:
        x = placed(values(12, rows, K), "i8")
        y = torch.empty(rows, N, device="cuda")
        layer.forward(x.t, y, x.scales)
        for n in (1, 5, 16, 33, 200, 1000, 3000):
            part = torch.empty(n, N, device="cuda")
            layer.forward(x.t[77:77 + n], part, x.scales[77:77 + n])
            R.same(part, y[77:77 + n])
        x.scales[::3] = NAN                                     # rows without a scale
        other = torch.empty_like(y)
        layer.forward(x.t, other, x.scales)
        assert torch.equal(other[1::3], y[1::3]) and torch.equal(other[2::3], y[2::3]) and bool(torch.isnan(other[::3]).all())


@pytest.mark.parametrize("rows", [3, 300, 5000])
def test_the_largest_sums(rows):
    """65536 products of the largest codes, -128 (which the quantizer never gives) among them: 2^30 and 2^30 - 2^17 fit 32 bits."""
    K, N = 65536, 70
    w, x = torch.full((N, K), 127, dtype=torch.int8, device="cuda"), torch.full((rows, K), 127, dtype=torch.int8, device="cuda")
    w[1], w[2], w[3, ::2], x[2] = -127, -128, -127, -128
    one = torch.ones(max(rows, N), device="cuda")
    h = M.mixaq_token_linear_create(w, one[:N])
    y = torch.empty(rows, N, device="cuda")
    M.mixaq_token_linear_forward(h, x, y, x_scales=one[:rows])
    torch.cuda.synchronize()
    M.mixaq_token_linear_destroy(h)
    want = x[:3].double() @ w.double().t()
    assert float(want.max()) == 2.0 ** 30 and torch.equal(y[:3].double(), want) and torch.equal(y[3:], y[:1].expand(rows - 3, N))


def test_scales_at_both_ends_of_their_range():
    with Layer(21, 200, 300) as layer:
        x = placed(values(22, 400, 300), "i8")
        x.scales[:100], x.scales[100:200] = 2.0 ** -107, 2.0 ** 110
        y = torch.empty(400, 200, device="cuda")
        layer.forward(x.t, y, x.scales)
        R.same(y, R.linear_bits(x.t, x.scales, *layer.matrix(), "f32"))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K,N", [(5, 208, 100), (16, 1000, 333), (60, 1024, 700)])
def test_values_without_a_scale(rows, K, N, kind):
    """A NaN or an infinity anywhere in a row makes its results NaN, and no other row's."""
    with Layer(23, N, K, act="relu") as layer:
        x = placed(values(24, rows, K), kind)
        x.t[1, K - 1], x.t[rows - 1, 0], x.t[2] = NAN, -float("inf"), 0.0
        y = torch.empty(rows, N, device="cuda")
        layer.forward(x.t, y)
        codes, scales = R.quantize(x.t)
        R.check(y, *layer.reference(codes, scales), "f32")
        assert torch.isnan(y).all(1).nonzero().flatten().tolist() == [1, rows - 1] and torch.isnan(y).any(1).sum() == 2


@pytest.mark.parametrize("act", ["none", "gelu", "silu", "relu"])
@pytest.mark.parametrize("rows", [16, 40000])
def test_activations_of_any_value(rows, act):
    """One input, one output, weight 1: the value is the row's scale, of either sign, from the smallest to infinity."""
    gen = torch.Generator().manual_seed(rows)
    v = 10.0 ** (76 * torch.rand(rows, generator=gen, dtype=torch.float64) - 38)
    v[::2] = 12 * torch.rand(len(v[::2]), generator=gen, dtype=torch.float64)
    v[:4] = torch.tensor([float("inf"), float("inf"), 3.4028234e38, 3.4028234e38])
    x, s = M.alloc_token_codes(rows, 1)
    x.copy_((1 - 2 * (torch.arange(rows) % 2)).view(-1, 1))
    s.copy_(v)
    w, one = M.alloc_token_codes(1, 1)
    w.fill_(1), one.fill_(1.0)
    y = torch.empty(rows, 1, device="cuda")
    h = M.mixaq_token_linear_create(w, one, None, act)
    M.mixaq_token_linear_forward(h, x, y, x_scales=s)
    torch.cuda.synchronize()
    M.mixaq_token_linear_destroy(h)
    v = s.double() * x[:, 0].double()
    assert float(y[0]) == float("inf") and float(y[1]) == (-float("inf") if act == "none" else 0.0)
    want, bound = R.activate(v[2:], torch.zeros_like(v[2:]), act)
    R.check(y[2:], want[:, None], bound[:, None], "f32")


def far(rows, cols, dtype, stride):
    """Rows whose offsets pass 2^32 bytes, in memory that is not filled."""
    return torch.empty(rows * stride, dtype=dtype, device="cuda").as_strided((rows, cols), (stride, 1))


@pytest.mark.parametrize("rows,stride", [(5, (1 << 30) + 16), (3000, 1 << 22), (40000, 1 << 17)])
def test_offsets_beyond_32_bits(rows, stride):
    K, N = 200, 333
    with Layer(31, N, K) as layer:
        q, s = far(rows, K, torch.int8, stride), torch.empty(rows, device="cuda")
        M.mixaq_token_quantize(values(32, rows, K), q, s)
        y = far(rows, N, torch.bfloat16, stride)
        layer.forward(q, y, s)
        codes, scales = R.quantize(values(32, rows, K))
        R.same(q, codes)
        R.same(y, R.linear_bits(codes, scales, *layer.matrix(), "bf16"))
        y.zero_()
        gather = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda")
        layer.grouped(q, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), y, s, gather=gather)
        R.same(y.flip(0), R.linear_bits(codes, scales, *layer.matrix(), "bf16"))


# ---------------------------------------------------------------- rows sorted by expert
def counts_of(seed, experts, rows, empty=()):
    share = torch.rand(experts, generator=torch.Generator().manual_seed(seed)) ** 2
    for e in empty:
        share[e] = 0.0
    n = (share / share.sum() * rows).int()
    n[int(share.argmax())] += rows - int(n.sum())
    return n.tolist()


def offsets_of(counts, first=0):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]) + first, dtype=torch.int32, device="cuda")


def check_sorted(layer, codes, scales, counts, first, y, kind, gather=None, weights=None):
    """Rows of y that no expert has hold the pattern."""
    at = first
    for e, n in enumerate(counts):
        if not n:
            continue
        rows = torch.arange(at, at + n, device="cuda")
        src = rows if gather is None else gather[at:at + n].long()
        known = (src >= 0) & (src < codes.shape[0])
        want, bound = layer.reference(codes[src[known]], scales[src[known]], e, None if weights is None else weights[rows[known]])
        R.check(y.t[rows[known]], want, bound, kind)
        assert bool((y.buffer[rows[~known]] == FILL).all())
        at += n
    assert bool((y.buffer[:first] == FILL).all() and (y.buffer[at:] == FILL).all())
    assert y.untouched()


@pytest.mark.parametrize("act,kind", [("none", "bf16"), ("silu", "f32"), ("gelu", "f16")])
@pytest.mark.parametrize("experts,rows,K,N,empty", S.SORTED)
def test_sorted_rows(experts, rows, K, N, empty, act, kind):
    counts, first, spare = counts_of(experts + rows, experts, rows, empty), 3, 130
    total = first + rows + spare
    with Layer(rows + K, N, K, experts, act) as layer:
        x = placed(values(rows, total, K), "i8", 0, 16)
        y = Room(total, N, kind, 0, 1)
        layer.grouped(x.t, offsets_of(counts, first), y.t, x.scales)
        check_sorted(layer, x.t, x.scales, counts, first, y, kind)


@pytest.mark.parametrize("x_kind", ["f32", "bf16", "i8"])
@pytest.mark.parametrize("experts,tokens,choices,K,N", [(8, 1, 2, 300, 100), (32, 8, 2, 1024, 256), (6, 17, 3, 130, 200), (16, 600, 2, 384, 300), (4, 3000, 2, 200, 500), (4, 20, 100, 64, 64)])
def test_gathered_and_weighted(experts, tokens, choices, K, N, x_kind):
    """Every token to several experts, some rows to none of the tokens: such rows keep what they held."""
    rows = tokens * choices
    counts = counts_of(experts * tokens, experts, rows, (1,))
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    gather = torch.randint(0, tokens, (rows + 50,), generator=gen, device="cuda", dtype=torch.int32)
    gather[::7] = -1
    gather[3::11] = tokens
    gather[5::13] = 2**31 - 1
    weights = torch.randn(rows + 50, generator=gen, device="cuda")
    with Layer(rows + K, N, K, experts, "silu") as layer:
        x = placed(values(rows, tokens, K), x_kind)
        codes, scales = (x.t, x.scales) if x_kind == "i8" else R.quantize(x.t)
        y = Room(rows + 50, N, "f32", 0, 1)
        layer.grouped(x.t, offsets_of(counts), y.t, x.scales, gather=gather, row_weights=weights)
        check_sorted(layer, codes, scales, counts, 0, y, "f32", gather, weights)


@pytest.mark.parametrize("x_kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("before", [0, 3])
@pytest.mark.parametrize("rows,K,N", [(1, 1, 1), (33, 7, 130), (33, 8, 40), (64, 9, 64), (5, 1017, 65), (64, 1024, 300), (64, 1025, 300), (65, 1024, 100)])
def test_few_sorted_rows_of_values_are_their_codes(rows, K, N, before, x_kind):
    """On both sides of where values are quantized on their way in; most rows to one expert, more than a tile of them."""
    counts = [1, 0, rows - 1, 0, 0, 0]
    gen = torch.Generator(device="cuda").manual_seed(rows)
    gather = torch.randint(0, rows, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    gather[3::11] = -1
    with Layer(rows + K, N, K, 6, "silu") as layer:
        x = placed(values(rows, rows, K), x_kind, before, 0)
        q = placed(values(rows, rows, K), "i8")
        codes, scales = R.quantize(x.t)
        q.t.copy_(codes)
        a, b = Room(rows, N, "f32"), Room(rows, N, "f32")
        if S.inside(rows, K, N, 6):
            M.mixaq_token_linear_forward_grouped(layer.h, x.t, offsets_of(counts), a.t, gather=gather)        # without a workspace
        else:
            layer.grouped(x.t, offsets_of(counts), a.t, gather=gather)
        layer.grouped(q.t, offsets_of(counts), b.t, scales, gather=gather)
        R.same(a.t, b.t)
        check_sorted(layer, codes, scales, counts, 0, a, "f32", gather)
        assert x.untouched()


@pytest.mark.parametrize("rows", [10, 3000])
def test_offsets_that_are_no_offsets(rows):
    """Beyond the rows they are cut off; falling ones leave rows undefined, and nothing outside the rows is read or written."""
    with Layer(41, 130, 100, 4) as layer:
        x = placed(values(42, rows, 100), "i8")
        y = Room(rows, 130, "f32", 0, 1)
        layer.grouped(x.t, torch.tensor([-7, 2, 2, 5, 2**31 - 1], dtype=torch.int32, device="cuda"), y.t, x.scales)
        check_sorted(layer, x.t, x.scales, [2, 0, 3, rows - 5], 0, y, "f32")
        for bad in ([5, 3, 9, -2**31, 2**31 - 1], [2**31 - 1] * 5, [-2**31] * 5, [rows, 0, rows, 0, rows]):
            y = Room(rows, 130, "f32", 0, 1)
            layer.grouped(x.t, torch.tensor(bad, dtype=torch.int32, device="cuda"), y.t, x.scales)
            torch.cuda.synchronize()
            assert y.untouched()


def test_rows_without_a_scale_stay_among_themselves():
    counts = [40, 0, 300, 7]
    with Layer(51, 200, 300, 4) as layer:
        v = values(52, 347, 300)
        x = placed(v, "bf16")
        x.t[5, 7], x.t[100, 0], x.t[346, 299] = NAN, float("inf"), NAN
        y = Room(347, 200, "f32")
        layer.grouped(x.t, offsets_of(counts), y.t)
        codes, scales = R.quantize(x.t)
        check_sorted(layer, codes, scales, counts, 0, y, "f32")
        assert torch.isnan(y.t).any(1).nonzero().flatten().tolist() == [5, 100, 346]


# ---------------------------------------------------------------- calls
def test_layer_refuses():
    with Layer(61, 40, 100, experts=2) as two, Layer(62, 40, 100) as one, Layer(62, 5000, 100) as wide:       # (the wide one quantizes values in a launch of its own)
        z = torch.empty(70, 5000, device="cuda")
        x, s, y = placed(values(63, 70, 100), "bf16"), placed(values(63, 70, 100), "i8"), Room(70, 40, "f32")
        off = offsets_of([30, 40])
        ws = M.alloc_token_linear_workspace(one.h, 70, torch.bfloat16)

        def refused(code, words, call):
            with pytest.raises(M.MixaqError) as e:
                call()
            assert e.value.code == code and words in str(e.value)

        refused(-2, "sorted by expert", lambda: M.mixaq_token_linear_forward(two.h, s.t, y.t, x_scales=s.scales))
        for call in (lambda w: M.mixaq_token_linear_forward_grouped(two.h, x.t, off, y.t, workspace=w), lambda w: M.mixaq_token_linear_forward(wide.h, x.t, z, workspace=w)):
            refused(-1, "workspace is NULL", lambda: call(None))
            refused(-4, "needed", lambda: call(ws[:-1]))
            refused(-4, "256-byte", lambda: call(torch.cat([ws, ws])[16:]))
        refused(-2, "without a list", lambda: two.grouped(s.t[:60], off, y.t, s.scales[:60]))
        codes, vals, out = M._token_rows(s.t, "x", 0, s.scales), M._rows(x.t, "x", 0), lambda at: M.Rows(at, 40, 0, None, 0)
        plain = lambda a, b, w=None, n=0: M._check(M.load().mixaq_token_linear_forward(one.h, a, 70, b, w, n, None))
        grouped = lambda b, o=off.data_ptr(), g=None, rw=None, x_=codes, w=None, n=0: \
            M._check(M.load().mixaq_token_linear_forward_grouped(two.h, x_, 70, o, g, rw, b, 70, w, n, None))
        Y, size, end = y.t.data_ptr(), 70 * 160, 69 * 112 + 100
        refused(-1, "offsets", lambda: grouped(out(Y), None))
        refused(-2, "x and y overlap", lambda: plain(codes, out(s.t.data_ptr() + end // 4 * 4 - 4)))
        refused(-2, "x and y overlap", lambda: plain(codes, out(s.scales.data_ptr() + 69 * 4)))
        for name, where in (("offsets", "o"), ("gather", "g"), ("row_weights", "rw")):
            refused(-2, "y and %s" % name, lambda: grouped(out(Y), **{where: Y + size - 4}))
            refused(-2, "%s is not aligned" % name, lambda: grouped(out(Y), **{where: off.data_ptr() + 2}))
            refused(-2, "workspace and %s" % name, lambda: grouped(out(Y), **{where: ws.data_ptr() + 256}, x_=vals, w=ws.data_ptr(), n=ws.numel()))
        refused(-2, "the workspace overlaps", lambda: grouped(out(ws.data_ptr() + 256), x_=vals, w=ws.data_ptr(), n=ws.numel()))
        refused(-2, "must be values", lambda: plain(vals, codes, ws.data_ptr(), ws.numel()))
        torch.cuda.synchronize()
        assert bool((y.buffer == FILL).all())
        # nothing to do
        M.mixaq_token_linear_forward(one.h, s.t[:0], y.t[:0], x_scales=s.scales[:0])
        two.grouped(s.t[:0], off, y.t, s.scales[:0], gather=torch.zeros(70, dtype=torch.int32, device="cuda"))
        two.grouped(s.t, off, y.t[:0], s.scales)
        torch.cuda.synchronize()
        assert bool((y.buffer == FILL).all())


def test_more_tiles_than_a_launch_holds_are_refused():
    rows, N = 1 << 30, 65536
    w, s_w = M.alloc_token_codes(N, 1)
    s_w.fill_(1.0)
    h = M.mixaq_token_linear_create(w, s_w)
    far_x, far_y = M.Rows(1 << 56, 16, 4, 1 << 57, 0), M.Rows(1 << 58, N, 2, None, 0)        # addresses that no call may touch
    assert M.load().mixaq_token_linear_forward(h, far_x, rows, far_y, None, 0, None) == -2 and b"too many" in M.load().mixaq_last_error()
    torch.cuda.synchronize()
    M.mixaq_token_linear_destroy(h)


def ffn(seed, C, hidden, experts):
    return Layer(seed, hidden, C, experts, "silu"), Layer(seed + 10, C, hidden, experts, "none")


@pytest.mark.parametrize("tokens,C,hidden,experts", [(8, 256, 512, 16), (2000, 96, 384, 8)])
def test_experts_captured_and_shared_out_anew(tokens, C, hidden, experts):
    """An expert FFN in a graph: the lists change between replays, with eager work beside them; every replay gives the eager call's bits."""
    rows, choices = 2 * tokens, 2
    fc1, fc2 = ffn(71, C, hidden, experts)
    with fc1, fc2:
        x = torch.empty(tokens, C, dtype=torch.bfloat16, device="cuda")
        off, gather, weights = torch.zeros(experts + 1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda")
        hid, out = (torch.zeros(rows, n, dtype=torch.bfloat16, device="cuda") for n in (hidden, C))
        ws = [M.alloc_token_linear_workspace(l.h, n, torch.bfloat16) for l, n in ((fc1, tokens), (fc2, rows))]

        def chain(h, o, work):
            M.mixaq_token_linear_forward_grouped(fc1.h, x, off, h, gather=gather, workspace=work[0])
            M.mixaq_token_linear_forward_grouped(fc2.h, h, off, o, row_weights=weights, workspace=work[1])

        def share_out(seed):
            gen = torch.Generator(device="cuda").manual_seed(seed)
            chosen = torch.rand(tokens, experts, generator=gen, device="cuda").topk(choices, 1).indices.flatten() % (experts - seed % 3)
            order = chosen.sort(stable=True).indices
            gather.copy_(order // choices)
            weights.copy_(torch.rand(rows, generator=gen, device="cuda"))
            off[1:] = torch.bincount(chosen, minlength=experts).cumsum(0)
            x.copy_(values(seed, tokens, C))

        share_out(1)
        chain(hid, out, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            chain(hid, out, ws)
        for seed in (2, 3, 4, 5):
            share_out(seed)
            h2, o2 = torch.zeros_like(hid), torch.zeros_like(out)
            chain(h2, o2, [None if w is None else torch.empty_like(w) for w in ws])
            hid.zero_(), out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            R.same(hid, h2)
            R.same(out, o2)
            graph.replay()
            R.same(out, o2)
            codes, scales = R.quantize(x)
            y = Room(rows, hidden, "bf16")
            y.t.copy_(hid)
            check_sorted(fc1, codes, scales, (off[1:] - off[:-1]).tolist(), 0, y, "bf16", gather)


def test_one_layer_on_two_streams_at_once():
    with Layer(81, 512, 384, act="gelu") as layer:
        streams = [torch.cuda.Stream() for _ in range(2)]
        x = [values(82 + i, 3000, 384).bfloat16() for i in range(2)]
        y = [torch.empty(3000, 512, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        ws = [M.alloc_token_linear_workspace(layer.h, 3000, torch.bfloat16) for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(5):
            for i in range(2):
                M.mixaq_token_linear_forward(layer.h, x[i], y[i], workspace=ws[i], stream=streams[i])
        torch.cuda.synchronize()
        for i in range(2):
            codes, scales = R.quantize(x[i])
            R.check(y[i], *layer.reference(codes, scales), "bf16")


def test_growing_rows_in_one_workspace():
    with Layer(91, 100, 300) as layer:
        ws = M.alloc_token_linear_workspace(layer.h, 2000, torch.float32)
        for rows in (1, 16, 17, 100, 2000, 3):
            x, y = values(rows, rows, 300), torch.empty(rows, 100, device="cuda")
            M.mixaq_token_linear_forward(layer.h, x, y, workspace=ws)
            R.same(y, R.linear_bits(*R.quantize(x), *layer.matrix(), "f32"))
