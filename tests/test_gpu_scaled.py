"""The 8-bit float linear layers and the norms between them on the GPU against 64-bit references, at the sizes, types, strides and values
where they can go wrong."""
import numpy as np
import pytest
import torch

import scaled_ref as R

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2507_19131_amd import binding as M

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
FILL = 0x5A                                                     # what unwritten bytes hold


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def values(seed, rows, cols):
    return normal(seed, rows, cols) * torch.exp(0.5 * normal(seed + 1, cols)) * torch.where(torch.arange(cols) % 37 == 5, 12.0, 1.0)


def as64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def bytes_of(codes):
    return codes.view(torch.uint8).cpu().numpy()


class Room:
    """A matrix inside a larger buffer: `before` columns in front of it, `after` columns and a row behind it, all filled with a pattern."""

    def __init__(self, rows, cols, kind, before=0, after=0, block_rows=1):
        es = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}[kind]
        width = before + cols + after
        if kind == "e4m3":
            width = -(-width // 16) * 16
        self.buffer = torch.full((rows + 1, width * es), FILL, dtype=torch.uint8, device="cuda")
        self.t = self.buffer.view(TYPES[kind])[:rows, before:before + cols]
        self.columns = (before * es, (before + cols) * es)
        self.scales = torch.full((R.blocks(cols), -(-rows // block_rows)), -1.0, device="cuda") if kind == "e4m3" else None

    def untouched(self):
        b = self.buffer.cpu()
        rows = self.t.shape[0]
        return bool((b[rows:] == FILL).all() and (b[:, :self.columns[0]] == FILL).all() and (b[:, self.columns[1]:] == FILL).all())


def placed(v, kind, before=0, after=0):
    room = Room(v.shape[0], v.shape[1], kind, before, after)
    room.t.copy_(v.to(TYPES[kind]))
    return room


def quantized(v, block_rows=1):
    """Reference codes of values, in GPU memory, with a pattern between the rows."""
    v = v.float()
    codes, scales = R.quantize(v.numpy(), block_rows)
    room = Room(v.shape[0], v.shape[1], "e4m3", 0, 0, block_rows)
    room.t.view(torch.uint8).copy_(torch.from_numpy(codes))
    room.scales.copy_(torch.from_numpy(scales.astype(np.float32)))
    return room, R.dequantize(codes, scales, block_rows)


# ---------------------------------------------------------------- quantizer
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,block_rows,before,after", [
    (1, 1, 1, 0, 0), (1, 128, 1, 0, 0), (49, 96, 1, 0, 0), (17, 129, 1, 1, 2), (130, 257, 1, 3, 5), (33, 1000, 1, 0, 8), (5, 4099, 1, 7, 0),
    (1, 1, 128, 0, 0), (128, 128, 128, 0, 0), (129, 100, 128, 0, 0), (300, 401, 128, 1, 1), (64, 1024, 128, 0, 0)])
def test_codes_are_the_references(kind, rows, cols, block_rows, before, after):
    x = placed(values(rows + cols, rows, cols), kind, before, after)
    q = Room(rows, cols, "e4m3", 16, 16 + before, block_rows)
    M.mixaq_scaled_quantize(x.t, q.t, q.scales, block_rows)
    codes, scales = R.quantize(as64(x.t).astype(np.float32), block_rows)
    assert np.array_equal(as64(q.scales), scales)
    assert np.array_equal(bytes_of(q.t), codes)
    assert q.untouched()


@pytest.mark.parametrize("block_rows", [1, 128])
def test_blocks_of_special_values(block_rows):
    inf, nan = float("inf"), float("nan")
    x = values(7, 11, 8 * 128 - 5)
    x[:, 128:256] = 0.0
    x[:, 256:384] *= 1e-42                                      # below the normal numbers
    x[0, 300] = -0.0
    x[3, 384 + 127] = inf
    x[4, 512] = nan
    x[4, 513] = -inf
    x[:, 640:768] = 3.4028234e38
    x[:, 768:896] = 2.0 ** -126
    x = x.cuda()
    q = Room(11, x.shape[1], "e4m3", 0, 0, block_rows)
    M.mixaq_scaled_quantize(x, q.t, q.scales, block_rows)
    codes, scales = R.quantize(x.cpu().numpy(), block_rows)
    assert np.array_equal(as64(q.scales), scales, equal_nan=True)
    assert np.array_equal(bytes_of(q.t), codes)


def test_a_single_value_per_row_far_apart():
    """Rows far apart in memory: offsets beyond 2^31 bytes and beyond 2^31 values."""
    stride = (1 << 30) + 16
    buffer = torch.empty(3 * stride, dtype=torch.float16, device="cuda")
    x = buffer.as_strided((3, 40), (stride, 1))
    x.copy_(values(3, 3, 40))
    out = torch.empty(3 * stride, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).as_strided((3, 40), (stride, 1))
    scales = torch.empty((1, 3), device="cuda")
    M.mixaq_scaled_quantize(x, out, scales)
    codes, want = R.quantize(as64(x).astype(np.float32))
    assert np.array_equal(as64(scales), want) and np.array_equal(bytes_of(out), codes)
    w, ww = quantized(normal(5, 24, 40), 128)
    h = M.mixaq_scaled_linear_create(w.t, w.scales)
    y = buffer.as_strided((3, 24), (stride, 1), 1 << 20)
    M.mixaq_scaled_linear_forward(h, out, y, x_scales=scales)
    M.mixaq_scaled_linear_destroy(h)
    want, bound = R.linear(R.dequantize(codes, want), ww, None, False, "f16")
    assert np.all(np.abs(as64(y) - want) <= R.allowed(want, bound, "f16"))


def far_rows(rows, cols, kind, stride):
    """Rows whose offsets pass 2^31 bytes and values, in memory that is not filled."""
    es = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}[kind]
    return torch.empty(rows * stride * es, dtype=torch.uint8, device="cuda").view(TYPES[kind]).as_strided((rows, cols), (stride, 1))


@pytest.mark.parametrize("K", [128, 257])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_many_rows_beyond_32_bit_offsets(K, kind):
    """Both tiled kernels, of either kind of sums; compared on rows from everywhere."""
    rows, N = 40000, 512
    with Layer(90, N, K) as layer:
        v = values(91, 2000, K).repeat(20, 1)
        x, scales = far_rows(rows, K, "e4m3", 65552), torch.empty((R.blocks(K), rows), device="cuda")
        M.mixaq_scaled_quantize(v.cuda(), x, scales)
        y = far_rows(rows, N, kind, 65536)
        ys = torch.empty((4, rows), device="cuda") if kind == "e4m3" else None
        M.mixaq_scaled_linear_forward(layer.h, x, y, x_scales=scales, y_scales=ys)
        at = torch.tensor([0, 1, 255, 256, 20000, 32767, 32768, 32769, 36000, 39998, 39999])
        codes, s64 = R.quantize(v[at].numpy())
        assert np.array_equal(as64(scales[:, at.cuda()]), s64)
        room = Room(len(at), N, kind)
        room.t.copy_(torch.stack([y[int(i)] for i in at]) if kind != "e4m3" else torch.stack([y[int(i)].view(torch.uint8) for i in at]).view(torch.float8_e4m3fn))
        if kind == "e4m3":
            room.scales.copy_(ys[:, at.cuda()])
        check_result(room, *layer.reference(R.dequantize(codes, s64), kind), kind)


def test_norms_of_many_rows_beyond_32_bit_offsets():
    rows, C = 40000, 96
    x, out = far_rows(rows, C, "bf16", 65536), far_rows(rows, C, "bf16", 65536)
    v = values(92, rows, C).bfloat16()
    x.copy_(v.cuda())
    M.mixaq_residual_norm(M.make_residual_norm(C), x, None, None, out)
    want, bound = R.norm(as64(v), "layer", float(np.float32(1e-5)), None, None, np.zeros((rows, C)))
    assert np.all(np.abs(as64(out) - want) <= R.allowed(want, bound, "bf16"))


# ---------------------------------------------------------------- linear layer
class Layer:
    def __init__(self, seed, N, K, bias=True, activation="none", w=None):
        v = normal(seed, N, K) / np.sqrt(K) if w is None else w
        self.w, self.w64 = quantized(v, 128)
        self.bias = normal(seed + 1, N).cuda() if bias else None
        self.h = M.mixaq_scaled_linear_create(self.w.t, self.w.scales, self.bias, activation)
        self.bias64, self.gelu = as64(self.bias) if bias else None, activation == "gelu"
        self.w.buffer.fill_(0x7F)                               # the handle keeps nothing of the caller's
        self.w.scales.fill_(float("nan"))
        if bias:
            self.bias.fill_(float("nan"))

    def __enter__(self):
        return self

    def __exit__(self, *a):
        M.mixaq_scaled_linear_destroy(self.h)

    def run(self, x, y, stream=None):
        ws = M.alloc_linear_workspace(self.h, x.t.shape[0], x.t.dtype, y.t.dtype)
        M.mixaq_scaled_linear_forward(self.h, x.t, y.t, x_scales=x.scales, y_scales=y.scales, workspace=ws, stream=stream)
        return ws

    def reference(self, x64, kind):
        return R.linear(x64, self.w64, self.bias64, self.gelu, kind)


def check_result(y, want, bound, kind):
    if kind == "e4m3":
        R.check_codes(bytes_of(y.t), as64(y.scales), want, bound)
    else:
        worst = float((np.abs(as64(y.t) - want) / R.allowed(want, bound, kind)).max())
        assert worst <= 1.0, worst


SIZES = [  # rows, K, N: one of everything, ends inside tiles, blocks and 16-byte chunks, each kernel's range and both sides of it
    (1, 1, 1), (1, 128, 128), (1, 1024, 512), (2, 96, 96), (3, 130, 40), (15, 1000, 333), (16, 384, 1536), (17, 257, 129), (31, 2048, 64),
    (33, 512, 200), (49, 768, 1000), (64, 129, 257), (65, 640, 72), (100, 4096, 136), (128, 128, 512), (129, 1536, 384), (200, 31, 1000),
    (257, 256, 256), (513, 1024, 1024), (1001, 1000, 333), (1024, 512, 2048), (2400, 384, 1536), (4704, 96, 384), (3000, 128, 512),
    (300, 4000, 600), (700, 1500, 700), (3001, 200, 600), (6200, 300, 2000), (12300, 520, 1000)]


@pytest.mark.parametrize("x_kind,y_kind", [("e4m3", "bf16"), ("e4m3", "e4m3"), ("e4m3", "f32"), ("bf16", "f16"), ("f32", "f32"), ("f16", "e4m3")])
@pytest.mark.parametrize("rows,K,N", SIZES)
def test_layer(rows, K, N, x_kind, y_kind):
    activation = "gelu" if (rows + K + N) % 2 else "none"
    with Layer(rows + K + N, N, K, bias=rows % 3 != 0, activation=activation) as layer:
        v = values(rows * 3 + K, rows, K)
        if x_kind == "e4m3":
            x, x64 = quantized(v)
        else:
            x = placed(v, x_kind, 1, 2)
            x64 = R.dequantize(*R.quantize(as64(x.t).astype(np.float32)))
        y = Room(rows, N, y_kind, 16, 3)
        layer.run(x, y)
        check_result(y, *layer.reference(x64, y_kind), y_kind)
        assert y.untouched()


@pytest.mark.parametrize("rows,K,N", [(1, 1024, 512), (40, 384, 200), (70, 200, 384), (300, 512, 300), (1, 4200, 64), (900, 300, 500), (300, 4000, 600), (2000, 256, 640), (3001, 200, 600), (6200, 300, 2000)])
@pytest.mark.parametrize("activation", ["none", "gelu"])
def test_values_and_codes_are_two_forms_of_one_call(rows, K, N, activation):
    """Values in: the result of quantizing them first.  Codes out: the 32-bit result quantized."""
    with Layer(5, N, K, activation=activation) as layer:
        x = placed(values(9, rows, K), "bf16")
        xq = Room(rows, K, "e4m3")
        M.mixaq_scaled_quantize(x.t, xq.t, xq.scales)
        a, b = Room(rows, N, "f32"), Room(rows, N, "f32")
        layer.run(x, a)
        layer.run(xq, b)
        assert torch.equal(a.t, b.t)
        q, direct = Room(rows, N, "e4m3"), Room(rows, N, "e4m3")
        M.mixaq_scaled_quantize(b.t, q.t, q.scales)
        layer.run(xq, direct)
        assert torch.equal(q.scales, direct.scales) and np.array_equal(bytes_of(q.t), bytes_of(direct.t))
        half = [Room(rows, N, "f16") for _ in range(2)]
        layer.run(x, half[0])
        layer.run(xq, half[1])
        assert torch.equal(half[0].t, half[1].t)


@pytest.mark.parametrize("rows", [3, 50, 300, 4000, 20000, 30000, 50000])
def test_a_row_depends_on_nothing_but_itself(rows):
    """A NaN, an infinity or a huge row changes no other row, and the bytes behind a row's columns change nothing."""
    K, N = 300, 200
    with Layer(21, N, K) as layer:
        v = values(22, rows, K)
        x, _ = quantized(v)
        v[1, 299], v[2, 0] = float("nan"), float("inf")
        z, _ = quantized(v)
        z.buffer[:, K:] = 0x7F                                  # NaN codes
        keep = [r for r in range(rows) if r not in (1, 2)]
        for kind in ("f32", "bf16"):                            # both kinds of sums
            a, b = Room(rows, N, kind), Room(rows, N, kind)
            layer.run(x, a)
            layer.run(z, b)
            assert torch.isnan(b.t[1:3]).all()
            assert torch.equal(a.t[keep], b.t[keep])
        c = Room(rows, N, "e4m3")
        layer.run(z, c)
        assert torch.isnan(c.scales[:, 1:3]).all() and (bytes_of(c.t)[1:3] & 0x7F == 0x7F).all() and not torch.isnan(c.scales[:, keep]).any()


def test_scales_at_both_ends_of_their_range():
    for size, back in ((1e30, 1e-30), (1e-30, 1e30), (1.0, 1e-36)):
        v, w = values(31, 20, 200) * size, normal(32, 140, 200) * back
        with Layer(0, 140, 200, bias=False, w=w) as layer:
            x, x64 = quantized(v)
            y = Room(20, 140, "f32")
            layer.run(x, y)
            want, bound = layer.reference(x64, "f32")
            check_result(y, want, bound, "f32")


def test_gelu_far_from_zero():
    """Products of one value with one weight are exact, so that the activation can be driven to any argument."""
    v = torch.linspace(-12.0, 12.0, 400)[:, None].repeat(1, 1)
    v[0], v[1], v[2] = -3e4, 3e4, 0.0
    with Layer(0, 16, 1, bias=False, activation="gelu", w=torch.ones(16, 1)) as layer:
        x, x64 = quantized(v)
        y = Room(400, 16, "f32")
        layer.run(x, y)
        want, bound = layer.reference(x64, "f32")
        check_result(y, want, bound, "f32")
        x.scales[0, 5], x.scales[0, 6] = float("inf"), float("nan")
        layer.run(x, y)
        assert torch.isinf(y.t[5]).all() or (y.t[5] == 0).all()          # the limit of its sign
        assert torch.isnan(y.t[6]).all()


def test_layer_refuses():
    with Layer(3, 100, 200) as layer:
        n = 10000                                               # (few rows need no workspace)
        x, y = placed(values(1, n, 200), "bf16"), Room(n, 100, "f32")
        ws = M.alloc_linear_workspace(layer.h, n, torch.bfloat16, torch.float32)
        assert ws.numel() and M.mixaq_scaled_linear_workspace_bytes(layer.h, 8, torch.bfloat16, torch.float32) == 0
        call = M.mixaq_scaled_linear_forward

        def refused(code, words, *a, **kw):
            with pytest.raises(M.MixaqError) as e:
                call(layer.h, *a, **kw)
            assert e.value.code == code and words in str(e.value), e.value

        refused(-1, "workspace is NULL", x.t, y.t)
        refused(-4, "needed", x.t, y.t, workspace=ws[:-1])
        refused(-4, "aligned", x.t, y.t, workspace=torch.empty(ws.numel() + 256, dtype=torch.uint8, device="cuda")[16:])
        refused(-2, "overlap", x.t, x.t[:, :100], workspace=ws)
        xq, yq = Room(n, 200, "e4m3"), Room(n, 100, "e4m3")
        refused(-2, "overlap", xq.t, yq.t, x_scales=xq.scales, y_scales=xq.scales[:1])           # scales written while they are read
        refused(-2, "workspace overlaps", x.t, yq.t, y_scales=ws.view(torch.float32)[:n].view(1, n), workspace=ws)
        large = torch.zeros(n * 512, dtype=torch.uint8, device="cuda")
        refused(-2, "workspace overlaps", large.view(torch.bfloat16)[:n * 200].view(n, 200), y.t, workspace=large)
        with pytest.raises(ValueError, match="do not fit"):
            call(layer.h, x.t[:, :199], y.t, workspace=ws)
        with pytest.raises(ValueError, match="scales"):
            call(layer.h, Room(n, 200, "e4m3").t, y.t, workspace=ws)
        with pytest.raises(ValueError, match="scales"):
            call(layer.h, x.t, y.t, x_scales=torch.ones((2, n), device="cuda"), workspace=ws)
        call(layer.h, x.t[:0], y.t[:0])                         # nothing to do
        wide = torch.zeros((n, 512), dtype=torch.bfloat16, device="cuda")
        call(layer.h, wide[:, :200], wide[:, 200:300], workspace=ws)     # columns of one matrix are no overlap


def test_weight_scales_in_a_wider_matrix():
    v = normal(8, 300, 300) / 17
    w, w64 = quantized(v, 128)
    wide = torch.full((3, 9), 7.0, device="cuda")
    wide[:, 2:5] = w.scales
    h = M.mixaq_scaled_linear_create(w.t, wide[:, 2:5])
    x, x64 = quantized(values(1, 33, 300))
    y = Room(33, 300, "f32")
    M.mixaq_scaled_linear_forward(h, x.t, y.t, x_scales=x.scales)
    M.mixaq_scaled_linear_destroy(h)
    check_result(y, *R.linear(x64, w64, None, False, "f32"), "f32")


# ---------------------------------------------------------------- norms
def vectors(seed, C, count=4):
    return [1.0 + 0.25 * normal(seed, C), 0.1 * normal(seed + 1, C), 1.0 + 0.25 * normal(seed + 2, C), 0.1 * normal(seed + 3, C)][:count]


def gate_of(seed, rows, span, C):
    g = 0.1 + 0.3 * normal(seed, -(-rows // span), C)
    return g, as64(g)[np.arange(rows) // span]


WIDTHS = [1, 2, 7, 8, 96, 127, 128, 129, 200, 256, 384, 385, 512, 513, 768, 1000, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 8192, 8193, 16384]


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("x_kind,branch_kind,out_kind,post,pre,span", [
    ("f32", "f32", "f32", "layer", "layer", 1000), ("bf16", "bf16", "bf16", "rms", "rms", 1), ("f16", "f32", "e4m3", "layer", "rms", 3),
    ("bf16", "f16", "e4m3", "none", "layer", None), ("f32", "bf16", "f16", "rms", "none", 2), ("bf16", "f32", "f32", "none", "rms", 5)])
def test_norms(C, x_kind, branch_kind, out_kind, post, pre, span):
    rows = 19 if C < 4000 else 5
    x, f = placed(values(C, rows, C), x_kind, 1, 2), placed(values(C + 9, rows, C) + 0.7, branch_kind, 3, 0)
    pg, pb, qg, qb = [v.cuda() for v in vectors(C + 3, C)]
    if post == "rms":
        pb = None
    if pre == "layer" and C % 2:
        qg = None                                               # a norm without gamma
    gate, gate64 = gate_of(C + 4, rows, span, C) if span else (None, None)
    norm = M.make_residual_norm(C, post, pre, 1e-5, 0.75, pg, pb, qg, qb, None if gate is None else gate.cuda(), span)
    y, out = Room(rows, C, x_kind, 2, 1), Room(rows, C, out_kind, 16, 5)
    M.mixaq_residual_norm(norm, x.t, f.t, y.t, out.t, out.scales)
    n64 = lambda v: None if v is None else as64(v)
    eps = float(np.float32(1e-5))
    (wy, by), (wo, bo) = R.residual_norm(as64(x.t), as64(f.t), 0.75, gate64, (post, eps, n64(pg), n64(pb)), (pre, eps, n64(qg), n64(qb)))
    assert np.all(np.abs(as64(y.t) - wy) <= R.allowed(wy, by, x_kind))
    check_result(out, wo, bo, out_kind)
    assert y.untouched() and out.untouched()


@pytest.mark.parametrize("C", [96, 700, 3000])
def test_first_and_last_norm_of_a_stream(C):
    """No branch: the norm in front of the first layer.  No out: the sum behind the last.  No y: the sum is not needed any more."""
    x, f = placed(values(1, 10, C), "bf16"), placed(values(2, 10, C), "bf16")
    first = M.make_residual_norm(C, "none", "layer")
    out = Room(10, C, "bf16")
    M.mixaq_residual_norm(first, x.t, None, None, out.t)
    want, bound = R.norm(as64(x.t), "layer", float(np.float32(1e-5)), None, None, np.zeros((10, C)))
    check_result(out, want, bound, "bf16")
    last = M.make_residual_norm(C, "layer", "none")
    y = Room(10, C, "bf16")
    M.mixaq_residual_norm(last, x.t, f.t, y.t)
    (want, bound), _ = R.residual_norm(as64(x.t), as64(f.t), 1.0, None, ("layer", float(np.float32(1e-5)), None, None), ("none", 1.0, None, None))
    check_result(y, want, bound, "bf16")


@pytest.mark.parametrize("C", [96, 300, 1000, 5000])
def test_in_place(C):
    """The residual stream and the branch may be overwritten by what replaces them."""
    norm = M.make_residual_norm(C, "layer", "rms", residual_scale=0.5)
    x, f = placed(values(1, 37, C), "bf16", 1, 0), placed(values(2, 37, C), "bf16", 0, 1)
    y, out = Room(37, C, "bf16"), Room(37, C, "bf16")
    M.mixaq_residual_norm(norm, x.t, f.t, y.t, out.t)
    M.mixaq_residual_norm(norm, x.t, f.t, x.t, f.t)
    assert torch.equal(x.t, y.t) and torch.equal(f.t, out.t) and x.untouched() and f.untouched()


def test_rows_without_spread_and_rows_with_nan():
    C = 300
    x = torch.zeros((6, C))
    x[1], x[2], x[3] = 1000.0, -3e38, 1e-30
    x[4] = values(3, 1, C)[0]
    x[5] = x[4]
    x[4, 17] = float("nan")
    norm = M.make_residual_norm(C, "none", "layer")
    out = torch.empty((6, C), device="cuda")
    M.mixaq_residual_norm(norm, x.cuda(), None, None, out)
    got = as64(out)
    assert np.all(got[0] == 0) and np.isnan(got[4]).all()
    # of equal values the mean is off by up to 76 U of them, which 1 / sqrt(eps) scales
    assert np.abs(got[1]).max() <= 76 * R.U * 1000 / np.sqrt(1e-5) * 1.01 and np.abs(got[3]).max() <= 1e-20
    want, bound = R.norm(as64(x[5:]), "layer", float(np.float32(1e-5)), None, None, np.zeros((1, C)))
    assert np.all(np.abs(got[5:] - want) <= bound)
    codes, scales = M.alloc_codes(6, C)
    M.mixaq_residual_norm(norm, x.cuda(), None, None, codes, scales)
    assert torch.isnan(scales[:, 4]).all() and not torch.isnan(scales[:, [0, 1, 3, 5]]).any()


def test_norm_refuses_too_few_gates():
    x = torch.zeros((10, 64), device="cuda")
    norm = M.make_residual_norm(64, "none", "layer", gate=torch.ones((3, 64), device="cuda"), rows_per_gate=3)
    with pytest.raises(ValueError, match="gate"):
        M.mixaq_residual_norm(norm, x, x.clone(), torch.empty_like(x), torch.empty_like(x))


# ---------------------------------------------------------------- together
class FeedForward:
    """norm -> codes -> FC1 + GELU -> codes -> FC2 -> norm behind the gate: the float FFN of a block."""

    def __init__(self, rows, C, hidden, kind):
        self.rows, self.kind = rows, kind
        self.fc1, self.fc2 = Layer(1, hidden, C, activation="gelu"), Layer(2, C, hidden)
        self.vec = [v.cuda() for v in vectors(5, C)]
        self.gate = (0.5 + 0.1 * normal(6, C)).cuda()
        self.first = M.make_residual_norm(C, "none", "layer", pre_gamma=self.vec[2], pre_beta=self.vec[3])
        self.last = M.make_residual_norm(C, "rms", "layer", post_gamma=self.vec[0], gate=self.gate)
        self.a, self.b, self.f = Room(rows, C, "e4m3"), Room(rows, hidden, "e4m3"), Room(rows, C, kind)
        self.y, self.out = Room(rows, C, kind), Room(rows, C, kind)

    def run(self, x, stream=None):
        M.mixaq_residual_norm(self.first, x, None, None, self.a.t, self.a.scales, stream=stream)
        M.mixaq_scaled_linear_forward(self.fc1.h, self.a.t, self.b.t, x_scales=self.a.scales, y_scales=self.b.scales, stream=stream)
        M.mixaq_scaled_linear_forward(self.fc2.h, self.b.t, self.f.t, x_scales=self.b.scales, stream=stream)
        M.mixaq_residual_norm(self.last, x, self.f.t, self.y.t, self.out.t, stream=stream)

    def check(self, x):
        """Every link against the reference of what the link before it left."""
        eps = float(np.float32(1e-5))
        v = [as64(t) for t in self.vec]
        want, bound = R.norm(as64(x), "layer", eps, v[2], v[3], np.zeros(x.shape))
        check_result(self.a, want, bound, "e4m3")
        check_result(self.b, *self.fc1.reference(R.dequantize(bytes_of(self.a.t), as64(self.a.scales)), "e4m3"), "e4m3")
        check_result(self.f, *self.fc2.reference(R.dequantize(bytes_of(self.b.t), as64(self.b.scales)), self.kind), self.kind)
        (wy, by), (wo, bo) = R.residual_norm(as64(x), as64(self.f.t), 1.0, as64(self.gate)[None], ("rms", eps, v[0], None), ("layer", eps, None, None))
        check_result(self.y, wy, by, self.kind)
        check_result(self.out, wo, bo, self.kind)

    def close(self):
        M.mixaq_scaled_linear_destroy(self.fc1.h)
        M.mixaq_scaled_linear_destroy(self.fc2.h)


@pytest.mark.parametrize("rows,C,hidden,kind", [(1, 1024, 4096, "bf16"), (49, 96, 384, "f32"), (333, 500, 1001, "f16"), (2401, 384, 1536, "bf16")])
def test_feed_forward(rows, C, hidden, kind):
    ffn = FeedForward(rows, C, hidden, kind)
    x = values(11, rows, C).to(TYPES[kind]).cuda()
    ffn.run(x)
    ffn.check(x)
    # against the same FFN in 64 bits without codes: two layers of codes, each half a step of e4m3 off at most per value, averaged over many
    f = R.gelu(R.norm(as64(x), "layer", 1e-5, as64(ffn.vec[2]), as64(ffn.vec[3]), np.zeros(x.shape))[0] @ ffn.fc1.w64.T + ffn.fc1.bias64)
    f = f @ ffn.fc2.w64.T + ffn.fc2.bias64
    off = np.linalg.norm(as64(ffn.f.t) - f) / np.linalg.norm(f)
    assert off <= 2 * R.HALF_STEP["e4m3"]
    ffn.close()


@pytest.mark.parametrize("rows,C,hidden", [(130, 384, 800), (3000, 256, 1024)])
def test_feed_forward_captured_and_on_streams(rows, C, hidden):
    """A captured run, replayed on new inputs among eager runs of another instance on other streams, gives the eager bits every time."""
    a, b = FeedForward(rows, C, hidden, "bf16"), FeedForward(rows, C, hidden, "bf16")
    xs = [values(40 + i, rows, C).bfloat16().cuda() for i in range(4)]
    x = xs[0].clone()
    eager = []
    for v in xs:
        b.run(v)
        eager.append((b.y.t.clone(), b.out.t.clone()))
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    a.run(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.run(x, stream=torch.cuda.current_stream())
    for i in (0, 1, 2, 3, 2, 0):
        x.copy_(xs[i])
        graph.replay()
        b.run(xs[(i + 1) % 4], stream=other)
        torch.cuda.synchronize()
        assert torch.equal(a.y.t, eager[i][0]) and torch.equal(a.out.t, eager[i][1])
        assert torch.equal(b.y.t, eager[(i + 1) % 4][0])
    a.close()
    b.close()


def test_one_layer_on_two_streams_at_once():
    """The handle is shared, the workspaces are not; every repetition gives the same bits."""
    with Layer(50, 640, 512, activation="gelu") as layer:
        x = [placed(values(60 + i, 2500 + 800 * i, 512), "bf16") for i in range(2)]
        want = [Room(v.t.shape[0], 640, "bf16") for v in x]
        for v, w in zip(x, want):
            layer.run(v, w)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        ws = [M.alloc_linear_workspace(layer.h, v.t.shape[0], torch.bfloat16, torch.bfloat16) for v in x]
        y = [Room(v.t.shape[0], 640, "bf16") for v in x]
        torch.cuda.synchronize()
        for _ in range(20):
            for i in range(2):
                M.mixaq_scaled_linear_forward(layer.h, x[i].t, y[i].t, workspace=ws[i], stream=streams[i])
        torch.cuda.synchronize()
        assert torch.equal(y[0].t, want[0].t) and torch.equal(y[1].t, want[1].t)


def test_larger_workspace_than_needed_and_growing_rows():
    with Layer(70, 300, 200) as layer:
        sizes = [M.mixaq_scaled_linear_workspace_bytes(layer.h, r, torch.float32, torch.float8_e4m3fn) for r in (0, 1, 5, 64, 65, 1000, 4000, 5000)]
        assert sizes == sorted(sizes)
        ws = torch.empty(sizes[-1], dtype=torch.uint8, device="cuda")
        assert sizes[-1] > 0
        for rows in (1, 5, 64, 65, 1000, 4000, 5000):            # what serves the most rows serves fewer
            x, y = placed(values(rows, rows, 200), "f32"), Room(rows, 300, "f32")
            M.mixaq_scaled_linear_forward(layer.h, x.t, y.t, workspace=ws)
            x64 = R.dequantize(*R.quantize(as64(x.t).astype(np.float32)))
            check_result(y, *layer.reference(x64, "f32"), "f32")
