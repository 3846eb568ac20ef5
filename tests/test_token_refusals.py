"""Calls of the int8 layers with a scale per token and of the group norm that are refused before any GPU call, and their 64-bit references against torch.
CPU only."""
import ctypes as C

import pytest
import torch

import token_ref as R
from paper_2507_19131_amd import binding as M
from test_scaled_refusals import calls  # noqa: F401 (a fixture: the binding with nothing called behind it)

NULL, SHAPE, WORKSPACE = -1, -2, -4
AT = 1 << 20                                              # addresses that no call may touch
X, Y, S, W, LIST = (AT + (i << 30) for i in range(5))


def values(data=X, stride=256, kind=2):
    return M.Rows(data, stride, kind, None, 0)


def codes(data=X, stride=256, scales=S):
    return M.Rows(data, stride, 4, scales, 0)


def refused(code, words, rc):
    assert rc == code and words in M.load().mixaq_last_error().decode(), (rc, M.load().mixaq_last_error())


# ---------------------------------------------------------------- quantizer
@pytest.mark.parametrize("code,words,x,rows,cols,q", [
    (SHAPE, "0 <= rows", values(), -1, 200, codes(Y)), (SHAPE, "0 <= rows", values(), 2**30 + 1, 200, codes(Y)), (SHAPE, "columns", values(), 3, 0, codes(Y)),
    (NULL, "x is NULL", values(None), 3, 200, codes(Y)), (SHAPE, "x must be values", codes(), 3, 200, codes(Y)), (SHAPE, "not int8", values(kind=3), 3, 200, codes(Y)),
    (SHAPE, "unknown type", values(kind=5), 3, 200, codes(Y)), (SHAPE, "stride", values(stride=199), 3, 200, codes(Y)), (SHAPE, "aligned", values(X + 1), 3, 200, codes(Y)),
    (NULL, "q is NULL", values(), 3, 200, codes(None)), (SHAPE, "q must be int8", values(), 3, 200, values(Y)), (NULL, "scales is NULL", values(), 3, 200, codes(Y, scales=None)),
    (SHAPE, "scales are not aligned", values(), 3, 200, codes(Y, scales=S + 2)), (SHAPE, "16 bytes", values(), 3, 200, codes(Y + 8)),
    (SHAPE, "16 bytes", values(), 3, 200, codes(Y, 200)), (SHAPE, "stride", values(), 3, 200, codes(Y, 192)), (SHAPE, "x and q overlap", values(), 3, 200, codes(X + 1024)),
    (SHAPE, "x and q overlap", values(), 3, 200, codes(Y, scales=X + 1420)), (SHAPE, "codes and scales", values(), 3, 200, codes(Y, scales=Y + 700))])
def test_quantizer_refuses(code, words, x, rows, cols, q):
    refused(code, words, M.load().mixaq_token_quantize(x, rows, cols, q, None))


@pytest.mark.parametrize("rows,cols", [(2**30, 3000), (2**26, 200), (2**23, 9000)])
def test_quantizer_refuses_more_than_a_launch_holds(rows, cols):
    """2^32 threads; whatever the form that the width asks for."""
    far = 1 << 54
    rc = M.load().mixaq_token_quantize(values(AT, 1 << 14), rows * 4 if rows * 4 <= 2**30 else rows, cols, codes(far, 1 << 14, far * 2), None)
    refused(SHAPE, "too many", rc)


# ---------------------------------------------------------------- layers
@pytest.mark.parametrize("code,words,desc,w,out", [
    (SHAPE, "outside", (0, 8, 1, 0), codes(), True), (SHAPE, "outside", (65537, 8, 1, 0), codes(stride=65552), True), (SHAPE, "outside", (8, 0, 1, 0), codes(), True),
    (SHAPE, "outside", (8, 65537, 1, 0), codes(), True), (SHAPE, "experts", (8, 8, 0, 0), codes(), True), (SHAPE, "experts", (8, 8, 4097, 0), codes(), True),
    (SHAPE, "2^24", (8, 65536, 257, 0), codes(), True), (SHAPE, "activation", (8, 8, 1, 4), codes(), True), (SHAPE, "activation", (8, 8, 1, -1), codes(), True),
    (SHAPE, "w must be int8", (8, 8, 1, 0), values(), True), (NULL, "w is NULL", (8, 8, 1, 0), codes(None), True), (NULL, "scales", (8, 8, 1, 0), codes(scales=None), True),
    (NULL, "out is NULL", (8, 8, 1, 0), codes(), False)])
def test_layers_that_are_not_made(code, words, desc, w, out):
    d, p, h = M.TokenLinearDesc(*desc), M.TokenLinearParams(w, None), C.c_void_p()
    refused(code, words, M.load().mixaq_token_linear_create(C.byref(d), C.byref(p), None, C.byref(h) if out else None))
    assert not h.value


def test_calls_without_a_layer():
    L, n = M.load(), C.c_size_t()
    refused(NULL, "layer", L.mixaq_token_linear_forward(None, values(), 3, values(Y), None, 0, None))
    refused(NULL, "layer", L.mixaq_token_linear_forward_grouped(None, values(), 3, LIST, None, None, values(Y), 3, None, 0, None))
    refused(NULL, "layer", L.mixaq_token_linear_workspace_bytes(None, 3, 0, C.byref(n)))
    assert L.mixaq_token_linear_destroy(None) == 0


# ---------------------------------------------------------------- group norm
def norm_call(desc=(96, 32, 10, 0, 1e-5), x=None, y=None, rows=20, ws=W, bytes_=1 << 20, gamma=None, beta=None, params=True):
    d, p = M.GroupNormDesc(*desc), M.GroupNormParams(gamma, beta)
    return M.load().mixaq_group_norm(C.byref(d), C.byref(p) if params else None, x or values(), y or values(Y), rows, ws, bytes_, None)


END = X + (19 * 256 + 96) * 2                             # behind x's last value
@pytest.mark.parametrize("code,words,kw", [
    (SHAPE, "C=", dict(desc=(0, 1, 10, 0, 1e-5))), (SHAPE, "C=", dict(desc=(8193, 1, 10, 0, 1e-5))), (SHAPE, "groups", dict(desc=(96, 0, 10, 0, 1e-5))),
    (SHAPE, "groups", dict(desc=(96, 36, 10, 0, 1e-5))), (SHAPE, "groups", dict(desc=(2048, 2048, 10, 0, 1e-5))), (SHAPE, "rows_per_image", dict(desc=(96, 32, 0, 0, 1e-5))),
    (SHAPE, "activation", dict(desc=(96, 32, 10, 4, 1e-5))), (SHAPE, "eps", dict(desc=(96, 32, 10, 0, 0.0))), (SHAPE, "eps", dict(desc=(96, 32, 10, 0, float("nan")))),
    (SHAPE, "eps", dict(desc=(96, 32, 10, 0, float("inf")))), (NULL, "params", dict(params=False)), (SHAPE, "whole images", dict(rows=25)),
    (SHAPE, "0 <= rows", dict(rows=-10)), (SHAPE, "x must be values", dict(x=codes())), (SHAPE, "not int8", dict(y=values(Y, kind=3))), (NULL, "x is NULL", dict(x=values(None))),
    (NULL, "y: scales", dict(y=codes(Y, scales=None))), (NULL, "workspace", dict(ws=None)), (WORKSPACE, "needed", dict(bytes_=100)), (WORKSPACE, "256", dict(ws=W + 128)),
    (SHAPE, "x and y overlap", dict(y=values(X + 2))), (SHAPE, "x and y overlap", dict(y=values(X, kind=1))), (SHAPE, "x and y overlap", dict(y=codes(Y, scales=END - 4))),
    (SHAPE, "workspace overlaps", dict(ws=X + 256)), (SHAPE, "workspace overlaps", dict(y=values(W + 512))), (SHAPE, "gamma overlaps", dict(gamma=Y + 100)),
    (SHAPE, "beta overlaps", dict(beta=W + 4)), (SHAPE, "gamma is not aligned", dict(gamma=LIST + 2)), (SHAPE, "gamma overlaps", dict(x=values(), y=values(), gamma=X))])
def test_norm_refuses(code, words, kw):
    refused(code, words, norm_call(**kw))


def test_norm_of_too_many_images():
    far = 1 << 54
    rc = norm_call((8, 1, 1, 0, 1e-5), values(AT, 8), values(far, 8), 2**30, far * 2, 1 << 60)
    refused(SHAPE, "too many", rc)


def test_nothing_to_do_is_no_error():
    assert M.load().mixaq_token_quantize(None, 0, 8, None, None) == 0
    assert norm_call(x=values(None), rows=0, ws=None, bytes_=0) == 0


# ---------------------------------------------------------------- the binding
def layer(K, N, experts=1):
    h = C.c_void_p(0)
    h.K, h.N, h.experts = K, N, experts
    return h


def room(rows, cols):
    return M.alloc_token_codes(rows, cols, device="cpu")


def test_binding_refuses_tensors_that_do_not_fit(calls):  # noqa: F811
    v, (q, s) = torch.zeros(5, 100), room(5, 100)
    i32 = lambda *a: torch.zeros(*a, dtype=torch.int32)
    y, e4m3 = torch.zeros(5, 8), torch.zeros((5, 100), dtype=torch.uint8).view(torch.float8_e4m3fn)
    grouped = lambda x=q, xs=s, offsets=i32(4), y=y, **kw: M.mixaq_token_linear_forward_grouped(layer(100, 8, 3), x, offsets, y, x_scales=xs, **kw)
    norm = M.make_group_norm(100, 4, 5)
    for words, call in (
            ("int8", lambda: M.mixaq_token_quantize(v, e4m3, s)), ("shape", lambda: M.mixaq_token_quantize(v, q[:4], s[:4])), ("scales must be", lambda: M.mixaq_token_quantize(v, q, s[:4])),
            ("scales must be", lambda: M.mixaq_token_quantize(v, q, s.double())), ("missing", lambda: M.mixaq_token_quantize(v, q, None)),
            ("2-D", lambda: M.mixaq_token_quantize(q, q, s)), ("adjacent", lambda: M.mixaq_token_quantize(torch.zeros(100, 5).t(), q, s)),
            ("side by side", lambda: M.mixaq_token_quantize(v, q, torch.zeros(10)[::2])),
            ("w must be int8", lambda: M.mixaq_token_linear_create(v, s)), ("no 2 matrices", lambda: M.mixaq_token_linear_create(q, s, experts=2)),
            ("bias must be", lambda: M.mixaq_token_linear_create(q, s, torch.zeros(4))), ("activation", lambda: M.mixaq_token_linear_create(q, s, activation="tanh")),
            ("do not fit", lambda: M.mixaq_token_linear_forward(layer(99, 8), v, y)), ("do not fit", lambda: M.mixaq_token_linear_forward(layer(100, 9), v, y)),
            ("rows, y", lambda: M.mixaq_token_linear_forward(layer(100, 8), v, y[:4])), ("not int8, but", lambda: M.mixaq_token_linear_forward(layer(100, 8), v, y, x_scales=s)),
            ("2-D tensor of", lambda: M.mixaq_token_linear_forward(layer(100, 8), v, room(5, 8)[0])), ("not float8", lambda: M.mixaq_token_linear_forward(layer(100, 8), e4m3, y)),
            ("missing", lambda: M.mixaq_token_linear_forward(layer(100, 8), q, y)), ("workspace must be contiguous", lambda: M.mixaq_token_linear_forward(layer(100, 8), v, y, workspace=y.t())),
            ("offsets", lambda: grouped(offsets=i32(3))), ("offsets", lambda: grouped(offsets=i32(4).long())), ("offsets", lambda: grouped(offsets=i32(8)[::2])),
            ("gather", lambda: grouped(gather=i32(4))), ("gather", lambda: grouped(gather=torch.zeros(5))), ("row_weights", lambda: grouped(row_weights=torch.zeros(5).half())),
            ("row_weights", lambda: grouped(row_weights=torch.zeros(6))), ("x must be of", lambda: M.mixaq_token_linear_workspace_bytes(layer(8, 8), 3, torch.float8_e4m3fn)),
            ("gamma", lambda: M.make_group_norm(100, 4, 5, gamma=torch.zeros(99))), ("activation", lambda: M.make_group_norm(100, 4, 5, activation="tanh")),
            ("channels", lambda: M.make_group_norm(2**32 + 8, 4, 5)), ("groups", lambda: M.make_group_norm(8, 2**32 + 4, 5)), ("rows_per_image", lambda: M.make_group_norm(8, 4, 2**32 + 1)),
            ("shape", lambda: M.mixaq_group_norm(norm, v, torch.zeros(4, 100))), ("shape", lambda: M.mixaq_group_norm(norm, v[:, :96], v[:, :96])),
            ("missing", lambda: M.mixaq_group_norm(norm, v, q))):
        with pytest.raises(ValueError, match=words):
            call()
    assert not calls
    grouped()
    grouped(v, None, gather=i32(5), row_weights=torch.zeros(5))
    M.mixaq_group_norm(norm, v, q, s)
    assert len(calls) == 3


@pytest.mark.parametrize("rows", [2**31, 2**32 + 3])
def test_more_rows_than_the_library_counts_are_refused(calls, rows):  # noqa: F811
    x, q, s = torch.zeros((1, 16)).expand(rows, 16), torch.zeros((1, 16), dtype=torch.int8).expand(rows, 16), torch.zeros(1).expand(rows)
    i32 = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: M.mixaq_token_quantize(x, q, s), lambda: M.mixaq_token_linear_forward(layer(16, 16), x, x), lambda: M.mixaq_token_linear_forward(layer(16, 16), q, x, x_scales=s),
                 lambda: M.mixaq_token_linear_forward_grouped(layer(16, 16), x[:5], i32.expand(2).contiguous(), x), lambda: M.mixaq_group_norm(M.make_group_norm(16, 1, 8), x, x),
                 lambda: M.mixaq_token_linear_workspace_bytes(layer(16, 16), rows, torch.float32), lambda: M.mixaq_group_norm_workspace_bytes(M.make_group_norm(16, 1, 8), rows)):
        with pytest.raises(ValueError, match="2\\^30 rows"):
            call()
    assert not calls


def test_codes_have_room_for_whole_16_bytes(calls):  # noqa: F811
    byte = lambda n: torch.zeros(n, dtype=torch.int8)
    y, s = torch.zeros((3, 8)), torch.ones(3)
    for x in (byte(100).view(1, 100), byte(111).view(1, 111)[:, :100], byte(2 * 112 + 100).as_strided((3, 100), (112, 1)), byte(116)[16:].view(1, 100)):
        with pytest.raises(ValueError, match="room"):
            M.mixaq_token_linear_forward(layer(100, 8), x, y[:len(x)], x_scales=s[:len(x)])
    assert not calls
    for x in (byte(112).view(1, 112)[:, :100], byte(3 * 112).as_strided((3, 100), (112, 1)), byte(100)[:0].view(0, 100)):
        M.mixaq_token_linear_forward(layer(100, 8), x, y[:len(x)], x_scales=s[:len(x)])
    assert len(calls) == 3


def test_a_norm_takes_rows_on_the_device_of_its_vectors(calls, monkeypatch):  # noqa: F811
    norms = M.make_group_norm(8, 2, 5, gamma=torch.ones(8)), M.make_group_norm(8, 2, 5, beta=torch.ones(8))
    monkeypatch.setattr(M, "_on_device", lambda t, name: 1)
    x = torch.zeros((5, 8))
    for norm in norms:
        with pytest.raises(ValueError, match="vectors"):
            M.mixaq_group_norm(norm, x, x)
    assert not calls


# ---------------------------------------------------------------- the references
def test_reference_norm_and_activations_are_torchs():
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(2 * 35, 24, generator=gen, dtype=torch.float64).float()
    gamma, beta = torch.randn(24, generator=gen), torch.randn(24, generator=gen)
    for act, f in (("none", lambda v: v), ("gelu", torch.nn.functional.gelu), ("silu", torch.nn.functional.silu), ("relu", torch.relu)):
        y, bound = R.group_norm(x, 2, 8, 1e-5, gamma, beta, act)
        want = f(torch.nn.functional.group_norm(x.double().view(2, 35, 24).transpose(1, 2), 8, gamma.double(), beta.double(), 1e-5)).transpose(1, 2).reshape(70, 24)
        assert torch.allclose(y, want, rtol=0, atol=1e-13) and bool((bound < 5e-6).all())


def test_reference_codes_hold_their_values_to_half_a_step():
    x = torch.randn(50, 77, generator=torch.Generator().manual_seed(5)) * 3
    codes, scales = R.quantize(x)
    assert bool((codes.abs().amax(1) == 127).all())
    assert bool(((codes.double() * scales.double()[:, None] - x.double()).abs() <= 0.5 * scales.double()[:, None] * (1 + 300 * R.U)).all())
    y, bound = R.linear(codes, scales, codes, scales, None, "none")
    assert bool(((R.linear_bits(codes, scales, codes, scales, None, "f32").double() - y).abs() <= bound).all())


def test_reference_sums_are_rounded_once():
    """A tie of the product that the bias, far below, takes to one side: against whole numbers in Python."""
    a, s, c = torch.tensor([3.0, 3.0, -5.0, 7.0, 1.0]), torch.tensor([1.0 + 2.0 ** -23] * 4 + [2.0 ** 100]), torch.tensor([2.0 ** -60, -2.0 ** -60, 2.0 ** -40, 0.1, 0.0])
    from fractions import Fraction
    got = R.fma(a.double(), s.double(), c.double())
    for i in range(5):
        exact = Fraction(float(a[i])) * Fraction(float(s[i])) + Fraction(float(c[i]))
        near = [torch.nextafter(got[i], torch.tensor(x)) for x in (float("inf"), -float("inf"))]
        assert all(abs(Fraction(float(got[i])) - exact) < abs(Fraction(float(n)) - exact) for n in near)
