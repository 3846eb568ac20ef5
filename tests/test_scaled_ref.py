"""The 64-bit reference of the 8-bit float layers against torch's own conversions, and what the entry points refuse before any GPU call.
CPU only."""
import ctypes as C

import numpy as np
import pytest
import torch

import scaled_ref as R
from paper_2507_19131_amd import binding as M

NULL, SHAPE, WORKSPACE = -1, -2, -4


def test_reference_codes_are_those_of_the_type():
    gen = np.random.default_rng(1)
    v = np.concatenate([gen.standard_normal(20000) * np.exp(gen.standard_normal(20000) * 3), R.POSITIVE, -R.POSITIVE,
                        (R.POSITIVE[1:] + R.POSITIVE[:-1]) / 2, [0.0, -0.0, 2.0 ** -10, 2.0 ** -11, 448.0]])
    v = np.clip(R.f32(v), -448, 448)
    t = torch.from_numpy(v.astype(np.float32)).to(torch.float8_e4m3fn)
    assert np.array_equal(t.view(torch.uint8).numpy(), R.nearest_code(v))
    decoded = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(decoded, R.DECODE, equal_nan=True)


def test_reference_quantizer_keeps_the_largest_value():
    x = np.random.default_rng(2).standard_normal((5, 300)).astype(np.float32)
    codes, scales = R.quantize(x)
    v = R.dequantize(codes, scales)
    at = np.abs(x[:, :128]).argmax(1)
    assert np.allclose(v[np.arange(5), at], x[np.arange(5), at], rtol=1e-6)
    assert np.abs(v - x).max() <= np.abs(x).max() * 2.0 ** -4


def test_reference_norm_is_torch_layer_norm():
    gen = np.random.default_rng(3)
    x, f, g, b = gen.standard_normal((4, 70)), gen.standard_normal((4, 70)), gen.standard_normal(70), gen.standard_normal(70)
    (y, _), (out, _) = R.residual_norm(x, f, 0.5, None, ("layer", 1e-5, g, b), ("rms", 1e-6, g, None))
    want = 0.5 * x + torch.nn.functional.layer_norm(torch.from_numpy(f), (70,), torch.from_numpy(g), torch.from_numpy(b), 1e-5).numpy()
    assert np.allclose(y, want, rtol=1e-12, atol=1e-12)
    assert np.allclose(out, want / np.sqrt((want ** 2).mean(1, keepdims=True) + 1e-6) * g, rtol=1e-12, atol=1e-12)


# ---------------------------------------------------------------- refusals: addresses that no call may touch
AT, FAR = 1 << 20, 1 << 30


def rows(data=AT, stride=256, kind=2, scales=None, scale_stride=0):
    return M.Rows(data, stride, kind, scales, scale_stride)


def codes(data=FAR, stride=256, scales=FAR + (1 << 24), scale_stride=64):
    return M.Rows(data, stride, 3, scales, scale_stride)


def refused(code, words, rc):
    assert rc == code, (rc, M.load().mixaq_last_error())
    assert words in M.load().mixaq_last_error().decode()


@pytest.mark.parametrize("code,words,x,n,cols,block,q", [
    (NULL, "x is NULL", None, 4, 200, 1, codes()),
    (NULL, "q is NULL", rows(), 4, 200, 1, codes(data=None)),
    (NULL, "scales is NULL", rows(), 4, 200, 1, codes(scales=None)),
    (SHAPE, "0 <= rows", rows(), -1, 200, 1, codes()),
    (SHAPE, "columns >= 1", rows(), 4, 0, 1, codes()),
    (SHAPE, "block_rows", rows(), 4, 200, 64, codes()),
    (SHAPE, "unknown type", rows(kind=4), 4, 200, 1, codes()),
    (SHAPE, "unknown type", rows(kind=-1), 4, 200, 1, codes()),
    (SHAPE, "x must be values", codes(data=AT), 4, 200, 1, codes()),
    (SHAPE, "q must be codes", rows(), 4, 200, 1, rows(data=FAR)),
    (SHAPE, "stride 199", rows(stride=199), 4, 200, 1, codes()),
    (SHAPE, "not aligned", rows(data=AT + 1), 4, 200, 1, codes()),
    (SHAPE, "multiples of 16", rows(), 4, 200, 1, codes(stride=200)),
    (SHAPE, "multiples of 16", rows(), 4, 200, 1, codes(data=FAR + 8)),
    (SHAPE, "scale_stride 63", rows(), 64, 200, 1, codes(scale_stride=63)),
    (SHAPE, "overlap", rows(), 4, 200, 1, codes(data=AT + 512)),
    (SHAPE, "overlap", rows(), 4, 200, 1, codes(scales=AT + 512)),
    (SHAPE, "codes and scales", rows(), 4, 200, 1, codes(scales=FAR + 512)),
    (SHAPE, "rows <= 2^30", rows(), 2**30 + 1, 200, 1, codes(scale_stride=2**31)),
    (SHAPE, "too many", rows(stride=65536), 2**30, 65536, 1, codes(data=1 << 60, stride=65536, scales=1 << 62, scale_stride=2**31)),
])
def test_quantizer_refuses(code, words, x, n, cols, block, q):
    refused(code, words, M.load().mixaq_scaled_quantize(x, n, cols, block, q, None))


def test_nothing_to_do_is_no_error():
    L = M.load()
    assert L.mixaq_scaled_quantize(None, 0, 200, 1, None, None) == 0
    d, p = M.ResidualNormDesc(200, 1, 1, 1, 1e-5, 1e-5, 1.0), M.ResidualNormParams()
    assert L.mixaq_residual_norm(C.byref(d), C.byref(p), None, rows(), rows(data=FAR), None, 0, None) == NULL     # no out for the norm
    d.pre_norm = 0
    assert L.mixaq_residual_norm(C.byref(d), C.byref(p), rows(data=None), rows(data=None), rows(data=None), None, 0, None) == 0


def norm_call(desc=None, x=None, branch=None, y=None, out=None, n=4, gate=None, **change):
    d = M.ResidualNormDesc(200, 1, 1, 4, 1e-5, 1e-5, 1.0)
    for k, v in change.items():
        setattr(d, k, v)
    p = M.ResidualNormParams(gate=gate)
    x = rows() if x is None else x
    branch = rows(data=AT + (1 << 16)) if branch is None else branch
    y = rows(data=FAR) if y is None else y
    out = rows(data=FAR + (1 << 16)) if out is None else out
    none = lambda v: None if v == "none" else v
    return M.load().mixaq_residual_norm(C.byref(d), C.byref(p), none(x), none(branch), none(y), none(out), n, None)


@pytest.mark.parametrize("code,words,kw", [
    (NULL, "x is NULL", dict(x=rows(data=None))),
    (NULL, "branch is NULL", dict(branch=rows(data=None))),
    (NULL, "both NULL", dict(y="none", out="none")),
    (NULL, "pre_norm without out", dict(out="none")),
    (NULL, "without branch", dict(branch="none")),
    (NULL, "without branch", dict(branch="none", post_norm=0, gate=AT)),
    (SHAPE, "C=0", dict(C=0)),
    (SHAPE, "C=16385", dict(C=16385)),
    (SHAPE, "0 <= rows", dict(n=-1)),
    (SHAPE, "rows <= 2^30", dict(n=2**30 + 1)),
    (SHAPE, "out and x overlap", dict(out=codes(scales=AT + 256))),
    (SHAPE, "y and out overlap", dict(out=codes(data=FAR + (1 << 20), scales=FAR + 256))),
    (SHAPE, "post_norm: unknown", dict(post_norm=3)),
    (SHAPE, "pre_norm: unknown", dict(pre_norm=-1)),
    (SHAPE, "post_norm: eps", dict(post_eps=0.0)),
    (SHAPE, "pre_norm: eps", dict(pre_eps=float("nan"))),
    (SHAPE, "rows_per_gate", dict(rows_per_gate=0, gate=AT)),
    (SHAPE, "x must be values", dict(x=codes(data=AT))),
    (SHAPE, "branch must be values", dict(branch=codes(data=AT))),
    (SHAPE, "type of x", dict(y=rows(data=FAR, kind=0))),
    (SHAPE, "out: stride", dict(out=rows(data=FAR, stride=100))),
    (SHAPE, "scale_stride", dict(out=codes(scale_stride=3))),
    (SHAPE, "y and x overlap", dict(y=rows(data=AT + 2))),
    (SHAPE, "out and branch overlap", dict(out=rows(data=AT + (1 << 16) + 4))),
    (SHAPE, "out and x overlap", dict(out=rows(kind=0))),
    (SHAPE, "y and out overlap", dict(out=rows(data=FAR))),
])
def test_norm_refuses(code, words, kw):
    refused(code, words, norm_call(**kw))


def test_layer_refuses_without_a_gpu():
    L, out = M.load(), C.c_void_p()
    p = M.ScaledLinearParams(codes())
    make = lambda d, p: L.mixaq_scaled_linear_create(C.byref(d) if d else None, C.byref(p) if p else None, None, C.byref(out))
    refused(NULL, "descriptor", make(None, p))
    refused(NULL, "params", make(M.ScaledLinearDesc(200, 100, 0), None))
    refused(NULL, "out is NULL", L.mixaq_scaled_linear_create(C.byref(M.ScaledLinearDesc(200, 100, 0)), C.byref(p), None, None))
    for d in ((0, 100, 0), (65537, 100, 0), (200, 0, 0), (200, 65537, 0), (200, 100, 2)):
        refused(SHAPE, "", make(M.ScaledLinearDesc(*d), p))
    refused(SHAPE, "must be codes", make(M.ScaledLinearDesc(200, 100, 0), M.ScaledLinearParams(rows())))
    refused(NULL, "scales", make(M.ScaledLinearDesc(200, 100, 0), M.ScaledLinearParams(codes(scales=None))))
    refused(SHAPE, "stride", make(M.ScaledLinearDesc(300, 100, 0), p))
    refused(SHAPE, "scale_stride", make(M.ScaledLinearDesc(200, 1000, 0), M.ScaledLinearParams(codes(scale_stride=7))))
    assert out.value is None
    refused(NULL, "layer", L.mixaq_scaled_linear_forward(None, rows(), 1, rows(data=FAR), None, 0, None))
    refused(NULL, "layer", L.mixaq_scaled_linear_workspace_bytes(None, 1, 0, 0, None))
    assert L.mixaq_scaled_linear_destroy(None) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    x = torch.zeros((4, 200))
    with pytest.raises(ValueError, match="current device|CUDA|device"):
        M.mixaq_scaled_quantize(x, torch.zeros((4, 208), dtype=torch.uint8).view(torch.float8_e4m3fn)[:, :200], torch.zeros((2, 4)))
    with pytest.raises(ValueError, match="2-D"):
        M._rows(x.double(), "x", 0)
    with pytest.raises(ValueError, match="2-D"):
        M._rows(x[0], "x", 0)
    with pytest.raises(ValueError, match="adjacent"):
        M._rows(x.t(), "x", 0)
    with pytest.raises(ValueError, match="block_rows"):
        M.mixaq_scaled_quantize(x, x, x, 2)
    with pytest.raises(ValueError, match="rows_per_gate"):
        M.make_residual_norm(200, gate=torch.zeros((3, 200)))
    with pytest.raises(ValueError, match="pre must be one of"):
        M.make_residual_norm(200, pre="batch")
    with pytest.raises(ValueError, match="post_gamma"):
        M.make_residual_norm(200, post="layer", post_gamma=torch.zeros(199))
