"""The int8 layers with a scale per token and the group norm in 64 bits, from their definitions, each with a bound of how far binary32 arithmetic
may take a kernel from it.  Torch on any device, elementary operations; nothing of the library."""
import torch

U = 2.0 ** -24                                   # half a step of binary32, relative
UD = 2.0 ** -53
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}
LEAST_STEP = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}       # of the values below the normal ones


def f32(v):
    return v.to(torch.float32).to(torch.float64)


def by_halves(t, op):
    """op over the last dimension, half of it with the other half: torch's reductions that go over several workgroups give a wrong sum now and then.  float64 means
    over 1856 x 399 of 27 groups, on the same data, in processes that load nothing but torch: 1 of 85208, and 5053 of 70765 with a sum over rows in
    between; a group's mean then lacks a part."""
    while t.shape[-1] > 1:
        m, half = t.shape[-1], (t.shape[-1] + 1) // 2
        t = torch.cat([op(t[..., :m - half], t[..., half:]), t[..., m - half:half]], -1)
    return t[..., 0]


def largest(t):
    return by_halves(t, torch.maximum)


def quantize(x):
    """Values [rows, cols] -> codes int8, scales [rows], each the definition's own bits."""
    v = x.double()
    top = largest(v.abs())
    bad = ~torch.isfinite(top)
    scale = f32(top.clamp_min(2.0 ** -100) / 127.0)
    inv = f32(1.0 / scale)
    codes = torch.where(bad[:, None], torch.zeros_like(v), torch.round(f32(v * inv[:, None])))
    return codes.to(torch.int8), torch.where(bad, torch.full_like(scale, float("nan")), scale).float()


def activate(v, bound, act):
    """An activation of values that are off by up to `bound`."""
    if act == "gelu":                            # |gelu'| < 1.13; to within 2.1e-7 of its argument
        return 0.5 * v * torch.erfc(-v * 0.5 ** 0.5), 1.13 * bound + 2.1e-7 * (v.abs() + bound)
    if act == "silu":                            # |silu'| < 1.1; to within 4e-7 of its argument
        return v * torch.sigmoid(v), 1.1 * bound + 4e-7 * (v.abs() + bound)
    return (v.clamp_min(0.0) if act == "relu" else v), bound


def linear(codes, scales, w, s_w, bias, act, weights=None):
    """codes [M, K] int8, w [N, K] int8 -> y and its bound before its rounding to y's type: the sum is exact, its conversion, the product of the scales and the
    fused multiply-add are off by half a step each (the first two of the product), a weight's product by another."""
    total = codes.double() @ w.double().t()      # whole numbers below 2^31
    s = scales.double()[:, None] * s_w.double()
    v = total * s + (0.0 if bias is None else bias.double())
    bound = 2.01 * U * (total * s).abs() + 1.01 * U * v.abs() + 2.0 ** -126 * U * total.abs()
    y, bound = activate(v, bound, act)
    if weights is None:
        return y, bound
    return y * weights.double()[:, None], (bound * (1 + U) + U * y.abs()) * weights.double().abs()[:, None]


def fma(a, b, c):
    """Of binary32 values in 64 bits, rounded once: the product is exact, and what its sum with c loses (by the six steps of an exact sum) makes the last of its 53
    bits odd, so that the second rounding meets no tie that is none."""
    p = a * b
    t = p + c
    back = t - p
    lost = (p - (t - back)) + (c - back)
    bits = t.view(torch.int64)
    towards = torch.where((lost > 0) == (t > 0), bits + 1, bits - 1)
    return torch.where((lost != 0) & (bits % 2 == 0), towards, bits).view(torch.float64).float()


def linear_bits(codes, scales, w, s_w, bias, kind):
    """Without an activation every step has one nearest result."""
    s = f32(scales.double()[:, None] * s_w.double())
    total = f32(codes.double() @ w.double().t())
    v = fma(total, s, bias.double().expand_as(s)) if bias is not None else (total * s).float()
    return v.to(TYPES[kind])


def same(a, b):
    if not torch.equal(a, b):
        at = (a != b).nonzero()
        raise AssertionError("%d of %d differ, first at %s: %s, %s" % (len(at), a.numel(), at[0].tolist(), a[tuple(at[0])].item(), b[tuple(at[0])].item()))


def group_norm(x, images, groups, eps, gamma, beta, act):
    """x [images * rows, C] -> y and its bound before its rounding.  The kernel: sums in binary64 of differences d from a group's first value; the mean as two
    binary32 numbers; then (x - hi) a + b, a = f32(f32(1 / sqrt) gamma), b = fma(-lo, a, beta)."""
    rows, C = x.shape[0] // images, x.shape[1]
    v = x.double().reshape(images, rows, groups, C // groups)
    first = v[:, :1, :, :1]
    d = v - first
    n = rows * (C // groups)
    mean_of = lambda t: by_halves(t.movedim(2, 1).reshape(images, groups, n), torch.add).reshape(images, 1, groups, 1) / n
    off = mean_of(d)
    var = mean_of((d - off).square())
    c = d - off
    r = 1.0 / torch.sqrt(var + eps)
    wide = lambda t: t.expand(v.shape).reshape(x.shape)
    c, r_, mean = c.reshape(x.shape), wide(r), wide(first + off)
    g = torch.ones(C, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    b = torch.zeros(C, dtype=torch.float64, device=x.device) if beta is None else beta.double()
    y = c * r_ * g + b
    e_mean = (n + 8) * UD * mean_of(d.abs()) + 4 * UD * (first + off).abs()
    e_var = 4 * (n + 8) * UD * mean_of(d.square())
    turn = wide(0.5 * e_var / (var + eps)) + 2.02 * U                            # of a, relative
    size = (c * r_ * g).abs()
    # the difference from hi: half a step of itself, where hi is off the mean by up to U |mean|, which b takes back
    bound = size * turn + 1.01 * U * (c.abs() + U * mean.abs()) * (r_ * g).abs() + (r_ * g).abs() * (wide(e_mean) + 3 * U * U * mean.abs()) + \
        1.01 * U * (b.abs() + U * mean.abs() * (r_ * g).abs()) + 1.01 * U * y.abs()
    return activate(y, bound, act)


def allowed(y, bound, kind):
    """The bound of a result that is rounded to a type at the end."""
    return bound + torch.finfo(TYPES[kind]).eps / 2 * (y.abs() + bound) + LEAST_STEP[kind]


def check(got, y, bound, kind):
    got = got.double()
    wrong = torch.isnan(y) != torch.isnan(got)
    assert not bool(wrong.any()), "NaN at %s" % (wrong.nonzero()[:3].tolist(),)
    off = (got - y).abs() - allowed(y, bound, kind)
    off = torch.where(torch.isnan(off), torch.zeros_like(off), off)
    assert bool((off <= 0).all()), "row, column %s: over by %g" % ((off > 0).nonzero()[:3].tolist(), float(off.max()))


def check_codes(codes, scales, y, bound):
    """Codes and scales of results y that are known to `bound`: the scale is the row's largest, the values lie within half a step, each widened by
    the bound."""
    top, off = largest(y.abs()).clamp_min(2.0 ** -100), largest(bound)
    s = scales.double()
    assert bool(((s * 127.0 - top).abs() <= off + 2 * U * (top + off)).all()), "scales"
    assert bool(((codes.double() * s[:, None] - y).abs() <= 0.5 * s[:, None] * (1 + 300 * U) + bound).all()), "codes"
