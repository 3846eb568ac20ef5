"""The 8-bit float linear layers and the norms between them in 64 bits, from their definitions, each with a bound of how far binary32
arithmetic may take a kernel from it.  Numpy; nothing of the library."""
import numpy as np

U = 2.0 ** -24                                   # half a step of binary32, relative
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8, "e4m3": 2.0 ** -4}
LEAST_STEP = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}       # of the values below the normal ones


def _decode(code):
    e, f = code >> 3 & 15, code & 7
    return (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)) if code & 127 != 127 else np.nan


POSITIVE = np.array([_decode(c) for c in range(127)])
DECODE = np.array([_decode(c & 127) * (-1 if c & 128 else 1) for c in range(256)])
assert POSITIVE[126] == 448.0 and np.all(np.diff(POSITIVE) > 0)


def nearest_code(v):
    """Codes 0..255 of values of at most 448 in size (NaN: 127), ties to the even code."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up = a - POSITIVE[lo] > POSITIVE[hi] - a
    tie = a - POSITIVE[lo] == POSITIVE[hi] - a
    c = np.where(up | (tie & (hi % 2 == 0)), hi, lo)
    return np.where(np.isnan(v), 127, np.where(np.signbit(v), c + 128, c)).astype(np.uint8)


def f32(v):
    return np.asarray(v, dtype=np.float64).astype(np.float32).astype(np.float64)


def blocks(n):
    return -(-n // 128)


def quantize(x, block_rows=1):
    """x: binary32 values [rows, cols] -> codes uint8 [rows, cols], scales [ceil(cols / 128), ceil(rows / block_rows)]."""
    rows, cols = x.shape
    v = np.pad(x.astype(np.float64), ((0, -rows % block_rows), (0, -cols % 128)))
    v = v.reshape(v.shape[0] // block_rows, block_rows, -1, 128)
    with np.errstate(invalid="ignore"):
        top = np.abs(v).max((1, 3))
        scale = np.where(np.isfinite(top), f32(np.maximum(top, 2.0 ** -100) / 448.0), np.nan)
        q = np.clip(f32(v * f32(1.0 / scale)[:, None, :, None]), -448.0, 448.0)
    codes = nearest_code(q).reshape(v.shape[0] * block_rows, -1)[:rows, :cols]
    return np.ascontiguousarray(codes), np.ascontiguousarray(scale.T)


def dequantize(codes, scales, block_rows=1):
    wide = np.repeat(np.repeat(scales.T, block_rows, 0), 128, 1)[:codes.shape[0], :codes.shape[1]]
    return DECODE[codes] * wide


def gelu(v):
    from scipy.special import erfc
    return 0.5 * v * erfc(-v / np.sqrt(2.0))


def linear(x, w, bias, with_gelu, kind):
    """Dequantized x [M, K] and w [N, K] -> y and its bound for a result of type `kind`.  Each block's 128 exact products are added one after
    another, each addition off by at most a step (2 U) of the sum of their sizes; then per block a product of the scales and a fused multiply-add,
    and the bias.  Of 16-bit results each group of eight neighbouring products keeps 14 bits, counted from the largest: the seven others are
    off by at most 2^-13 of it, and it is at most the product of the group's largest operands."""
    y = x @ w.T + (0.0 if bias is None else bias)
    size = np.abs(x) @ np.abs(w).T + (0.0 if bias is None else np.abs(bias))
    bound = (128 * 2 * U + (blocks(x.shape[1]) + 3) * U) * size
    if kind in ("f16", "bf16"):
        top = lambda v: np.abs(np.pad(v, ((0, 0), (0, -v.shape[1] % 8)))).reshape(v.shape[0], -1, 8).max(2)
        bound = bound + 7 * 2.0 ** -13 * (top(x) @ top(w).T)
    if not with_gelu:
        return y, bound
    # |gelu'| < 1.13; an approximation of Phi to 0.75e-7 (relative to v), and the roundings of its steps
    return gelu(y), 1.13 * bound + np.abs(y) * (0.75e-7 + 16 * U)


def norm(v, kind, eps, gamma, beta, err):
    """A norm of values that are off by up to err -> result and bound.  Sums: up to 8 x 8 values a lane, then at most 10 levels."""
    depth = 76
    if kind == "none":
        return v, err
    mean = v.mean(1, keepdims=True) if kind == "layer" else np.zeros((v.shape[0], 1))
    c = v - mean
    r = 1.0 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    g = 1.0 if gamma is None else gamma
    out = c * r * g + (0.0 if beta is None else beta)
    e = err + (err.mean(1, keepdims=True) + (depth + 2) * U * np.abs(v).mean(1, keepdims=True) if kind == "layer" else 0.0)
    turn = r * np.sqrt((e * e).mean(1, keepdims=True)) + (depth + 8) * U      # of r, relative
    # where the errors are as large as the values themselves (a row of equal values behind a tiny eps) the root is no bound any more
    turn = np.minimum(turn, 1e3)
    bound = np.abs(g) * r * e * (1 + turn) + np.abs(c * r * g) * (turn + 4 * U) + 2 * U * np.abs(out) + (0.0 if beta is None else 2 * U * np.abs(beta))
    return out, bound


def residual_norm(x, branch, alpha, gate_rows, post, pre):
    """post, pre: (kind, eps, gamma, beta).  Returns (y, bound), (out, bound)."""
    if branch is None:
        v, e = np.zeros_like(x), np.zeros_like(x)
    else:
        v, e = norm(branch, *post, np.zeros_like(branch))
    if gate_rows is not None:
        v, e = v * gate_rows, (e + U * np.abs(v)) * np.abs(gate_rows)
    y = alpha * x + v
    e = e + 3 * U * (np.abs(alpha * x) + np.abs(v))
    return (y, e), norm(y, *pre, e)


def allowed(y, bound, kind):
    """The bound of a result that is rounded to a type at the end."""
    return bound + HALF_STEP[kind] * (np.abs(y) + bound) + LEAST_STEP[kind]


def check_codes(codes, scales, y, bound):
    """Codes and scales [blocks, rows] of results y that are known to `bound`: the scale is its block's largest, the values lie within half a
    step of e4m3 (below 2^-6 steps of 2^-9), each widened by the bound."""
    for b in range(blocks(y.shape[1])):
        part, e = y[:, b * 128:(b + 1) * 128], bound[:, b * 128:(b + 1) * 128]
        top, off = np.maximum(np.abs(part).max(1), 2.0 ** -100), e.max(1)
        assert np.all(np.abs(scales[b] * 448.0 - top) <= off + 2 * U * (top + off)), "scales of block %d" % b
        value = DECODE[codes[:, b * 128:(b + 1) * 128]] * scales[b][:, None]
        half = np.maximum(HALF_STEP["e4m3"] * (np.abs(part) + e), 2.0 ** -10 * scales[b][:, None])
        assert np.all(np.abs(value - part) <= half * (1 + 8 * U) + e), "codes of block %d" % b
