"""The 8-bit float linear layers and the norms between them: what is measured of them, beside their plain forms.

A case is one call of one operator:
  quantize   values to e4m3 codes with one scale per 1 x 128 block (activations) or 128 x 128 block (weights):
             mixaq_scaled_quantize
  linear     act(x w^T + bias) on such codes, x given as codes or as values, y as values or as codes again:
             mixaq_scaled_linear_forward
  norm       y = residual_scale * x + gate * post_norm(branch), out = pre_norm(y), out as values or as codes:
             mixaq_residual_norm

Rows are tokens: 49 to a window, windows as in the Swin-T and Swin-B-shaped feature maps of the benchmark.  Inputs are drawn on the
GPU from the seed: normal values whose channels differ in size, a few of them by far, as activations behind a residual stream do.
"""
import math
from types import SimpleNamespace

import torch
import torch.nn.functional as F

own = False

BLOCK = 128                       # columns that share a scale
E4M3_MAX = 448.0
LEAST = 2.0 ** -100               # the smallest magnitude a block is scaled for
EPS = 1e-5                        # of the norms
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
MAX_BYTES = 1.8e8                 # of a drawn case: about the listed ones that move the most
MAX_FLOPS = 5.0e11


def listed():
    return [
        # one window of stage 1 on its way into an 8-bit layer: nothing but latency
        dict(name="quantize 49x96", op="quantize", rows=49, cols=96, type="f32", block_rows=1),
        # the hidden activations of stage 1's FFN on a detection map (1392 windows), where bandwidth counts
        dict(name="quantize 68208x384", op="quantize", rows=68208, cols=384, type="bf16", block_rows=1),
        # a trained weight matrix on its way into a layer, rows and columns that end inside a block
        dict(name="quantize weights 4000x1000", op="quantize", rows=4000, cols=1000, type="f32", block_rows=128),
        # a single token through FC1, values in and out: the weights' way to the chip and the launch
        dict(name="linear 1x1024x4096 gelu", op="linear", rows=1, cols=1024, outs=4096, x="bf16", y="bf16", gelu=True, bias=True),
        # a classifier's head on a batch of pooled rows, in 32 bits; the output ends inside a block
        dict(name="linear 50x768x1000", op="linear", rows=50, cols=768, outs=1000, x="f32", y="f32", gelu=False, bias=True),
        # an odd layer between odd layers: every size ends inside a tile
        dict(name="linear 1001x1000x333", op="linear", rows=1001, cols=1000, outs=333, x="e4m3", y="f16", gelu=False, bias=False),
        # FC1 and FC2 of the deep stage 3 on one image (96 windows), codes handed from layer to layer
        dict(name="linear 4704x384x1536 gelu", op="linear", rows=4704, cols=384, outs=1536, x="e4m3", y="e4m3", gelu=True, bias=True),
        # FC1 of the wider backbone's stage 1 on a batch of four (5476 windows): codes in, codes out, one block deep
        dict(name="linear 268324x128x512 gelu", op="linear", rows=268324, cols=128, outs=512, x="e4m3", y="e4m3", gelu=True, bias=True),
        # a large product, where the matrix cores count
        dict(name="linear 16384x4096x3840", op="linear", rows=16384, cols=4096, outs=3840, x="e4m3", y="bf16", gelu=False, bias=True),
        # a single token between two layers
        dict(name="norm 1x1024", op="norm", rows=1, cols=1024, x="bf16", branch="bf16", out="bf16", post="rms", pre="rms", gate="channel"),
        # norms before and after the blocks of stage 1 on a detection map, in 32 bits, codes for the layer that follows
        dict(name="norm 68208x96", op="norm", rows=68208, cols=96, x="f32", branch="f32", out="e4m3", post="layer", pre="layer", gate="channel"),
        # wide rows of several images, each with a gate of its own, and a width that is odd
        dict(name="norm 8190x4095", op="norm", rows=8190, cols=4095, x="bf16", branch="bf16", out="bf16", post="none", pre="layer", gate="image"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width over the range: mostly one that layers have (a multiple of 32), now and then an odd one."""
    v = _log_uniform(rng, lo, hi)
    return v if v < 32 or rng.random() < 0.25 else v // 32 * 32


def draw(rng):
    op = rng.choice(("quantize", "linear", "linear", "norm"))
    while True:
        if op == "quantize":
            case = dict(op=op, rows=_log_uniform(rng, 1, 300000), cols=_width(rng, 1, 8192), type=rng.choice(("f32", "f16", "bf16")),
                        block_rows=rng.choice((1, 1, 128)))
        elif op == "linear":
            case = dict(op=op, rows=_log_uniform(rng, 1, 270000), cols=_width(rng, 16, 8192), outs=_width(rng, 8, 8192),
                        x=rng.choice(("e4m3", "e4m3", "bf16", "f16", "f32")), y=rng.choice(("e4m3", "bf16", "bf16", "f16", "f32")),
                        gelu=rng.random() < 0.5, bias=rng.random() < 0.7)
        else:
            x = rng.choice(("f32", "f16", "bf16"))
            case = dict(op=op, rows=_log_uniform(rng, 1, 300000), cols=_width(rng, 8, 8192), x=x, branch=rng.choice((x, "bf16")),
                        out=rng.choice(("e4m3", x, "bf16")), post=rng.choice(("none", "layer", "rms")), pre=rng.choice(("layer", "rms")),
                        gate=rng.choice(("none", "channel", "image")))
        w = work(case)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS:
            return case


# ---------------------------------------------------------------- what a pass cannot do without
def _size(name):
    return {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}[name]


def _blocks(n):
    return -(-n // BLOCK)


def _rows_bytes(rows, cols, name):
    return rows * cols * _size(name) + (4 * rows * _blocks(cols) if name == "e4m3" else 0)


def work(case):
    """Bytes: every input and output once, scales among them.  Operations: a product's multiplications and additions, and of the others one
    per value for each step of their formulas (magnitude, maximum, product, rounding; the moments and products of a norm)."""
    R, C = case["rows"], case["cols"]
    if case["op"] == "quantize":
        return {"bytes": R * C * (_size(case["type"]) + 1) + 4 * _blocks(C) * -(-R // case["block_rows"]), "flops": 4 * R * C}
    if case["op"] == "linear":
        N = case["outs"]
        return {"bytes": _rows_bytes(R, C, case["x"]) + _rows_bytes(R, N, case["y"]) + N * C + 4 * _blocks(N) * _blocks(C) + (4 * N if case["bias"] else 0),
                "flops": 2 * R * C * N}
    vectors = 4 * C * (2 * (case["post"] == "layer") + (case["post"] == "rms") + 2 * (case["pre"] == "layer") + (case["pre"] == "rms"))
    gate = {"none": 0, "channel": 1, "image": _images(case)}[case["gate"]] * C * 4
    return {"bytes": 2 * R * C * _size(case["x"]) + R * C * _size(case["branch"]) + _rows_bytes(R, C, case["out"]) + vectors + gate, "flops": 16 * R * C}


def _images(case):
    """Rows of a batch of images; each image has as many, the last one perhaps fewer."""
    return min(4, case["rows"])


# ---------------------------------------------------------------- inputs
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _values(gen, rows, cols):
    """Channels of different sizes, every fiftieth or so twelve times as large."""
    size = torch.exp(0.5 * _normal(gen, cols))
    size = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.02, 12.0 * size, size)
    return _normal(gen, rows, cols) * size


def _room_for_codes(rows, cols, block_rows=1):
    """Rows of codes start at multiples of 16 bytes; zeros fill the rest of a row."""
    codes = torch.zeros((rows, -(-cols // 16) * 16), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :cols]
    return codes, torch.empty((_blocks(cols), -(-rows // block_rows)), device="cuda")


def _as_codes(v, block_rows=1):
    """Codes and scales of values, as an earlier layer leaves them."""
    codes, scales = _room_for_codes(v.shape[0], v.shape[1], block_rows)
    c, s = _quantize(v, block_rows)
    codes.view(torch.uint8).copy_(c.view(torch.uint8))
    scales.copy_(s)
    return codes, scales


def _empty_rows(rows, cols, name):
    return _room_for_codes(rows, cols) if name == "e4m3" else (torch.empty((rows, cols), dtype=TYPES[name], device="cuda"), None)


class _Layer:
    """A layer's handle, destroyed with the state."""

    def __init__(self, w, s_w, bias, gelu):
        from paper_2507_19131_amd import binding as M
        self.M, self.handle = M, M.mixaq_scaled_linear_create(w, s_w, bias, "gelu" if gelu else "none")

    def __del__(self):
        if hasattr(self, "handle"):
            self.M.mixaq_scaled_linear_destroy(self.handle)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    R, C = case["rows"], case["cols"]
    s = SimpleNamespace(case=case)
    if case["op"] == "quantize":
        # weights are smaller and more even than activations
        s.x = (0.02 * _normal(gen, R, C) if case["block_rows"] > 1 else _values(gen, R, C)).to(TYPES[case["type"]])
        if own:
            s.codes, s.scales = _room_for_codes(R, C, case["block_rows"])
    elif case["op"] == "linear":
        N = case["outs"]
        v = _values(gen, R, C)
        s.x, s.x_scales = _as_codes(v) if case["x"] == "e4m3" else (v.to(TYPES[case["x"]]), None)
        s.w, s.s_w = _as_codes(_normal(gen, N, C) / math.sqrt(C), BLOCK)
        s.bias = 0.1 * _normal(gen, N) if case["bias"] else None
        if own:
            s.layer = _Layer(s.w, s.s_w, s.bias, case["gelu"])
            s.y, s.y_scales = _empty_rows(R, N, case["y"])
            s.workspace = s.layer.M.alloc_linear_workspace(s.layer.handle, R, s.x.dtype, s.y.dtype)
    else:
        s.x, s.branch = _values(gen, R, C).to(TYPES[case["x"]]), _values(gen, R, C).to(TYPES[case["branch"]])
        s.residual_scale = 0.75
        s.rows_per_gate = -(-R // _images(case)) if case["gate"] == "image" else max(R, 1)
        s.gate = None if case["gate"] == "none" else 0.1 + 0.3 * _normal(gen, -(-R // s.rows_per_gate), C)
        for side in ("post", "pre"):
            kind = case[side]
            setattr(s, side + "_gamma", (1.0 + 0.25 * _normal(gen, C)) if kind != "none" else None)
            setattr(s, side + "_beta", 0.1 * _normal(gen, C) if kind == "layer" else None)
        if own:
            from paper_2507_19131_amd import binding as M
            s.norm = M.make_residual_norm(C, post=case["post"], pre=case["pre"], eps=EPS, residual_scale=s.residual_scale, post_gamma=s.post_gamma,
                                          post_beta=s.post_beta, pre_gamma=s.pre_gamma, pre_beta=s.pre_beta, gate=s.gate, rows_per_gate=s.rows_per_gate)
            s.y = torch.empty_like(s.x)
            s.out, s.out_scales = _empty_rows(R, C, case["out"])
    if own:
        from paper_2507_19131_amd import binding as M
        s.M = M
    return s


# ---------------------------------------------------------------- plain forms, 32 bits
def _in_blocks(v, block_rows):
    """[rows, cols] -> [row blocks, block_rows, column blocks, 128], zeros beyond the edges."""
    rows, cols = v.shape
    v = F.pad(v, (0, -cols % BLOCK, 0, -rows % block_rows))
    return v.view(-1, block_rows, v.shape[1] // BLOCK, BLOCK)


def _scales(amax):
    """The scale and its inverse, each the nearest 32-bit value; the division is taken in 64 bits, which gives the same."""
    scale = (amax.clamp_min(LEAST).double() / torch.full_like(amax, E4M3_MAX, dtype=torch.float64)).float()
    scale = torch.where(torch.isfinite(amax), scale, torch.full_like(amax, math.nan))
    return scale, (torch.ones_like(scale, dtype=torch.float64) / scale.double()).float()


def _quantize(x, block_rows=1):
    v = _in_blocks(x.float(), block_rows)
    scale, inv = _scales(v.abs().amax(dim=(1, 3)))
    q = (v * inv[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q.view(torch.uint8).view(v.shape[0] * block_rows, -1)[:x.shape[0], :x.shape[1]].contiguous().view(torch.float8_e4m3fn), scale.t().contiguous()


def _dequantize(codes, scales, block_rows=1):
    v = _in_blocks(codes.float(), block_rows) * scales.t()[:, None, :, None]
    return v.view(v.shape[0] * block_rows, -1)[:codes.shape[0], :codes.shape[1]]


def _plain_rows(v, name):
    if name == "e4m3":
        codes, scales = _quantize(v)
        return {"codes": codes, "scales": scales}
    return {"values": v.to(TYPES[name])}


def _plain_norm(v, kind, gamma, beta):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    v = v * torch.rsqrt(v.square().mean(dim=1, keepdim=True) + EPS) * gamma
    return v if beta is None else v + beta


def _plain(s):
    case = s.case
    if case["op"] == "quantize":
        codes, scales = _quantize(s.x, case["block_rows"])
        return {"codes": codes, "scales": scales}
    if case["op"] == "linear":
        x = _dequantize(s.x, s.x_scales) if case["x"] == "e4m3" else _dequantize(*_quantize(s.x))
        y = x @ _dequantize(s.w, s.s_w, BLOCK).t()
        if s.bias is not None:
            y = y + s.bias
        if case["gelu"]:
            y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
        return _plain_rows(y, case["y"])
    v = _plain_norm(s.branch.float(), case["post"], s.post_gamma, s.post_beta)
    if s.gate is not None:
        v = v * s.gate.repeat_interleave(s.rows_per_gate, 0)[:v.shape[0]]
    y = s.residual_scale * s.x.float() + v
    return {"y": y.to(s.x.dtype), "out": _plain_rows(_plain_norm(y, case["pre"], s.pre_gamma, s.pre_beta), case["out"])}


def run(state):
    if not own:
        return _plain(state)
    s, M = state, state.M
    if s.case["op"] == "quantize":
        M.mixaq_scaled_quantize(s.x, s.codes, s.scales, s.case["block_rows"])
        return {"codes": s.codes, "scales": s.scales}
    if s.case["op"] == "linear":
        M.mixaq_scaled_linear_forward(s.layer.handle, s.x, s.y, x_scales=s.x_scales, y_scales=s.y_scales, workspace=s.workspace)
        return {"values": s.y} if s.y_scales is None else {"codes": s.y, "scales": s.y_scales}
    M.mixaq_residual_norm(s.norm, s.x, s.branch, s.y, s.out, out_scales=s.out_scales)
    return {"y": s.y, "out": {"values": s.out} if s.out_scales is None else {"codes": s.out, "scales": s.out_scales}}


# ---------------------------------------------------------------- the definition in 64 bits
def _f32(v):
    """The nearest 32-bit value, where the definition has one."""
    return v.to(torch.float32).to(torch.float64)


def _nearest_code(v):
    """The e4m3 value next to v (at most 448 in size), ties to the even one: three bits behind the leading one, steps of 2^-9 at the bottom."""
    _, e = torch.frexp(v)
    step = ((e.to(torch.int64) - 1).clamp_min(-6) - 3 + 1023 << 52).view(torch.float64)          # powers of two, from their bits
    return torch.round(v / step) * step


def _exact_codes(v, block_rows=1):
    """Values [rows, cols] in 64 bits that are 32-bit values -> codes as values, scales."""
    rows, cols = v.shape
    big = torch.zeros((-(-rows // block_rows) * block_rows, _blocks(cols) * BLOCK), dtype=torch.float64, device=v.device)
    big[:rows, :cols] = v
    top = big.abs().unflatten(1, (-1, BLOCK)).amax(dim=2).unflatten(0, (-1, block_rows)).amax(dim=1)
    scale = _f32(torch.maximum(top, torch.full_like(top, LEAST)) / torch.full_like(top, E4M3_MAX))
    inv = _f32(torch.ones_like(scale) / scale)
    wide = inv.repeat_interleave(block_rows, 0).repeat_interleave(BLOCK, 1)[:rows, :cols]
    return _nearest_code(torch.clamp(_f32(v * wide), -E4M3_MAX, E4M3_MAX)), scale.t().contiguous()


def _exact_values(codes, scales, block_rows=1):
    wide = scales.double().t().repeat_interleave(block_rows, 0).repeat_interleave(BLOCK, 1)
    return codes.to(torch.float64) * wide[:codes.shape[0], :codes.shape[1]]


def _exact_rows(v, name):
    if name != "e4m3":
        return {"values": v}
    codes, scales = _exact_codes(_f32(v))
    return {"codes": codes, "scales": scales}


def _exact_norm(v, kind, gamma, beta):
    if kind == "none":
        return v
    centre = v.mean(dim=1, keepdim=True) if kind == "layer" else 0.0
    spread = ((v - centre) ** 2).sum(dim=1, keepdim=True) / v.shape[1]
    v = (v - centre) / torch.sqrt(spread + EPS) * gamma.double()
    return v if beta is None else v + beta.double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        codes, scales = _exact_codes(s.x.double(), case["block_rows"])
        return {"codes": codes, "scales": scales}
    if case["op"] == "linear":
        x = _exact_values(s.x, s.x_scales) if case["x"] == "e4m3" else _exact_values(*_exact_codes(s.x.double()))
        y = x @ _exact_values(s.w, s.s_w, BLOCK).t()
        y = y if s.bias is None else y + s.bias.double()
        return _exact_rows(y * 0.5 * torch.erfc(-y * math.sqrt(0.5)) if case["gelu"] else y, case["y"])
    v = _exact_norm(s.branch.double(), case["post"], s.post_gamma, s.post_beta)
    if s.gate is not None:
        rows = torch.arange(v.shape[0], device=v.device) // s.rows_per_gate
        v = v * s.gate.double()[rows]
    y = s.residual_scale * s.x.double() + v
    return {"y": y, "out": _exact_rows(_exact_norm(y, case["pre"], s.pre_gamma, s.pre_beta), case["out"])}
