"""Linear layers on 8-bit integer codes with a scale per token and channel, their form for rows sorted by expert, and the group norm of
channels-last maps: what is measured of them, beside their plain forms.

A case is one call of one operator:
  quantize   values to int8 codes with one scale per row (a token, or a channel of weights): mixaq_token_quantize
  linear     act(x w^T + bias) on such codes, x given as codes or as values: mixaq_token_linear_forward
  experts    the same with weights of its own for each of a number of experts, rows sorted by expert, read through an index and weighted:
             mixaq_token_linear_forward_grouped
  group      act(group norm) of a batch of channels-last maps: mixaq_group_norm

Rows are tokens: 49 to a window, windows as in the Swin-T and Swin-B-shaped feature maps of the benchmark.  Inputs are drawn on the
GPU from the seed: normal values whose channels differ in size, a few of them by far, as activations behind a residual stream do.
"""
import math
from types import SimpleNamespace

import torch

own = False

LEAST = 2.0 ** -100               # the smallest magnitude a row is scaled for
TOP = 127.0
EPS = 1e-5
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}
SIZES = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}
MAX_BYTES = 2.7e8                 # of a drawn case: about the listed ones that move the most
MAX_FLOPS = 5.1e11


def listed():
    return [
        # one window of stage 1 on its way into an 8-bit layer: nothing but latency
        dict(name="quantize 49x96", op="quantize", rows=49, cols=96, type="f32"),
        # the hidden activations of stage 1's FFN on a detection map (1392 windows), where bandwidth counts
        dict(name="quantize 68208x384", op="quantize", rows=68208, cols=384, type="bf16"),
        # a single token through FC1, values in and out: the weights' way to the chip and the launch
        dict(name="linear 1x1024x4096 gelu", op="linear", rows=1, cols=1024, outs=4096, x="bf16", y="bf16", act="gelu", bias=True),
        # an odd layer between odd layers, in 32 bits: every size ends inside a tile
        dict(name="linear 1001x1000x333", op="linear", rows=1001, cols=1000, outs=333, x="i8", y="f32", act="none", bias=False),
        # FC1 of the deep stage 3 on one image (96 windows), codes in
        dict(name="linear 4704x384x1536 gelu", op="linear", rows=4704, cols=384, outs=1536, x="i8", y="bf16", act="gelu", bias=True),
        # a large product, where the matrix cores count
        dict(name="linear 16384x4096x3840", op="linear", rows=16384, cols=4096, outs=3840, x="i8", y="bf16", act="none", bias=True),
        # eight tokens sent to two experts of 32 each, FC1 of an expert FFN, values in: the hit experts' weights and nothing else
        dict(name="experts 16 of 32x1024x2048", op="experts", rows=16, choices=2, experts=32, cols=1024, outs=2048, x="bf16", y="bf16", act="silu", bias=True,
             weighted=False, spare=0),
        # the windows of one image's stage 3 through eight experts' FC1, codes in, an odd share for each
        dict(name="experts 4704 of 8x384x1536", op="experts", rows=4704, choices=1, experts=8, cols=384, outs=1536, x="i8", y="f16", act="gelu", bias=True,
             weighted=False, spare=0),
        # FC2 of an expert FFN on a large batch, two experts a token, results weighted by the router; room for more rows than there are
        dict(name="experts 32768 of 64x2048x1024", op="experts", rows=32768, choices=2, experts=64, cols=2048, outs=1024, x="i8", y="bf16", act="none", bias=False,
             weighted=True, spare=512),
        # the neck's smallest map (stage 4 of one image): latency
        dict(name="group 1x25x42x256", op="group", images=1, rows=1050, cols=256, groups=32, x="f16", y="f16", act="relu"),
        # stage 1's map in 32 bits, three channels a group: groups that end inside a vector
        dict(name="group 1x200x336x96", op="group", images=1, rows=67200, cols=96, groups=32, x="f32", y="f32", act="none"),
        # the wider backbone's stage 1 on a batch of four: bandwidth
        dict(name="group 4x256x256x128 silu", op="group", images=4, rows=65536, cols=128, groups=32, x="bf16", y="bf16", act="silu"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width over the range: mostly one that layers have (a multiple of 32), now and then an odd one."""
    v = _log_uniform(rng, lo, hi)
    return v if v < 32 or rng.random() < 0.25 else v // 32 * 32


def draw(rng):
    op = rng.choice(("quantize", "linear", "linear", "experts", "experts", "group", "group"))
    while True:
        if op == "quantize":
            case = dict(op=op, rows=_log_uniform(rng, 1, 300000), cols=_width(rng, 1, 8192), type=rng.choice(("f32", "f16", "bf16")))
        elif op == "linear":
            case = dict(op=op, rows=_log_uniform(rng, 1, 270000), cols=_width(rng, 16, 8192), outs=_width(rng, 8, 8192),
                        x=rng.choice(("i8", "i8", "bf16", "f16", "f32")), y=rng.choice(("bf16", "bf16", "f16", "f32")),
                        act=rng.choice(("none", "none", "gelu", "silu", "relu")), bias=rng.random() < 0.7)
        elif op == "experts":
            choices = rng.choice((1, 2, 4))
            case = dict(op=op, rows=choices * _log_uniform(rng, 1, 16384), choices=choices, experts=_log_uniform(rng, 4, 64), cols=_width(rng, 16, 4096),
                        outs=_width(rng, 8, 4096), x=rng.choice(("i8", "i8", "bf16", "f16", "f32")), y=rng.choice(("bf16", "bf16", "f16", "f32")),
                        act=rng.choice(("none", "none", "gelu", "silu", "relu")), bias=rng.random() < 0.5, weighted=rng.random() < 0.5,
                        spare=rng.choice((0, 0, 100)))
        else:
            groups = rng.choice((1, 4, 8, 16, 32, 32))
            cols = groups * max(1, _width(rng, 32, 2048) // groups)
            x = rng.choice(("f32", "f16", "bf16"))
            case = dict(op=op, images=rng.choice((1, 1, 2, 3, 4, 8)), rows=_log_uniform(rng, 1, 70000), cols=cols, groups=groups, x=x, y=rng.choice((x, x, "bf16")),
                        act=rng.choice(("none", "relu", "silu", "silu", "gelu")))
        w = work(case)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS:
            return case


# ---------------------------------------------------------------- what a pass cannot do without
def _codes_bytes(rows, cols, name):
    return rows * cols * SIZES[name] + (4 * rows if name == "i8" else 0)


def work(case):
    """Bytes: every input and output once, scales among them; of experts those that rows are likely to hit.  Operations: a product's multiplications
    and additions, and of the others one per value for each step of their formulas."""
    R, C = case["rows"], case["cols"]
    if case["op"] == "quantize":
        return {"bytes": R * C * (SIZES[case["type"]] + 1) + 4 * R, "flops": 4 * R * C}
    if case["op"] == "group":
        return {"bytes": case["images"] * R * C * (SIZES[case["x"]] + SIZES[case["y"]]) + 8 * C, "flops": 8 * case["images"] * R * C}
    N = case["outs"]
    layer = N * C + 4 * N + (4 * N if case["bias"] else 0)
    if case["op"] == "linear":
        return {"bytes": _codes_bytes(R, C, case["x"]) + R * N * SIZES[case["y"]] + layer, "flops": 2 * R * C * N}
    hit = case["experts"] * (1.0 - (1.0 - 1.0 / case["experts"]) ** R)
    return {"bytes": _codes_bytes(R // case["choices"], C, case["x"]) + R * N * SIZES[case["y"]] + hit * layer + 4 * R + (4 * R if case["weighted"] else 0) +
            4 * (case["experts"] + 1), "flops": 2 * R * C * N}


# ---------------------------------------------------------------- inputs
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _values(gen, rows, cols):
    """Channels of different sizes, every fiftieth or so twelve times as large."""
    size = torch.exp(0.5 * _normal(gen, cols))
    size = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.02, 12.0 * size, size)
    return _normal(gen, rows, cols) * size


def _room_for_codes(rows, cols):
    """Rows of codes start at multiples of 16 bytes; zeros fill the rest of a row."""
    return torch.zeros((rows, -(-cols // 16) * 16), dtype=torch.int8, device="cuda")[:, :cols], torch.empty(rows, device="cuda")


def _as_codes(v):
    """Codes and scales of values, as an earlier layer leaves them."""
    codes, scales = _room_for_codes(*v.shape)
    c, s = _quantize(v)
    codes.copy_(c)
    scales.copy_(s)
    return codes, scales


class _Layer:
    """A layer's handle, destroyed with the state."""

    def __init__(self, w, s_w, bias, act, experts):
        from paper_2507_19131_amd import binding as M
        self.M, self.handle = M, M.mixaq_token_linear_create(w, s_w, bias, act, experts)

    def __del__(self):
        if hasattr(self, "handle"):
            self.M.mixaq_token_linear_destroy(self.handle)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    R, C = case["rows"], case["cols"]
    s = SimpleNamespace(case=case)
    if case["op"] == "quantize":
        s.x = _values(gen, R, C).to(TYPES[case["type"]])
        if own:
            s.codes, s.scales = _room_for_codes(R, C)
    elif case["op"] == "group":
        rows = case["images"] * R
        s.x = (_values(gen, rows, C) + 0.5 * _normal(gen, C)).to(TYPES[case["x"]])
        s.gamma, s.beta = 1.0 + 0.25 * _normal(gen, C), 0.1 * _normal(gen, C)
        if own:
            from paper_2507_19131_amd import binding as M
            s.norm = M.make_group_norm(C, case["groups"], R, eps=EPS, gamma=s.gamma, beta=s.beta, activation=case["act"])
            s.y = torch.empty(rows, C, dtype=TYPES[case["y"]], device="cuda")
            s.workspace = M.alloc_group_norm_workspace(s.norm, rows)
    else:
        N, experts = case["outs"], case.get("experts", 1)
        tokens = R // case.get("choices", 1)
        v = _values(gen, tokens, C)
        s.x, s.x_scales = _as_codes(v) if case["x"] == "i8" else (v.to(TYPES[case["x"]]), None)
        s.w, s.s_w = _as_codes(_normal(gen, experts * N, C) / math.sqrt(C))
        s.bias = 0.1 * _normal(gen, experts * N) if case["bias"] else None
        if case["op"] == "experts":
            # an uneven router: experts differ in how much they are liked, and every token chooses by itself
            liking = 0.5 * _normal(gen, experts) + _normal(gen, tokens, experts)
            chosen = liking.topk(case["choices"], dim=1).indices.flatten()
            s.group, order = chosen.sort(stable=True)
            s.gather = (order // case["choices"]).to(torch.int32)
            counts = torch.bincount(chosen, minlength=experts)
            s.most = int(counts.max())
            s.offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
            s.offsets[1:] = counts.cumsum(0)
            s.weights = torch.rand(R, generator=gen, device="cuda") if case["weighted"] else None
        if own:
            rows = R + case.get("spare", 0)
            s.layer = _Layer(s.w, s.s_w, s.bias, case["act"], experts)
            s.y = torch.zeros((rows, N), dtype=TYPES[case["y"]], device="cuda")
            if case["op"] == "experts" and case["spare"]:       # the list and the weights are as long as y; what stands behind the last row is not read
                s.gather = torch.cat([s.gather, torch.zeros(case["spare"], dtype=torch.int32, device="cuda")])
                s.weights = None if s.weights is None else torch.cat([s.weights, torch.zeros(case["spare"], device="cuda")])
            s.workspace = s.layer.M.alloc_token_linear_workspace(s.layer.handle, tokens, s.x.dtype)
    if own:
        from paper_2507_19131_amd import binding as M
        s.M = M
    return s


# ---------------------------------------------------------------- plain forms, 32 bits
def _quantize(x):
    """The scale and its inverse are each the nearest 32-bit value; the divisions are taken in 64 bits, which gives the same."""
    v = x.float()
    top = v.abs().amax(dim=1)
    scale = (top.clamp_min(LEAST).double() / TOP).float()
    inv = (1.0 / scale.double()).float()
    return (v * inv[:, None]).round().to(torch.int8), scale


def _activate(v, act):
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v.clamp_min(0.0) if act == "relu" else v


def _plain_experts(s):
    """Each expert's rows side by side in a matrix of their own, filled up with zeros to the longest."""
    case, N, C = s.case, s.case["outs"], s.case["cols"]
    codes, scales = (s.x, s.x_scales) if case["x"] == "i8" else _quantize(s.x)
    place = torch.arange(case["rows"], device="cuda") - s.offsets[s.group]
    gather = s.gather[:case["rows"]]
    x = torch.zeros((case["experts"], s.most, C), device="cuda")
    x[s.group, place] = codes[gather].float()
    y = torch.bmm(x, s.w.view(case["experts"], N, C).float().transpose(1, 2).contiguous())[s.group, place]
    y = y * scales[gather][:, None] * s.s_w.view(-1, N)[s.group]
    y = _activate(y if s.bias is None else y + s.bias.view(-1, N)[s.group], case["act"])
    y = y if s.weights is None else y * s.weights[:case["rows"], None]
    out = torch.zeros((case["rows"] + case["spare"], N), dtype=TYPES[case["y"]], device="cuda")
    out[:case["rows"]] = y
    return out


def _plain(s):
    case = s.case
    if case["op"] == "quantize":
        codes, scales = _quantize(s.x)
        return {"codes": codes, "scales": scales}
    if case["op"] == "experts":
        return _plain_experts(s)
    if case["op"] == "linear":
        codes, scales = (s.x, s.x_scales) if case["x"] == "i8" else _quantize(s.x)
        y = codes.float() @ s.w.float().t() * scales[:, None] * s.s_w
        return _activate(y if s.bias is None else y + s.bias, case["act"]).to(TYPES[case["y"]])
    v = s.x.float().view(case["images"], case["rows"], case["groups"], -1)
    v = v - v.mean(dim=(1, 3), keepdim=True)
    v = v * torch.rsqrt(v.square().mean(dim=(1, 3), keepdim=True) + EPS)
    return _activate(v.view(-1, case["cols"]) * s.gamma + s.beta, case["act"]).to(TYPES[case["y"]])


def run(state):
    if not own:
        return _plain(state)
    s, M = state, state.M
    if s.case["op"] == "quantize":
        M.mixaq_token_quantize(s.x, s.codes, s.scales)
        return {"codes": s.codes, "scales": s.scales}
    if s.case["op"] == "linear":
        return M.mixaq_token_linear_forward(s.layer.handle, s.x, s.y, x_scales=s.x_scales, workspace=s.workspace)
    if s.case["op"] == "experts":
        return M.mixaq_token_linear_forward_grouped(s.layer.handle, s.x, s.offsets, s.y, x_scales=s.x_scales, gather=s.gather, row_weights=s.weights,
                                                    workspace=s.workspace)
    return M.mixaq_group_norm(s.norm, s.x, s.y, workspace=s.workspace)


# ---------------------------------------------------------------- the definition in 64 bits
def _f32(v):
    """The nearest 32-bit value, where the definition has one."""
    return v.to(torch.float32).to(torch.float64)


def _exact_codes(x):
    v = x.double()
    top = torch.maximum(v.max(dim=1).values, -v.min(dim=1).values)
    scale = _f32(torch.maximum(top, torch.full_like(top, LEAST)) / torch.full_like(top, TOP))
    return torch.round(_f32(v * _f32(torch.ones_like(scale) / scale).unsqueeze(1))), scale


def _exact_activate(v, act):
    if act == "gelu":
        return v * 0.5 * torch.erfc(-v * math.sqrt(0.5))
    if act == "silu":
        return v * torch.sigmoid(v)
    return torch.where(v > 0, v, torch.zeros_like(v)) if act == "relu" else v


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        codes, scales = _exact_codes(s.x)
        return {"codes": codes.to(torch.int8), "scales": scales}
    if case["op"] == "group":
        v = s.x.double().reshape(case["images"], case["rows"], case["groups"], case["cols"] // case["groups"]).transpose(1, 2)
        flat = v.reshape(case["images"] * case["groups"], -1)
        centre = flat.sum(dim=1, keepdim=True) / flat.shape[1]
        flat = (flat - centre) / torch.sqrt(((flat - centre) ** 2).sum(dim=1, keepdim=True) / flat.shape[1] + EPS)
        y = flat.reshape(v.shape).transpose(1, 2).reshape(-1, case["cols"])
        return _exact_activate(y * s.gamma.double() + s.beta.double(), case["act"])
    codes, scales = (s.x.double(), s.x_scales.double()) if case["x"] == "i8" else _exact_codes(s.x)
    values = codes * scales[:, None]
    N, experts = case["outs"], case.get("experts", 1)
    bias = torch.zeros(experts * N, dtype=torch.float64, device="cuda") if s.bias is None else s.bias.double()
    if experts == 1 and case["op"] == "linear":
        return _exact_activate(values @ (s.w.double() * s.s_w.double()[:, None]).t() + bias, case["act"])
    y = torch.zeros((case["rows"] + case["spare"], N), dtype=torch.float64, device="cuda")
    ends = s.offsets.tolist()
    for e in range(experts):
        if ends[e] < ends[e + 1]:
            mine = slice(e * N, (e + 1) * N)
            y[ends[e]:ends[e + 1]] = values[s.gather[ends[e]:ends[e + 1]].long()] @ (s.w[mine].double() * s.s_w[mine].double()[:, None]).t() + bias[mine]
    y[:case["rows"]] = _exact_activate(y[:case["rows"]], case["act"])
    if s.weights is not None:
        y[:case["rows"]] *= s.weights[:case["rows"], None].double()
    return y
