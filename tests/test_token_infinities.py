"""Results of the int8 layers and the group norm that are infinite, or too large for their type: compared so that a finite result or the other sign in such a place fails."""
import pytest
import torch

import token_forms as S
import token_ref as R
from paper_2507_19131_amd import binding as M

INF = float("inf")


def within(got, y, bound, kind):
    """A result known to `bound` before its rounding lies between the rounded ends (rounding keeps the order, and takes what is too large to infinity); an infinite one is known."""
    assert bool((torch.isfinite(bound) | ~torch.isfinite(y)).all()), "a bound that bounds nothing"
    bound = torch.where(torch.isfinite(y), bound, torch.zeros_like(y))
    low, high = ((y + s * bound).float().to(R.TYPES[kind]) for s in (-1.0, 1.0))
    wrong = ~(((got >= low) & (got <= high)) | (torch.isnan(y) & torch.isnan(got)))
    assert not bool(wrong.any()), "%d of %d, first at %s" % (int(wrong.sum()), wrong.numel(), wrong.nonzero()[0].tolist())


def linear(codes, scales, w, s_w, bias, act, weights=None):
    """The layer with every step of binary32 that can overflow, and the bound of the others."""
    s = R.f32(scales.double()[:, None] * s_w.double())
    total = codes.double() @ w.double().t()
    v = total * s + bias.double()
    bound = torch.where(torch.isinf(v), torch.zeros_like(v), 1.01 * R.U * ((total * s).abs() + v.abs()))       # the sum's rounding and the multiply-add's
    y, b = R.activate(v, bound, act)
    b = torch.where(torch.isinf(v), torch.zeros_like(b), b)
    if act in ("gelu", "silu"):                              # (0 times infinity in 64 bits; the limit is 0)
        y = torch.where(v == -INF, torch.zeros_like(y), y)
    if weights is None:
        return y, b
    return y * weights.double()[:, None], (b * (1 + R.U) + R.U * y.abs()) * weights.double().abs()[:, None]


def inputs(rows, K, N, experts=1, device="cuda"):
    """Codes whose rows' scales go from ordinary ones over those of which half precision has no results to those of which no type has, one infinite, one NaN; a channel of weights with
    a scale that takes the product of the scales beyond binary32 by itself, and no codes but 0 (no number); biases that are infinite."""
    gen = torch.Generator().manual_seed(rows + K + N)
    room = lambda n: torch.zeros((n, -(-K // 16) * 16), dtype=torch.int8)[:, :K]
    x, w = room(rows), room(experts * N)
    x.copy_(torch.randint(-127, 128, x.shape, generator=gen))
    w.copy_(torch.randint(-127, 128, w.shape, generator=gen))
    s, s_w = torch.full((rows,), 0.01), torch.full((experts * N,), 2.0 ** -12)
    s[1::5], s[2::5], s[4::5], s[rows // 2], s[rows // 3] = 2.0 ** 20, 3e38, 2.0 ** 105, INF, float("nan")
    s_w[3], s_w[N - 1] = 2.0 ** 100, 2.0 ** 100
    w[3] = 0
    bias = torch.randn(experts * N, generator=gen)
    bias[1], bias[-2] = INF, -INF
    return [t.to(device) if t.dtype is not torch.int8 else placed(t, device) for t in (x, s, w, s_w, bias)]


def placed(t, device):
    codes, _ = M.alloc_token_codes(*t.shape, device=device)
    return codes.copy_(t)


FORMS = {"few": (33, 200, 40), "mid": (700, 1500, 200), "split": (1100, 640, 1024), "tile": (2100, 384, 1500), "wide": (9000, 790, 1300)}
SORTED = {"few": (20, 150, 300, 260), "tile": (8, 900, 384, 500), "wide": (16, 9000, 300, 1030)}


def test_the_sizes_reach_every_kernel():
    assert all(S.form(*size) == name for name, size in FORMS.items()) and all(S.form(*size[1:], size[0]) == name for name, size in SORTED.items())


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_the_comparison_fails_where_it_has_to(kind):
    """Mistakes in an infinite place, planted in copies of the reference."""
    y, b = linear(*inputs(40, 100, 30, device="cpu"), "none")
    right = y.float().to(R.TYPES[kind])
    within(right, y, b, kind)
    assert bool(torch.isinf(right).any() & torch.isnan(right).any()) and bool((right == INF).any() & (right == -INF).any())
    at = tuple(torch.isinf(y).nonzero()[0].tolist())
    for wrong in (-right[at], 1.0, float("nan"), torch.finfo(R.TYPES[kind]).max):
        bad = right.clone()
        bad[at] = wrong
        with pytest.raises(AssertionError, match="of 1200, first"):
            within(bad, y, b, kind)
    with pytest.raises(AssertionError, match="bounds nothing"):
        within(right, y, torch.full_like(b, INF), kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu", "relu"])
@pytest.mark.parametrize("form", FORMS)
def test_layers(form, act, kind):
    rows, K, N = FORMS[form]
    x, s, w, s_w, bias = inputs(rows, K, N)
    h = M.mixaq_token_linear_create(w, s_w, bias, act)
    y = torch.zeros((rows, N), dtype=R.TYPES[kind], device="cuda")
    M.mixaq_token_linear_forward(h, x, y, x_scales=s)
    torch.cuda.synchronize()
    M.mixaq_token_linear_destroy(h)
    within(y, *linear(x, s, w, s_w, bias, act), kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("form", SORTED)
def test_sorted_rows(form, act, kind):
    """Infinite weights of rows too: of a result of 0 no number."""
    experts, rows, K, N = SORTED[form]
    x, s, w, s_w, bias = inputs(rows, K, N, experts)
    weights = torch.ones(rows, device="cuda")
    weights[::7], weights[3::7], weights[5::7] = INF, -INF, 1e30
    ends = [rows * (e + 1) * (e + 1) // (experts * experts) for e in range(experts)]
    h = M.mixaq_token_linear_create(w, s_w, bias, act, experts)
    y = torch.zeros((rows, N), dtype=R.TYPES[kind], device="cuda")
    M.mixaq_token_linear_forward_grouped(h, x, torch.tensor([0] + ends, dtype=torch.int32, device="cuda"), y, x_scales=s, row_weights=weights)
    torch.cuda.synchronize()
    M.mixaq_token_linear_destroy(h)
    for e, (first, end) in enumerate(zip([0] + ends, ends)):
        if first < end:
            mine, at = slice(e * N, (e + 1) * N), slice(first, end)
            within(y[at], *linear(x[at], s[at], w[mine], s_w[mine], bias[mine], act, weights[at]), kind)


@pytest.mark.gpu
@pytest.mark.parametrize("y_kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu", "relu"])
@pytest.mark.parametrize("images,rows,C,groups", [(2, 300, 96, 32), (2, 300, 128, 4), (1, 5000, 96, 32), (1, 40, 4104, 27), (3, 50, 6, 2)])
def test_norms(images, rows, C, groups, act, y_kind):
    """Channels whose results pass half precision, a beta that is infinite, a group with an infinity in it."""
    gen = torch.Generator(device="cuda").manual_seed(C + rows)
    x = torch.randn(images * rows, C, generator=gen, device="cuda")
    gamma, beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    gamma[::5], beta[1], beta[C - 2], x[rows // 2, 0] = 1e5, INF, -INF, INF
    norm = M.make_group_norm(C, groups, rows, gamma=gamma, beta=beta, activation=act)
    y = torch.zeros((images * rows, C), dtype=R.TYPES[y_kind], device="cuda")
    M.mixaq_group_norm(norm, x, y, workspace=M.alloc_group_norm_workspace(norm, len(x)))
    infinite = torch.where(torch.isinf(beta), beta.double(), torch.zeros_like(beta, dtype=torch.float64))
    want, bound = R.group_norm(x, images, groups, 1e-5, gamma, torch.where(torch.isinf(beta), torch.zeros_like(beta), beta), act)
    limit = infinite if act == "none" else infinite.clamp_min(0.0)
    want = torch.where(torch.isnan(want) | (infinite == 0.0), want, limit.expand_as(want))
    within(y, want, bound, y_kind)
