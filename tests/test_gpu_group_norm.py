"""The group norm on the GPU against its 64-bit reference, and a neck and an expert FFN behind a stage of two-branch blocks."""
import pytest
import torch

import token_ref as R
from test_gpu_token import FILL, Layer, NAN, Room, check_sorted, normal, offsets_of, placed, values

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2507_19131_amd import binding as M


def run(x, y, images, groups, gamma=None, beta=None, act="none", eps=1e-5, y_scales=None):
    norm = M.make_group_norm(x.shape[1], groups, x.shape[0] // images, eps, gamma, beta, act)
    return M.mixaq_group_norm(norm, x, y, y_scales, M.alloc_group_norm_workspace(norm, x.shape[0]))


# images, rows, channels, groups: small maps that one kernel takes (of 8 channels and of 24; at, and one row behind, the most that a workgroup holds), widths that are no
# multiple of 8, groups of a part of 8, of 8 and of more, one channel a group, the most groups and channels
SIZES = [(2, 4096, 32, 4), (1, 4097, 32, 4), (2, 1364, 48, 16), (1, 1365, 48, 16), (3, 16, 2048, 1), (1, 17, 2048, 1), (1, 1, 1, 1), (1, 1, 8, 8), (2, 3, 5, 5), (1, 50, 7, 1), (3, 49, 96, 32), (2, 100, 10, 5), (1, 1050, 256, 32), (2, 333, 129, 3), (4, 17, 264, 11), (1, 5000, 24, 3),
         (2, 700, 1000, 8), (1, 300, 2048, 32), (5, 9, 1024, 1024), (2, 40, 4095, 35), (1, 30, 8192, 64), (3, 5, 8191, 1), (700, 4, 32, 4), (1, 20000, 96, 32), (8, 2500, 128, 32)]


@pytest.mark.parametrize("x_kind,y_kind,act", [("f32", "f32", "none"), ("bf16", "bf16", "silu"), ("f16", "f32", "gelu"), ("f32", "i8", "relu"), ("bf16", "i8", "none"), ("f16", "f16", "relu")])
@pytest.mark.parametrize("images,rows,C,groups", SIZES)
def test_norm(images, rows, C, groups, x_kind, y_kind, act):
    x = placed(values(rows + C, images * rows, C) + normal(C, C), x_kind, 3, 2)
    gamma, beta = 1.0 + 0.25 * normal(1, C), 0.1 * normal(2, C)
    y = Room(images * rows, C, y_kind, 16 if y_kind == "i8" else 5, 3)
    run(x.t, y.t, images, groups, gamma, beta, act, y_scales=y.scales)
    want, bound = R.group_norm(x.t, images, groups, 1e-5, gamma, beta, act)
    if y_kind == "i8":
        R.check_codes(y.t, y.scales, want, bound)
    else:
        R.check(y.t, want, bound, y_kind)
    assert y.untouched() and x.untouched()


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("images,rows,C,groups", [(1, 20000, 96, 32), (2, 3000, 128, 1), (1, 6000, 100, 4), (1, 300, 8192, 64)])
def test_rows_that_start_at_16_bytes(images, rows, C, groups, kind):
    """Their whole pieces take another way to memory; what lies between the rows keeps its pattern."""
    x, y = placed(values(C, images * rows, C), kind), Room(images * rows, C, kind, 8, 8 + -C % 8)
    run(x.t, y.t, images, groups, act="silu")
    R.check(y.t, *R.group_norm(x.t, images, groups, 1e-5, None, None, "silu"), kind)
    assert y.untouched()


@pytest.mark.parametrize("gamma,beta", [(True, False), (False, True), (False, False)])
def test_without_vectors(gamma, beta):
    x = values(3, 200, 96)
    g, b = (normal(i, 96) if on else None for i, on in ((1, gamma), (2, beta)))
    y = torch.empty_like(x)
    run(x, y, 2, 8, g, b)
    R.check(y, *R.group_norm(x, 2, 8, 1e-5, g, b, "none"), "f32")


@pytest.mark.parametrize("C,groups", [(96, 32), (128, 32), (100, 4), (260, 4), (4, 2)])
def test_in_place_and_codes_agree(C, groups):
    """Written over x: the same bits.  Codes: those of the binary32 results."""
    x = values(5, 3 * 801, C)
    y, z, q = torch.empty_like(x), x.clone(), Room(len(x), C, "i8")
    run(x, y, 3, groups, act="silu")
    run(z, z, 3, groups, act="silu")
    run(x, q.t, 3, groups, act="silu", y_scales=q.scales)
    codes, scales = R.quantize(y)
    R.same(y, z)
    R.same(q.t, codes)
    R.same(q.scales, scales)


@pytest.mark.parametrize("rows,C,groups", [(1, 64, 8), (900, 96, 32), (5000, 256, 32)])
def test_a_large_mean_costs_no_digits(rows, C, groups):
    """Equal values leave nothing; a spread far below the mean is kept, by the bound of the reference."""
    beta = normal(4, C)
    for value in (1000.0, -77777.7, 1e30):
        x = torch.full((2 * rows, C), value, device="cuda")
        y = torch.empty_like(x)
        run(x, y, 2, groups, None, beta)
        R.same(y, beta.expand_as(y))
        x += 2.0 ** -10 * abs(value) * normal(6, *x.shape)
        x[0] = 3 * value                                        # the pivot far from the others
        run(x, y, 2, groups, None, beta)
        R.check(y, *R.group_norm(x, 2, groups, 1e-5, None, beta, "none"), "f32")


def test_groups_with_nan_and_infinity_stay_among_themselves():
    x = values(7, 3 * 500, 96)
    x[600, 10], x[1400, 50], x[1000, 95] = NAN, float("inf"), -float("inf")
    y, q = torch.empty_like(x), Room(1500, 96, "i8")
    run(x, y, 3, 8)                                             # groups of 12: image 1 group 0, image 2 groups 4 and 7
    want, bound = R.group_norm(x, 3, 8, 1e-5, None, None, "none")
    R.check(y, want, bound, "f32")
    bad = torch.isnan(y).view(3, 500, 8, 12)
    assert bool(bad[1, :, 0].all() and bad[2, :, 4].all() and bad[2, :, 7].all()) and int(bad.sum()) == 3 * 500 * 12
    run(x, q.t, 3, 8, y_scales=q.scales)                        # a row of codes has one scale
    assert bool(torch.isnan(q.scales[500:]).all() and (q.t[500:] == 0).all() and torch.isfinite(q.scales[:500]).all())


def test_an_image_depends_on_nothing_but_itself():
    x = values(8, 6 * 700, 96).bfloat16()
    y, one = torch.empty_like(x), torch.empty_like(x[:700])
    run(x, y, 6, 32, act="gelu")
    again = torch.empty_like(x)
    run(x, again, 6, 32, act="gelu")
    R.same(y, again)  # no order of additions that changes
    run(x[1400:2100], one, 1, 32, act="gelu")
    want, bound = R.group_norm(x[1400:2100], 1, 32, 1e-5, None, None, "gelu")
    R.check(one, want, bound, "bf16")
    R.check(y[1400:2100], want, bound, "bf16")


def test_offsets_beyond_32_bits():
    rows, C, stride = 70000, 40, 1 << 16
    x = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").as_strided((rows, C), (stride, 1))
    x.copy_(values(9, rows, C))
    want, bound = R.group_norm(x, 1, 5, 1e-5, None, None, "none")
    run(x, x, 1, 5)
    R.check(x, want, bound, "bf16")


def test_captured_and_on_a_stream():
    norms = [M.make_group_norm(96, 32, 1000, activation="silu"), M.make_group_norm(96, 32, 50)]
    x = [values(i, n, 96) for i, n in ((11, 2000), (12, 50))]
    y = [torch.empty_like(t) for t in x]
    ws = [M.alloc_group_norm_workspace(n, len(t)) for n, t in zip(norms, x)]
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        for a in zip(norms, x, y, ws):
            M.mixaq_group_norm(*a[:3], workspace=a[3])
    for seed in (13, 14, 15):
        for i, t in enumerate(x):
            t.copy_(values(seed + i, *t.shape))
        graph.replay()
        torch.cuda.synchronize()
        for n, a, b, w in zip(norms, x, y, ws):
            c = torch.empty_like(a)
            M.mixaq_group_norm(n, a, c, workspace=torch.empty_like(w), stream=stream)
            torch.cuda.synchronize()
            R.same(b, c)


@pytest.mark.parametrize("H,W", [(28, 35), (61, 40)])
def test_neck_and_experts_behind_a_stage(H, W):
    """A stage's map through a group norm to codes, a layer on them, and an expert FFN whose experts the windows' branch chooses: the high-bit
    windows' rows to one, the others to another, by the stage's own list."""
    import gpu_harness as gh
    from paper_2507_19131_amd import synth
    spec = synth.BlockSpec(1, H, W, 96, 3)
    inp = synth.make_block_inputs(spec, 3)
    m = torch.from_numpy(synth.make_feature_map(spec, 3, blobs=True)).cuda()
    block = gh.GpuBlock(inp)
    k = M.mixaq_keep_count(spec.nW, 0.5)
    scores, perm = torch.empty((1, spec.nW), dtype=torch.float64, device="cuda"), torch.empty((1, spec.nW), dtype=torch.int32, device="cuda")
    y, tmp = torch.empty_like(m), torch.empty_like(m)
    M.mixaq_stage_forward([block.blk], m, [k], None, y, tmp, scores, perm, M.alloc_workspace(block.blk))
    rows = y.view(-1, 96)
    # a list of pixels, window by window in the order of the branches; -1 where a window hangs over the map
    nh, nw = -(-H // 7), -(-W // 7)
    pixel = torch.full((nh * 7, nw * 7), -1, dtype=torch.int32, device="cuda")
    pixel[:H, :W] = torch.arange(H * W, device="cuda", dtype=torch.int32).view(H, W)
    gather = pixel.view(nh, 7, nw, 7).transpose(1, 2).reshape(nh * nw, 49)[perm[0].long()].flatten().contiguous()
    counts = [k * 49, (spec.nW - k) * 49]
    off = offsets_of(counts)
    norm = M.make_group_norm(96, 32, H * W, activation="silu")
    q, h, o = Room(H * W, 96, "i8"), Room(len(gather), 384, "bf16"), Room(len(gather), 96, "f32")
    with Layer(21, 384, 96, 2, "gelu") as fc1, Layer(22, 96, 384, 2) as fc2:
        M.mixaq_group_norm(norm, rows, q.t, q.scales, M.alloc_group_norm_workspace(norm, H * W))
        fc1.grouped(q.t, off, h.t, q.scales, gather=gather)
        hidden = torch.where((gather >= 0)[:, None], h.t, torch.zeros_like(h.t))              # (rows without a pixel were left as they were)
        fc2.grouped(hidden, off, o.t)
        torch.cuda.synchronize()
        R.check_codes(q.t, q.scales, *R.group_norm(rows, 1, 32, 1e-5, None, None, "silu"))
        check_sorted(fc1, q.t, q.scales, counts, 0, h, "bf16", gather)
        check_sorted(fc2, *R.quantize(hidden), counts, 0, o, "f32")
        assert int((gather < 0).sum()) == nh * 7 * nw * 7 - H * W and bool((h.buffer[:-1][gather < 0] == FILL).all())
    block.close()
