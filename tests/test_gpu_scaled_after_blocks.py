"""A float FFN behind a stage of two-branch blocks: the stage's map, seen as rows of tokens, goes into the norm and the 8-bit float layers as it lies."""
import numpy as np
import pytest
import torch

import gpu_harness as gh
import scaled_ref as R
from paper_2507_19131_amd import binding as M
from paper_2507_19131_amd import synth

pytestmark = pytest.mark.gpu
EPS = float(np.float32(1e-5))


def as64(t):
    return t.detach().cpu().double().numpy()


def as_bytes(t):
    return t.view(torch.uint8).cpu().numpy()


def layer(gen, N, K, activation):
    """A layer of random weights, its weights and bias in 64 bits."""
    w, bias = torch.randn((N, K), generator=gen).cuda() / K ** 0.5, torch.randn(N, generator=gen).cuda()
    codes, scales = M.alloc_codes(N, K, 128)
    M.mixaq_scaled_quantize(w, codes, scales, 128)
    return M.mixaq_scaled_linear_create(codes, scales, bias, activation), R.dequantize(as_bytes(codes), as64(scales), 128), as64(bias)


@pytest.mark.parametrize("B,H,W,C", [(1, 33, 40, 96), (2, 28, 28, 384)])
def test_float_ffn_behind_a_stage(B, H, W, C):
    spec = synth.BlockSpec(B, H, W, C, C // 32)
    gen = torch.Generator().manual_seed(C)
    blocks = [gh.GpuBlock(synth.make_block_inputs(spec, 50 + i), shift) for i, shift in enumerate((0, 3))]
    fc1, w1, b1 = layer(gen, 4 * C, C, "gelu")
    fc2, w2, b2 = layer(gen, C, 4 * C, "none")
    gate = 0.1 + 0.3 * torch.randn((B, C), generator=gen)
    gamma, beta = 1.0 + 0.25 * torch.randn(C, generator=gen), 0.1 * torch.randn(C, generator=gen)
    rows = B * H * W
    before = M.make_residual_norm(C, pre="layer", pre_gamma=gamma.cuda(), pre_beta=beta.cuda())
    after = M.make_residual_norm(C, post="rms", pre="none", gate=gate.cuda(), rows_per_gate=H * W)
    a, a_scales = M.alloc_codes(rows, C)
    b, b_scales = M.alloc_codes(rows, 4 * C)
    f = torch.empty((rows, C), device="cuda")
    x = torch.from_numpy(synth.make_feature_map(spec, 77, blobs=True)).cuda()
    y, tmp = torch.empty_like(x), torch.empty_like(x)
    scores, perm = (torch.empty((B, spec.nW), dtype=t, device="cuda") for t in (torch.float64, torch.int32))

    def run():
        M.mixaq_stage_forward([block.blk for block in blocks], x, [spec.nW // 2], None, y, tmp, scores, perm, blocks[0].ws)
        tokens = y.view(rows, C)
        M.mixaq_residual_norm(before, tokens, out=a, out_scales=a_scales)
        M.mixaq_scaled_linear_forward(fc1, a, b, x_scales=a_scales, y_scales=b_scales)
        M.mixaq_scaled_linear_forward(fc2, b, f, x_scales=b_scales)
        stage = tokens.clone()
        M.mixaq_residual_norm(after, tokens, f, y=tokens)      # the map takes the sum in place
        return stage

    stage = run()
    try:
        n64 = lambda v: v.double().numpy()
        R.check_codes(as_bytes(a), as64(a_scales), *R.norm(as64(stage), "layer", EPS, n64(gamma), n64(beta), np.zeros((rows, C))))
        R.check_codes(as_bytes(b), as64(b_scales), *R.linear(R.dequantize(as_bytes(a), as64(a_scales)), w1, b1, True, "e4m3"))
        want, bound = R.linear(R.dequantize(as_bytes(b), as64(b_scales)), w2, b2, False, "f32")
        assert np.all(np.abs(as64(f) - want) <= R.allowed(want, bound, "f32"))
        (want, bound), _ = R.residual_norm(as64(stage), as64(f), 1.0, np.repeat(n64(gate), H * W, 0), ("rms", EPS, None, None), ("none", 1.0, None, None))
        assert np.all(np.abs(as64(y.view(rows, C)) - want) <= R.allowed(want, bound, "f32"))
        first = y.clone()
        again = run()
        assert torch.equal(stage, again) and torch.equal(first, y)
    finally:
        for h in (fc1, fc2):
            M.mixaq_scaled_linear_destroy(h)
        for block in blocks:
            block.close()
