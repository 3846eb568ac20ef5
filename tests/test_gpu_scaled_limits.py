"""The 8-bit float layers and norms on the GPU at the ends of their arguments' ranges."""
import numpy as np
import pytest
import torch

import scaled_ref as R

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2507_19131_amd import binding as M


def test_a_row_of_nearly_2_31_columns():
    cols = 2**31 - 1
    x = torch.full((1, cols), 0.25, dtype=torch.float16, device="cuda")
    ends = [(0, 384), (2**30, 384), (cols // 128 * 128 - 256, 256 + cols % 128)]
    gen = torch.Generator().manual_seed(4)
    for at, n in ends:
        x[0, at:at + n] = torch.randn(n, generator=gen).half().cuda()
    codes, scales = M.alloc_codes(1, cols)
    M.mixaq_scaled_quantize(x, codes, scales)
    for at, n in ends:
        want, s = R.quantize(x[:, at:at + n].float().cpu().numpy())
        assert np.array_equal(codes[:, at:at + n].view(torch.uint8).cpu().numpy(), want)
        assert np.array_equal(scales[at // 128:at // 128 + s.shape[0]].cpu().double().numpy(), s)


def test_a_product_of_too_many_tiles_is_refused_before_anything_runs():
    """Values are not quantized either."""
    rows, N = 1 << 22, 65536
    w, s_w = M.alloc_codes(N, 1, 128)
    s_w.fill_(1.0)
    h = M.mixaq_scaled_linear_create(w, s_w)
    x = torch.ones((rows, 1), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((M.mixaq_scaled_linear_workspace_bytes(h, rows, torch.bfloat16, torch.bfloat16),), 0x5A, dtype=torch.uint8, device="cuda")
    y = M.Rows(1 << 56, N, 2, None, 0)                     # an address that no call may touch
    rc = M.load().mixaq_scaled_linear_forward(h, M._rows(x, "x", 0), rows, y, ws.data_ptr(), ws.numel(), None)
    assert rc == -2 and b"too many" in M.load().mixaq_last_error()
    torch.cuda.synchronize()
    M.mixaq_scaled_linear_destroy(h)
    assert bool((ws == 0x5A).all())


def test_a_layer_that_finds_no_memory_leaves_no_error_behind():
    """The refusal is the creation's own: the calls after it are not taken for failed ones."""
    n = 65536                                              # 4.3 GB of codes
    w, s_w = M.alloc_codes(n, n, 128)
    s_w.fill_(1.0)
    free, _ = torch.cuda.mem_get_info()
    rest = torch.empty(free - (2 << 30), dtype=torch.uint8, device="cuda")
    with pytest.raises(M.MixaqError) as e:
        M.mixaq_scaled_linear_create(w, s_w)
    assert e.value.code == -5 and "hipMalloc" in str(e.value)
    x = torch.ones((3, 8), device="cuda")
    codes, scales = M.alloc_codes(3, 8)
    M.mixaq_scaled_quantize(x, codes, scales)
    M.mixaq_residual_norm(M.make_residual_norm(8), x, out=torch.empty_like(x))
    torch.cuda.synchronize()
    assert bool((codes.view(torch.uint8) == 0x7E).all())
    del rest, w, s_w
    torch.cuda.empty_cache()
