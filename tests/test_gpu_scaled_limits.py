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
