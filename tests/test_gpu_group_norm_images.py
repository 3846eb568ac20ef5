"""The group norm of more images than one kernel takes in a launch of a workgroup for each part of an image's channels."""
import pytest
import torch

import token_ref as R
from paper_2507_19131_amd import binding as M
from test_token_refusals import SHAPE, norm_call, refused, values as rows_at


def norm(x, images, groups, y, act="none", y_scales=None):
    n = M.make_group_norm(x.shape[1], groups, len(x) // images, activation=act)
    return M.mixaq_group_norm(n, x, y, y_scales, M.alloc_group_norm_workspace(n, len(x)))


# 1024 parts of 8 channels: 2^22 workgroups of 1024 threads from 4096 images on, which the two kernels of larger maps take; 1024 parts of two rows; one part, of few and of many channels
@pytest.mark.gpu
@pytest.mark.parametrize("images,rows,C,groups,kind", [(4095, 1, 8192, 1024, "bf16"), (4096, 1, 8192, 1024, "bf16"), (4097, 2, 8192, 1024, "f16"), (65537, 1, 512, 64, "f32"),
                                                       ((1 << 22) + 3, 1, 8, 1, "bf16"), ((1 << 22) + 3, 1, 5, 5, "f32")])
def test_many_images(images, rows, C, groups, kind):
    x = torch.randn(images * rows, C, generator=torch.Generator(device="cuda").manual_seed(images), device="cuda").to(R.TYPES[kind])
    y = torch.full_like(x, float("nan"))
    norm(x, images, groups, y, "silu")
    for first in range(0, images, 1 << 15):
        part = slice(first * rows, min(first + (1 << 15), images) * rows)
        R.check(y[part], *R.group_norm(x[part], len(x[part]) // rows, groups, 1e-5, None, None, "silu"), kind)


# (half as many threads a workgroup up to 4096 channels)
@pytest.mark.parametrize("C,images", [(8, 1 << 23), (4096, 1 << 23), (4097, 1 << 22), (8192, 1 << 22)])
def test_more_images_than_a_launch_holds_are_refused(C, images):
    far = 1 << 54
    refused(SHAPE, "too many", norm_call((C, 1, 1, 0, 1e-5), rows_at(1 << 20, C), rows_at(far, C), images, far * 2, 1 << 60))
