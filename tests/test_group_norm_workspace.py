"""The workspace of the group norm: one that is enough for many images is enough for fewer."""
import ctypes as C

import pytest
import torch

import token_ref as R
from paper_2507_19131_amd import binding as M

# C, groups, rows of an image: maps of one kernel and of two, one channel and the most, images of a single row
MAPS = [(128, 32, 65536), (256, 32, 49), (96, 32, 1), (1, 1, 5000), (8192, 1024, 700), (4104, 27, 333), (8, 1, 1 << 22)]


def size(channels, groups, rows_per_image, images):
    d, n = M.GroupNormDesc(channels, groups, rows_per_image, 0, 1e-5), C.c_size_t()
    assert M.load().mixaq_group_norm_workspace_bytes(C.byref(d), images * rows_per_image, C.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("channels,groups,rows_per_image", MAPS)
def test_more_images_need_no_less(channels, groups, rows_per_image):
    counts = [n for n in (*range(600), 1000, 1001, 4096, 1 << 20, (1 << 20) + 1, 1 << 30) if n * rows_per_image <= 1 << 30]
    sizes = [size(channels, groups, rows_per_image, n) for n in counts]
    assert sizes[0] == 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))


@pytest.mark.gpu
def test_fewer_images_in_the_workspace_of_many():
    """Of every count the workspace that its larger neighbour asks for, cut to those bytes; what lies behind keeps its pattern."""
    rows, channels, groups, most = 300, 40, 5, 300
    x = torch.randn(most * rows, channels, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    norm = M.make_group_norm(channels, groups, rows)
    for larger, images in ((300, 300), (300, 255), (256, 255), (300, 129), (129, 128), (128, 86), (8, 7), (4, 3), (4, 1)):
        n = M.mixaq_group_norm_workspace_bytes(norm, larger * rows)
        room = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        y = torch.empty_like(x[:images * rows])
        M.mixaq_group_norm(norm, x[:images * rows], y, workspace=room[:n])
        R.check(y, *R.group_norm(x[:images * rows], images, groups, 1e-5, None, None, "none"), "f32")
        assert bool((room[n:] == 0x5A).all())
