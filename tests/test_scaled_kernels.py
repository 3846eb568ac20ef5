"""Registers and scratch memory of the kernels of the 8-bit float layers and norms, from the built library's metadata.  CPU only."""
import re

import pytest

from paper_2507_19131_amd import binding as M
from test_kernel_resources import _code_objects, _kernels


@pytest.fixture(scope="module")
def kernels():
    M.load()
    with open(M.lib_path(), "rb") as f:
        data = f.read()
    return {name: k for elf in _code_objects(data) for name, k in _kernels(elf)}


def test_products_keep_out_of_scratch_memory(kernels):
    """A launch with scratch memory takes longer, however little of it is used."""
    found = {n: k for n, k in kernels.items() if re.search("N_11(1tile|2split)_kernelILi", n)}
    assert len(found) >= 28
    for name, k in found.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name


def test_large_tiles_run_two_waves_a_simd_and_fit_the_lds(kernels):
    found = {n: k for n, k in kernels.items() if "N_111tile_kernelILi" in n}
    assert len(found) == 8
    for name, k in found.items():
        assert k[".vgpr_count"] + k.get(".agpr_count", 0) <= 512 and k[".group_segment_fixed_size"] <= 160 * 1024, name
        if k[".max_flat_workgroup_size"] == 256:                # two workgroups a CU
            assert 2 * k[".group_segment_fixed_size"] <= 160 * 1024 and k[".vgpr_count"] <= 256, name
        else:
            assert k[".vgpr_count"] <= 256, name


def test_norms_up_to_8192_channels_keep_out_of_scratch_memory(kernels):
    found = {n: k for n, k in kernels.items() if "residual_norm_kernel" in n}
    assert len(found) >= 81
    for name, k in found.items():
        if "Li1024ELi2" not in name:
            assert k[".vgpr_spill_count"] == 0, name
