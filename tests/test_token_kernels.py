"""Registers, LDS and scratch memory of the kernels of the int8 layers and of the group norm, from the built library's metadata.  CPU only."""
from test_kernel_resources import workgroups_per_cu
from test_scaled_kernels import kernels  # noqa: F401 (a fixture)


def found(kernels, name, at_least):  # noqa: F811
    k = {n: v for n, v in kernels.items() if name in n}
    assert len(k) >= at_least
    return k.items()


def test_no_kernel_uses_scratch_memory(kernels):  # noqa: F811
    """A launch with scratch memory takes longer, however little of it is used."""
    for name, count in (("token_few_kernel", 30), ("token_tile_kernel", 6), ("token_wide_kernel", 6), ("token_quantize", 33), ("group_small_kernel", 6), ("group_sums_kernel", 18), ("group_norm_kernel", 9)):
        for n, k in found(kernels, name, count):
            assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, n


def test_two_workgroups_of_tiles_share_a_cu(kernels):  # noqa: F811
    """One's end and the other's start then run beside products."""
    for name in ("token_tile_kernel", "token_wide_kernel"):
        for n, k in found(kernels, name, 6):
            assert workgroups_per_cu(k) == 2, n
