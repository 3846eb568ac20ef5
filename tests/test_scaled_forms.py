"""Which kernel takes a linear layer in 8-bit float: both sides of every line of the rule, and that the sizes of the GPU tests reach every kernel in
every form.  CPU only."""
import pytest

import scaled_forms as S


def test_few_rows():
    assert S.form(16, 65536, 65536, "f32") == "few" and S.form(17, 65536, 65536, "f32") != "few"
    # tiles of 16 x 16 times blocks of K: 5000 and 1400 a block, at most 16384
    assert S.form(16 * 100, 128, 1024, "f32") == "few" and S.form(16 * 101, 128, 1024, "f32") != "few"           # 6400, 6464
    assert S.form(16 * 64, 2048, 256, "f32") == "few" and S.form(16 * 65, 2048, 256, "f32") == "mid"             # 16384, 16640


@pytest.mark.parametrize("kind", S.KINDS)
def test_tiles_of_32_64_and_128(kind):
    assert S.form(64 * 23, 2048, 512, kind) == "mid" and S.form(64 * 24, 2048, 512, kind) == "split"             # 184, 192 of 64 x 64
    assert S.form(128 * 23, 1024, 512, kind) == "split" and S.form(128 * 24, 1024, 512, kind) == "tile"          # 92, 96 of 128 x 128
    assert S.form(128 * 47, 33 * 128, 512, kind) == "split" and S.form(128 * 48, 33 * 128, 512, kind) != "split"           # 188, 192
    assert S.form(128 * 24, 32 * 128, 512, kind) == "tile"
    assert S.form(20000, 1024, 512, kind, ldx=(1 << 22) - 16) in ("tile", "large") and S.form(20000, 1024, 512, kind, ldx=1 << 22) == "split"


@pytest.mark.parametrize("gelu", [False, True])
def test_large_tiles(gelu):
    for kind in ("f32", "f16", "e4m3"):                                       # 256 x 128
        assert S.form(256 * 55, 384, 512, kind, gelu) == "tile" and S.form(256 * 56, 384, 512, kind, gelu) == "large"
        assert S.form(256 * 56, 256, 512, kind, gelu) == "tile"
    least = 6 if gelu else 2                                                  # 256 x 256
    assert S.form(256 * 95, 128 * least, 512, "bf16", gelu) == "tile" and S.form(256 * 96, 128 * least, 512, "bf16", gelu) == "large"
    assert S.form(256 * 96, 128 * (least - 1), 512, "bf16", gelu) == "tile"


@pytest.mark.parametrize("rows,K,N", S.SIZES)
def test_a_kernel_goes_by_its_sums_and_not_by_what_becomes_of_them(rows, K, N):
    """So 32-bit results, and the same results as codes, are one and the same."""
    for gelu in (False, True):
        assert len({S.form(rows, K, N, kind, gelu) for kind in ("f32", "f16", "e4m3")}) == 1


def test_values_are_quantized_inside_in_few_rows_alone():
    for rows in (1, 16, 17, 64, 256, 257, 1000, 5000):
        for K in (1, 128, 1024, 4096, 4097, 65536):
            for N in (1, 129, 1024, 65536):
                assert not S.inside(rows, K, N) or S.form(rows, K, N, "f32") == "few"
    # a workspace that serves some rows serves fewer
    for K, N in ((128, 128), (1024, 512), (4096, 4096), (700, 65536)):
        within = [S.inside(rows, K, N) for rows in range(1, 3000)]
        assert within == sorted(within, reverse=True)


@pytest.mark.parametrize("kind", S.KINDS)
@pytest.mark.parametrize("gelu", [False, True])
def test_the_sizes_compared_with_the_reference_reach_every_kernel(kind, gelu):
    """Every kernel, of every kind of results, with and without a GELU, with each way that K and N can end."""
    at = {name: [s for s in S.SIZES if S.form(*s, kind, gelu) == name] for name in S.NAMES}
    for name, sizes in at.items():
        assert any(K % 16 for _, K, _ in sizes), name                                 # inside 16 codes
        assert any(K % 128 and K % 16 == 0 for _, K, _ in sizes), name             # between two 16s of a block
        assert any(K % 128 == 0 for _, K, _ in sizes), name
        assert any(N % 128 for _, _, N in sizes) and any(rows % 32 for rows, _, _ in sizes), name
        assert any(N % 128 == 0 for _, _, N in sizes), name
        if name in ("few", "mid", "split"):
            assert any(K > 32 * 128 for _, K, _ in sizes), name
    assert any(S.blocks(N) % 2 for _, _, N in at["large"])


@pytest.mark.parametrize("kind", S.KINDS)
def test_the_sizes_that_tell_exact_sums_from_others_reach_every_kernel(kind):
    from test_gpu_scaled_sums import SIZES
    assert {S.form(*size, kind) for size in SIZES} == set(S.NAMES)


def test_the_bound_of_gelu_sees_small_mistakes():
    """What the bound must not let through: a tail that is cut off, erf from a three-term approximation, one coefficient's last digits."""
    import torch
    from test_gpu_scaled_forms import gelu, gelu_bound
    v = torch.linspace(-8.0, 8.0, 200001, dtype=torch.float64)
    want = gelu(v)
    bound = gelu_bound(v, want) + 2.0 ** -24 * want.abs()
    cut = torch.where(v < -4.2, torch.zeros_like(v), want)
    z = v.abs() * 0.5 ** 0.5
    t = 1.0 / (1.0 + 0.47047 * z)
    erf = 1.0 - (0.3480242 * t - 0.0958798 * t ** 2 + 0.7478556 * t ** 3) * torch.exp(-z * z)
    few = 0.5 * v * (1.0 + erf * torch.sign(v))

    def fit(first):                                       # the kernel's form, evaluated exactly
        u, p = v * v, 0.0
        for c in ("0x1.67ab6cp-28", "-0x1.9e7b64p-22", "0x1.80c28cp-17", "-0x1.4e76fep-13", "-0x1.8fb242p-14", "0x1.ad6ad0p-4"):
            p = p * u + float.fromhex(c)
        return v / (1.0 + torch.exp2(-v * (p * u + first)))

    first = float.fromhex("0x1.26aebcp+1")
    for wrong in (cut, few, fit(first * (1 + 2e-6))):
        assert bool(((wrong - want).abs() > bound).any())
    assert bool(((fit(first) - want).abs() <= bound).all())
