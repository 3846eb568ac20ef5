"""Which kernel takes a linear layer on int8 codes: both sides of each line, and that the sizes of the GPU tests reach every kernel.  CPU only."""
import pytest

import token_forms as S


def test_few_rows_and_few_tiles():
    assert S.form(16, 65536, 65536) == "few" and S.form(17, 4096, 65536) != "few"
    assert S.form(128, 1024, 1024) == "few" and S.form(144, 1024, 1024) == "mid"                              # 512 of 16 x 16
    assert S.form(256, 4096, 1024) == "mid" and S.form(257, 4096, 1024) == "few"                              # 256 of 32 x 32, of more than four blocks of K
    assert S.form(512, 512, 1024) == "mid" and S.form(513, 512, 1024) == "few"
    assert S.form(704, 1024, 1024) == "few" and S.form(705, 1024, 1024) == "split"                            # 192 of 64 x 64


def test_tiles():
    assert S.form(1408, 1024, 1024) == "split" and S.form(1409, 1024, 1024) == "tile"                         # 96 of 128 x 128
    assert S.form(8064, 1024, 1024) == "tile" and S.form(8065, 1024, 1024) == "wide"                          # 256 of 128 x 256
    assert S.form(70000, 128, 1024) == "tile" and S.form(70000, 129, 1024) == "wide" and S.form(70000, 1024, 128) == "tile"
    far = 1 << 25                                                                                             # bytes between rows: 128 of them are 4 GB
    assert S.form(20000, 1024, 1024, stride=far) == "split" and S.form(20000, 1024, 1024, stride=far - 16) == "wide"
    assert S.form(16, 1024, 1024, stride=far) == "few"


def test_rows_sorted_by_expert():
    assert S.form(32 * 17 - 1, 1024, 2048, 32) == "few" and S.form(32 * 17, 1024, 2048, 32) == "wide"
    assert S.form(31 * 17, 1024, 2048, 31) == "tile" and S.form(64 * 17, 128, 2048, 64) == "tile"
    assert S.form(64 * 17, 1024, 2048, 64, stride=1 << 22) == "split"                                         # 1088 rows of 4 MB: a tile's may be anywhere


def test_values_are_quantized_inside_in_few_rows_alone():
    assert S.inside(32, 1024, 4096) and not S.inside(33, 1024, 4096) and not S.inside(1, 1025, 128) and S.inside(1024, 1024, 128)
    assert S.inside(1, 8, 128) and not S.inside(1, 7, 128) and S.inside(1, 1024, 8192) and not S.inside(1, 1024, 8193)
    assert S.inside(64, 1024, 2048, 32) and not S.inside(65, 1024, 2048, 32) and not S.inside(64, 1024, 2049, 32) and not S.inside(64, 1024, 2048, 33)
    assert S.inside(64, 1024, 100, 4) and not S.inside(64, 1024, 100, 3) and S.inside(16, 1024, 100, 1) and not S.inside(17, 1024, 100, 1)
    assert not S.inside(1, 1024, 1 << 12, 1 << 12)
    for rows, K, N in S.SIZES:
        assert not S.inside(rows, K, N) or S.form(rows, K, N) == "few"
    for experts, rows, K, N, _ in S.SORTED:
        assert not S.inside(rows, K, N, experts) or S.form(rows, K, N, experts) == "few"
    assert any(S.inside(rows, K, N, experts) for experts, rows, K, N, _ in S.SORTED)


@pytest.mark.parametrize("sizes,experts", [(S.SIZES, False), (S.SORTED, True)])
def test_the_sizes_compared_with_the_reference_reach_every_kernel(sizes, experts):
    for name in S.NAMES:
        at = [s for s in sizes if (S.form(s[1], s[2], s[3], s[0]) if experts else S.form(*s)) == name]
        if experts and name in ("mid", "split"):
            assert not at                                                     # none, and rows that lie far apart
            continue
        K, N = [s[2 if experts else 1] for s in at], [s[3 if experts else 2] for s in at]
        assert at and any(k % 128 for k in K) and any(n % 128 for n in N), name
        if name in ("tile", "wide"):
            assert any(k % 64 for k in K) and any(n % 16 for n in N) and any(-(-n // 128) % 2 for n in N), name
