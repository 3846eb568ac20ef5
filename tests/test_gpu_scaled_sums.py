"""How the 8-bit float layers take their sums: in 32 bits for every result but bf16, in every kernel."""
import numpy as np
import pytest
import torch

import scaled_ref as R

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2507_19131_amd import binding as M

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


def product(x_codes, w_codes, kind):
    """Codes [rows, K] and [N, K] (values, with scales of 1) -> results as 64-bit values."""
    (rows, K), N = x_codes.shape, w_codes.shape[0]
    x, s_x = M.alloc_codes(rows, K)
    w, s_w = M.alloc_codes(N, K, 128)
    x.view(torch.uint8).copy_(x_codes.to(TYPES["e4m3"]).view(torch.uint8))
    w.view(torch.uint8).copy_(w_codes.to(TYPES["e4m3"]).view(torch.uint8))
    s_x.fill_(1.0)
    s_w.fill_(1.0)
    h = M.mixaq_scaled_linear_create(w, s_w)
    y, s_y = M.alloc_codes(rows, N) if kind == "e4m3" else (torch.empty((rows, N), dtype=TYPES[kind], device="cuda"), None)
    M.mixaq_scaled_linear_forward(h, x, y, x_scales=s_x, y_scales=s_y)
    torch.cuda.synchronize()
    M.mixaq_scaled_linear_destroy(h)
    v = y.cpu().double().numpy()
    return v if s_y is None else v * np.repeat(s_y.cpu().double().numpy().T, 128, 1)[:, :N]


def cancelling(rows, K, N):
    """In every eight neighbours 448 * 448 - 448 * 448 + 1 * a, a by the row, each product at places of its own: sums of a, and every partial sum of
    the products, in whatever order, is a whole number below 2^24."""
    x, w = torch.zeros((rows, K)), torch.zeros((N, K))
    for g in range(K // 8):
        p, q, r = (8 * g + (g + d) % 8 for d in (0, 3, 5))
        x[:, p], w[:, p] = 448.0, 448.0
        x[:, q], w[:, q] = 448.0, -448.0
        x[:, r], w[:, r] = 1.0 + torch.arange(rows) % 4, 1.0
    return x, w, (K // 8 * (1.0 + torch.arange(rows) % 4)).double().numpy()[:, None].repeat(N, 1)


# few rows; 32 x 32; 64 x 64; tiles of 128 x 128; large tiles
SIZES = [(1, 1024, 512), (40, 1000, 333), (700, 1504, 700), (2000, 256, 640), (6000, 128, 512), (8200, 400, 1500)]


@pytest.mark.parametrize("rows,K,N", SIZES)
@pytest.mark.parametrize("kind", ["f32", "f16", "e4m3"])
def test_small_products_beside_large_ones_that_cancel(rows, K, N, kind):
    x, w, want = cancelling(rows, K, N)
    got = product(x.cuda(), w.cuda(), kind)
    if kind == "e4m3":                                    # 448 times f32(a / 448), a code and a scale that are off by half a step of 32 bits
        assert np.all(np.abs(got - want) <= 2 * R.U * want)
    else:
        assert np.array_equal(got, want)


@pytest.mark.parametrize("rows,K,N", SIZES)
def test_bf16_results_keep_14_bits_of_a_group(rows, K, N):
    """What is lost is below 7 * 2^-13 of the largest product of each group; results that need no more bits are exact."""
    x, w, want = cancelling(rows, K, N)
    got = product(x.cuda(), w.cuda(), "bf16")
    assert np.all(np.abs(got - want) <= K // 8 * 7 * 2.0 ** -13 * 448 ** 2 + R.HALF_STEP["bf16"] * want)
    gen = torch.Generator().manual_seed(rows)
    x, w = (torch.randint(-1, 2, shape, generator=gen).float() for shape in ((rows, K), (N, K)))
    got = product(x.cuda(), w.cuda(), "bf16")
    want = (x.double() @ w.double().T).bfloat16().double().numpy()
    assert np.array_equal(got, want)
