"""Every kernel of the 8-bit float layers, in every form, against 64 bits: on whole numbers, whose sums are exact in 32 bits whatever their order, so that
a product is right to the last bit or wrong."""
import numpy as np
import pytest
import torch

import scaled_forms as S
import scaled_ref as R

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2507_19131_amd import binding as M

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
FIT = 9.4e-8                      # how far the fit of GELU's Phi may be off, absolutely


def whole(gen, rows, cols, most):
    """Whole numbers up to `most` in size, as codes in GPU memory with a pattern (NaN) behind the columns."""
    codes = torch.full((rows, -(-cols // 16) * 16), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :cols]
    v = torch.randint(-most, most + 1, (rows, cols), generator=gen, device="cuda", dtype=torch.int8)
    codes.view(torch.uint8).copy_(v.float().to(torch.float8_e4m3fn).view(torch.uint8))
    return codes, v


def powers(gen, *shape):
    """Scales 0.5, 1 and 2."""
    return torch.exp2(torch.randint(-1, 2, shape, generator=gen, device="cuda").float())


def wide(scales, block_rows, rows, cols):
    return scales.t().repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols].double()


def gelu(v):
    return 0.5 * v * torch.special.erfc(-v * 0.5 ** 0.5)


def gelu_bound(v, y):
    """v times the fit of Phi.  And relative to the result: the logarithm of Phi's odds is off by 8 U of its size (seven steps and a product), which is
    below 0.75 v^2 + 2 left of zero, and right of it comes to 2.3 U at most; exponential, sum, reciprocal and product are off by a step (2 U) each.
    Below 2^-126 there is nothing."""
    return FIT * v.abs() + y.abs() * R.U * (8 * (0.75 * v * v + 2) * (v < 0) + 24) + 1e-37


class Product:
    def __init__(self, rows, K, N, with_gelu, most, seed, shrink=1.0, far=None, weights=None):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.rows, self.N, self.gelu = rows, N, with_gelu
        self.x, x = whole(gen, rows, K, most)
        w, wv = whole(gen, N, K, most)
        self.s_x = powers(gen, S.blocks(K), rows)
        s_w = powers(gen, S.blocks(K), S.blocks(N)) * shrink
        bias = torch.randint(-20, 21, (N,), generator=gen, device="cuda").float() * shrink if seed % 3 else None
        assert most * most * K * 16 + 80 < 2 ** 24                          # of steps of a quarter: every partial sum is exact
        self.h = M.mixaq_scaled_linear_create(w, s_w, bias, "gelu" if with_gelu else "none")
        self.w64 = wv.double() * wide(s_w, 128, N, K)
        self.x64 = lambda a, b: x[a:b].double() * wide(self.s_x[:, a:b], 1, b - a, K)
        self.bias = 0.0 if bias is None else bias.double()
        if far:                                                             # the same rows far apart
            room = torch.empty(rows * far, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).as_strided((rows, K), (far, 1))
            room.view(torch.uint8).copy_(self.x.view(torch.uint8))
            self.x = room

    def run(self, kind):
        y, s_y = M.alloc_codes(self.rows, self.N) if kind == "e4m3" else (torch.empty((self.rows, self.N), dtype=TYPES[kind], device="cuda"), None)
        M.mixaq_scaled_linear_forward(self.h, self.x, y, x_scales=self.s_x, y_scales=s_y)
        return y, s_y

    def sums(self, a, b):
        return self.x64(a, b) @ self.w64.t() + self.bias

    def check(self, kind, step=8192):
        y, s_y = self.run(kind)
        for a in range(0, self.rows, step):
            b = min(a + step, self.rows)
            v, got = self.sums(a, b), y[a:b]
            if not self.gelu and kind != "e4m3":
                assert torch.equal(got, v.to(TYPES[kind])), (a, int((got != v.to(TYPES[kind])).sum()))
            elif not self.gelu:
                codes, scales = R.quantize(v.float().cpu().numpy())
                assert np.array_equal(got.view(torch.uint8).cpu().numpy(), codes) and np.array_equal(s_y[:, a:b].cpu().double().numpy(), scales)
            else:
                want = gelu(v)
                bound = gelu_bound(v, want)
                if kind == "e4m3":
                    R.check_codes(got.view(torch.uint8).cpu().numpy(), s_y[:, a:b].cpu().double().numpy(), want.cpu().numpy(), bound.cpu().numpy())
                else:
                    off = (got.double() - want).abs() / (bound + R.HALF_STEP[kind] * (want.abs() + bound) + R.LEAST_STEP[kind])
                    assert float(off.max()) <= 1.0, (a, float(off.max()))

    def close(self):
        M.mixaq_scaled_linear_destroy(self.h)


@pytest.mark.parametrize("kind", S.KINDS)
@pytest.mark.parametrize("with_gelu", [False, True])
@pytest.mark.parametrize("rows,K,N", S.SIZES)
def test_whole_numbers(rows, K, N, with_gelu, kind):
    """(With a GELU the sums are made smaller, to a root mean square of about 3.)"""
    shrink = 2.0 ** -round(np.log2(25.0 * K ** 0.5)) if with_gelu else 1.0
    p = Product(rows, K, N, with_gelu, 15, rows + K + N, shrink)
    p.check(kind)
    p.close()


@pytest.mark.parametrize("kind", S.KINDS)
@pytest.mark.parametrize("rows,K,N", [(3000, 200, 512), (40, 300, 100)])
def test_rows_four_megabytes_apart(rows, K, N, kind):
    """Which the tiles leave to other kernels, since they count in 32 bits; on both sides of that line."""
    for far in ((1 << 22) - 16, 1 << 22, (1 << 22) + 16):
        p = Product(rows, K, N, False, 15, rows, far=far)
        p.check(kind)
        p.close()
        del p
    assert S.form(rows, K, N, kind, ldx=1 << 22) in ("split", "few")


@pytest.mark.parametrize("rows,K,N", [(1, 65536, 300), (200, 65536, 300), (2000, 65535, 600), (13000, 65536, 250), (57400, 65536, 250)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_the_deepest_products(rows, K, N, kind):
    """512 blocks of K: in every kernel."""
    assert S.form(rows, K, N, kind) == {1: "few", 200: "mid", 2000: "split", 13000: "tile", 57400: "large"}[rows]
    p = Product(rows, K, N, False, 3, rows)
    p.check(kind, 2048)
    p.close()


@pytest.mark.parametrize("rows", [2000, 300000])
def test_gelu_of_any_value(rows):
    """One code of 1 times one weight of 1, scaled by any number: the activation alone, in the kernel of few rows and in a tile."""
    far = torch.tensor([0.0, -0.0, 1e-45, -1e-45, 2e-38, -2e-38, 1e-20, -1e-20, 7.0, -7.0, 13.0, -13.0, 40.0, -40.0, 1e19, -1e19, 2e19, -2e19, 3.4e38, -3.4e38])
    v = torch.cat([far, torch.linspace(-14.0, 14.0, rows - len(far))]).cuda()
    codes, _ = M.alloc_codes(rows, 1)
    codes.view(torch.uint8).fill_(0x38)
    w, s_w = M.alloc_codes(16, 1, 128)
    w.view(torch.uint8).fill_(0x38)
    s_w.fill_(1.0)
    h = M.mixaq_scaled_linear_create(w, s_w, None, "gelu")
    y = torch.empty((rows, 16), device="cuda")
    M.mixaq_scaled_linear_forward(h, codes, y, x_scales=v[None])
    assert bool((y == y[:, :1]).all())
    want = gelu(v.double())
    want = torch.where(v > 40, v.double(), want)             # (0.5 times them passes no border)
    off = (y[:, 0].double() - want).abs() - gelu_bound(v.double().clamp(-1e3, 1e3), want) - R.HALF_STEP["f32"] * want.abs()
    assert float(off.max()) <= 0.0, float(v[off.argmax()])
    v[0], v[1], v[2] = float("inf"), float("-inf"), float("nan")
    M.mixaq_scaled_linear_forward(h, codes, y, x_scales=v[None])
    M.mixaq_scaled_linear_destroy(h)
    assert bool((y[0] == float("inf")).all()) and bool((y[1] == 0).all()) and bool(y[2].isnan().all())
