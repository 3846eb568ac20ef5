"""Norms of rows whose mean is large beside their spread, against 64 bits."""
import numpy as np
import pytest
import torch

import scaled_ref as R

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2507_19131_amd import binding as M

EPS = float(np.float32(1e-5))
# Additions that a value goes through in a row's sum: up to 2 x 8 of a lane, 6 levels of a wave, 2 + 4 of the sums of sixteen waves.
DEPTH = 28
WIDTHS = [1, 5, 9, 96, 100, 129, 300, 384, 700, 1000, 1500, 3000, 4095, 5000, 9001, 16384]


def layer_norm(x):
    """The norm of 64-bit values that are 32-bit values, and how far 32-bit steps may be off.  The mean m is off by (DEPTH + 2) U of the mean size
    (sum, 1/C and their product); the values c behind it by U of their own size; what is left of m in them is found to (DEPTH + 2) U of the mean
    size of c, and their mean square, less that left squared, likewise; and a root, a quotient and three products follow."""
    U = R.U
    c = x - x.mean(1, keepdims=True)
    var = (c * c).mean(1, keepdims=True)
    r = 1.0 / np.sqrt(var + EPS)
    left = (DEPTH + 2) * U * np.abs(x).mean(1, keepdims=True)
    size = np.abs(c) + left
    off = 2 * U * size + (DEPTH + 3) * U * size.mean(1, keepdims=True)
    square = (DEPTH + 6) * U * (size * size).mean(1, keepdims=True)          # of the mean square
    turn = square / (2 * (var + EPS)) + 6 * U                                # of r, relative
    return c * r, r * off * (1 + turn) + np.abs(c * r) * turn + 2 * U * (np.abs(c * r) + r * left)


@pytest.mark.parametrize("C", WIDTHS)
def test_equal_values_leave_nothing(C):
    x = torch.tensor([1000.0, -1000.0, 1e6, 0.1, 3.0, 1234.567, -77777.7, 1e-3])[:, None].repeat(1, C)
    out = torch.empty((8, C), device="cuda")
    M.mixaq_residual_norm(M.make_residual_norm(C), x.cuda(), out=out)
    want, bound = layer_norm(x.double().numpy())
    assert np.all(np.abs(out.cpu().double().numpy() - want) <= bound), float(np.abs(out.cpu()).max())


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("spread", [1.0, 0.01])
def test_a_large_mean(C, spread):
    gen = torch.Generator().manual_seed(C)
    x = 1000.0 + spread * torch.randn((7, C), generator=gen)
    out, f = torch.empty((7, C), device="cuda"), x.cuda()
    M.mixaq_residual_norm(M.make_residual_norm(C), x.cuda(), out=out)
    want, bound = layer_norm(x.double().numpy())
    assert np.all(np.abs(out.cpu().double().numpy() - want) <= bound)
    y = torch.empty((7, C), device="cuda")                    # the norm behind a block: y = 0 x + norm(f)
    M.mixaq_residual_norm(M.make_residual_norm(C, post="layer", pre="none", residual_scale=0.0), torch.ones_like(f), f, y)
    assert np.all(np.abs(y.cpu().double().numpy() - want) <= bound)
