"""Products that the kernel for few rows computes, with and without DR_FAST_SUMS: their sums lose no more than fp32 does.

Every eighth column holds 16 in both operands and the others 1/8, so that a group of 8 columns has one product of 2^8 and seven
of 2^-6: an addition that drops what lies below 2^-13 of the largest product's power of two loses all seven, 7 * 2^-6 of
a group, and K / 8 times that of a result.

Tolerance: that of the exact sums, (K padded to 128, and 64 to join partial sums) * 2^-23 * sum |a||b|.  For K up to 2000
that is below 3/4 of the loss.
"""
import pytest
import torch

from oracle import quant
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def _rows(rows, k, seed):
    """[rows, k]: 16 in the columns 0, 8, ..., else 1/8; each row times a power of two."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.full((rows, k), 0.125)
    x[:, ::8] = 16.0
    return x * torch.exp2(torch.randint(-2, 3, (rows, 1), generator=gen).float())


@pytest.mark.parametrize("m,n,k", [(1, 50, 128), (1, 4097, 2000), (4, 300, 520), (16, 16385, 264), (17, 300, 130), (32, 9300, 520),
                                   (64, 2000, 2000), (200, 688, 256)])
@pytest.mark.parametrize("fast", [False, True])
def test_small_products_beside_large_ones_count(m, n, k, fast):
    from paper_2607_22614_amd import dr
    say("few rows, small beside large", m, n, k, fast)
    x, w = _rows(m, k, 1), _rows(n, k, 2)
    want, size = quant.product(x.double().numpy(), w.double().numpy())
    tol = (-(-k // 128) * 128 + 64) * 2.0**-23 * size
    x_small, w_small = x.clone(), w.clone()
    x_small[:, ::8], w_small[:, ::8] = 0, 0
    assert (tol < 0.75 * quant.product(x_small.double().numpy(), w_small.double().numpy())[0]).all()
    a, b = dr.QMatrix.empty(m, k, 1), dr.QMatrix.empty(n, k, 128)
    dr.dr_quantize(x.cuda(), a), dr.dr_quantize(w.cuda(), b)
    out = torch.empty((m, n), device="cuda")
    ws = torch.empty((dr.dr_qmatmul_workspace(m, n, k),), dtype=torch.uint8, device="cuda")
    dr.dr_qmatmul(a, b, out, fast=fast, workspace=ws)
    assert (abs(out.double().cpu().numpy() - want) <= tol).all()
    y = torch.empty((m, n), device="cuda")
    ws = torch.empty((dr.dr_qlinear_workspace(m, b),), dtype=torch.uint8, device="cuda")
    dr.dr_qlinear(x.cuda(), b, y, fast=fast, workspace=ws)
    assert (abs(y.double().cpu().numpy() - want) <= tol).all()
