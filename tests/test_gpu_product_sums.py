"""Every product counts once, and what the sums lose is what dr.h says, on each of the products' kernels.

Whole numbers from -3 to 3 are exact in e4m3 and so are their products; their sums stay below 9 K < 2^24, and within 8 columns no
product is 2^-13 of another, so that exact and fast sums are both equal to the product's, and a bf16 result is that
rounded once.  For normal values the norm of the error is compared with the result's: fast sums lose 1.5e-5 of it (2e-5
allows for the inputs), exact ones round K / 16 times at most, by 2^-24 of a partial sum no larger than the result
as a rule, with signs of their own: 2^-24 * sqrt(K / 16), and twice that is allowed.
"""
import pytest
import torch

from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

# few rows, quantized inside or not; small products; one block of columns; a tile to a CU; splits; 256 x 256; quarters
SHAPES = [(3, 500, 700), (16, 5000, 5120), (31, 4100, 1000), (33, 6912, 5120), (64, 2000, 2000), (200, 688, 256), (300, 1000, 128), (301, 1001, 100),
          (512, 6912, 5120), (777, 9728, 896), (777, 9729, 896), (1200, 2000, 2000), (2600, 2600, 300), (4100, 4360, 5120), (5000, 7000, 640)]


def _matrices(x, w):
    from paper_2607_22614_amd import dr
    (m, k), n = x.shape, w.shape[0]
    a, b = dr.QMatrix.empty(m, k, 1), dr.QMatrix.empty(n, k, 128)
    dr.dr_quantize(x, a), dr.dr_quantize(w, b)
    return dr, a, b, torch.empty((dr.dr_qmatmul_workspace(m, n, k),), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("fast", [False, True])
def test_whole_numbers(m, n, k, fast):
    say("whole numbers", m, n, k, fast)
    gen = torch.Generator(device="cuda").manual_seed(m + n + k)
    x, w = (torch.randint(-3, 4, (rows, k), generator=gen, device="cuda").to(torch.bfloat16) for rows in (m, n))
    dr, a, b, ws = _matrices(x, w)
    want = x.double() @ w.double().t()
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((m, n), 7.0, dtype=dtype, device="cuda")
        dr.dr_qmatmul(a, b, out, fast=fast, workspace=ws)
        assert torch.equal(out, want.to(torch.float32).to(dtype))
    out = torch.full((m, n), 7.0, device="cuda")
    dr.dr_qmatmul(a, b, out, accumulate=True, fast=fast, workspace=ws)
    assert torch.equal(out.double(), want + 7.0)
    y = torch.empty((m, n), device="cuda")
    dr.dr_qlinear(x, b, y, fast=fast, workspace=torch.empty((dr.dr_qlinear_workspace(m, b),), dtype=torch.uint8, device="cuda"))
    assert torch.equal(y.double(), want)


def _values(q):
    scales = torch.exp2(q.scales.permute(0, 2, 1).reshape(-1, q.scales.shape[1]).t().double() - 127)[:, :q.data.shape[1] // 128]
    full = scales.repeat_interleave(q.block_rows, 0)[:q.rows].repeat_interleave(128, 1)
    return (q.data.view(torch.float8_e4m3fn).double() * full)[:, :q.cols]


@pytest.mark.parametrize("m,n,k", [s for s in SHAPES if s[0] * s[1] > 1 << 18])
def test_normal_values(m, n, k):
    """The same result each time, too."""
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    x, w = (torch.randn((rows, k), generator=gen, device="cuda") for rows in (m, n))
    dr, a, b, ws = _matrices(x, w)
    want = _values(a) @ _values(b).t()
    for fast, bound in ((True, 2e-5), (False, 2 * 2.0**-24 * (k / 16)**0.5)):
        say("normal values", m, n, k, fast)
        out, again = torch.empty((m, n), device="cuda"), torch.empty((m, n), device="cuda")
        dr.dr_qmatmul(a, b, out, fast=fast, workspace=ws)
        dr.dr_qmatmul(a, b, again, fast=fast, workspace=ws)
        assert torch.equal(out, again)
        assert float((out - want).norm()) <= bound * float(want.norm())
