"""Products into rows that begin 16 MiB apart, a little less and more, and into results of 64 GiB.

All values are -1, 0 and 1, so that every sum is a whole number below 2^8, which fp32 and bf16 hold: results are equal to the
product's, whatever the order of the sums.
"""
import pytest
import torch

from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def _operands(m, n, k):
    from paper_2607_22614_amd import dr
    gen = torch.Generator(device="cuda").manual_seed(m + n + k)
    x, w = (torch.randint(-1, 2, (rows, k), generator=gen, device="cuda", dtype=torch.int8).to(torch.bfloat16) for rows in (m, n))
    a, b = dr.QMatrix.empty(m, k, 1), dr.QMatrix.empty(n, k, 128)
    dr.dr_quantize(x, a), dr.dr_quantize(w, b)
    return dr, x, w, a, b


@pytest.mark.parametrize("m,n,k", [(5, 300, 250), (40, 1000, 250), (300, 1000, 250), (300, 520, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("more", [-16, 0, 16])
def test_rows_far_apart(m, n, k, dtype, more):
    """16 MiB and `more` bytes from row to row; nothing beside c's columns is written."""
    say("rows far apart", m, n, k, dtype, more)
    dr, x, w, a, b = _operands(m, n, k)
    stride = ((1 << 24) + more) // dtype.itemsize
    buf = torch.full((m, stride), 3.0, dtype=dtype, device="cuda")
    out = buf[:, 8:8 + n]
    want = x.float() @ w.float().t()
    ws = torch.empty((dr.dr_qmatmul_workspace(m, n, k),), dtype=torch.uint8, device="cuda")
    dr.dr_qmatmul(a, b, out, workspace=ws)
    assert torch.equal(out.float(), want)
    if dtype == torch.float32:
        dr.dr_qmatmul(a, b, out, accumulate=True, fast=True, workspace=ws)
        assert torch.equal(out, 2 * want)
    assert (buf[:, :8] == 3.0).all() and (buf[:, 8 + n:] == 3.0).all()


def test_more_workgroups_than_a_launch_holds():
    """2^35 results: 2^24 workgroups of 256 lanes of the kernel for few rows, 2^32 lanes."""
    m, n, k = 4096, 1 << 23, 128
    say("64 GiB of results", m, n, k)
    dr, x, w, a, b = _operands(m, n, k)
    out = torch.full((m, n), 3.0, dtype=torch.bfloat16, device="cuda")
    dr.dr_qmatmul(a, b, out, workspace=torch.empty((dr.dr_qmatmul_workspace(m, n, k),), dtype=torch.uint8, device="cuda"))
    x = x.float()
    step = 1 << 18
    for at in range(0, n, step):
        assert torch.equal(out[:, at:at + step].float(), x @ w[at:at + step].float().t()), at
