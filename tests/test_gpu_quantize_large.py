"""Calls large enough to be streamed whose rows are ragged inside an aligned stride, or aligned throughout."""
import pytest
import torch

from oracle import quant
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,stride", [(12800, 4101, 4104), (12800, 4104, 4112), (12801, 4100, 4104)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_large_strided_sources(rows, cols, stride, dtype, block_rows):
    """Rows alone, both ways and the transpose alone: the oracle's codes and scales at the matrix's ends and inside, the same
    from each call, and nothing of what lies between the rows."""
    from paper_2607_22614_amd import dr
    say("large, strided", rows, cols, stride, dtype, block_rows)
    gen = torch.Generator(device="cuda").manual_seed(cols)
    buf = torch.full((rows, stride), float("nan"), dtype=dtype, device="cuda")
    buf[:, :cols] = torch.randn((rows, cols), generator=gen, device="cuda").to(dtype)
    x = buf[:, :cols]
    q, qt = dr.QMatrix.empty(rows, cols, block_rows), dr.QMatrix.empty(cols, rows, block_rows)
    q1, qt1 = dr.QMatrix.empty(rows, cols, block_rows), dr.QMatrix.empty(cols, rows, block_rows)
    dr.dr_quantize(x, q, qt)
    dr.dr_quantize(x, q1)
    dr.dr_quantize(x, None, qt1)
    assert torch.equal(q.data, q1.data) and torch.equal(q.scales, q1.scales)
    assert torch.equal(qt.data, qt1.data) and torch.equal(qt.scales, qt1.scales)
    for m, src in ((q, x), (qt, x.t())):
        for at in (0, 128, src.shape[0] // 256 * 128, src.shape[0] // 128 * 128):
            ref = src[at:at + 128].to(torch.float64).cpu().numpy()
            codes, scales = quant.quantize(ref, block_rows)
            assert (m.data[at:at + 128].cpu().numpy() == codes).all()
            block = at // block_rows
            assert (m.scales[:, block:block + scales.shape[1]].cpu().numpy() == scales).all()
