"""The norm of gradient lists that take several launches, on the GPU against 64-bit sums."""
import pytest
import torch

from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16
M = 1 << 20


def _grads(sizes, types, seed, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        buf = torch.zeros((n + offset + 3,), dtype=types[i % len(types)], device="cuda")
        buf[offset:offset + n] = (torch.randn((n,), generator=gen, device="cuda") * 0.05).to(buf.dtype)
        out.append(buf[offset:offset + n])
    return out


def _ws(dr):
    return torch.full((dr.dr_grad_workspace(),), 0xFF, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("small", [[1] * 112, [3, 0] * 150, [17] * 500])
def test_a_large_tensor_behind_small_ones_has_as_many_workgroups(small):
    """Each workgroup of the norm leaves a sum in the workspace: 40 million elements are more chunks than 2048 workgroups take at once,
    wherever in the list they stand, and as many sums."""
    from paper_2607_22614_amd import dr
    say("small ones first", len(small))
    large = _grads([40 * M], (B,), 3)
    for before, behind in ((small, []), ([], small), (small, small)):
        lst = dr.GradList(_grads(before, (F,), 4) + large + _grads(behind, (F,), 5))
        ws, total = _ws(dr), torch.empty((1,), dtype=torch.float64, device="cuda")
        dr.dr_grad_norm(lst, ws, total)
        want = sum(float((g.to(torch.float64)**2).sum()) for g in lst.grads)
        assert abs(float(total) - want) <= 1e-12 * want
        written = (ws.view(torch.int64) != -1).nonzero().flatten()
        assert written.numel() == 2048 and int(written[-1]) == 2047
