"""Gradient lists whose chunks are long ones, and lists that a norm takes in several launches, on the GPU against 64-bit sums.

Tolerance.  The squares are summed in fp64, so the norm is the oracle's rounded to fp32: one unit of 2^-24, and one more where
the two sums lie on either side of a tie.  Factor and product are held in fp64 and rounded once: 2^-24 relative and as
much for the oracle's norm, 2^-8 in bf16 (through fp32).
"""
import numpy as np
import pytest
import torch

from oracle import quant
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16
M = 1 << 20
LISTS = {"shards": [M + 3] * 9, "exact_chunks": [M] * 6, "small_first": [11] * 130 + [M + 3] * 9, "many": [(M >> 3) + 5] * 120 + [777] * 30,
         "one": [9 * M + 1]}


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


def _check(outs, norm, refs, max_norm):
    want_norm, want = quant.clip(refs, max_norm)
    assert abs(float(norm) - want_norm) <= 2 * 2.0**-24 * want_norm
    for o, w in zip(outs, want):
        tol = np.abs(w) * (2 * 2.0**-24 + (2.0**-8 if o.dtype == B else 0)) + 2.0**-149
        assert (np.abs(o.to(torch.float64).cpu().numpy() - w) <= tol).all()


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("types", [(F,), (B,), (F, B)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("offset", [0, 1])
def test_clip(name, types, offset):
    """To another place in either type, then in place."""
    from paper_2607_22614_amd import dr
    say("long lists", name, types, offset)
    grads = _grads(LISTS[name], types, 1, offset)
    refs = [g.to(torch.float64).cpu().numpy() for g in grads]
    norm = torch.empty((1,), device="cuda")
    for out_type in (F, B):
        outs = [torch.empty((g.numel() + offset,), dtype=out_type, device="cuda")[offset:] for g in grads]
        dr.dr_grad_clip(dr.GradList(grads, outs), 0.01, norm, _ws(dr))
        _check(outs, norm, refs, 0.01)
    dr.dr_grad_clip(dr.GradList(grads), 1e6, norm, _ws(dr))
    _check(grads, norm, refs, 1e6)
    dr.dr_grad_clip(dr.GradList(grads), 0.5, norm, _ws(dr))
    _check(grads, norm, refs, 0.5)


@pytest.mark.parametrize("name", LISTS)
def test_norm_repeats_itself(name):
    from paper_2607_22614_amd import dr
    say("norm", name)
    grads = dr.GradList(_grads(LISTS[name], (F, B), 2))
    want = sum(float((g.to(torch.float64)**2).sum()) for g in grads.grads)
    sums = [torch.empty((1,), dtype=torch.float64, device="cuda") for _ in range(3)]
    for s in sums:
        dr.dr_grad_norm(grads, _ws(dr), s)
    assert abs(float(sums[0]) - want) <= 1e-12 * want
    assert torch.equal(sums[0], sums[1]) and torch.equal(sums[0], sums[2])


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
