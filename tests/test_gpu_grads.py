"""dr_grad_norm, dr_grad_scale and dr_grad_clip on the GPU against 64-bit sums.

Tolerance.  The squares are summed in fp64: n elements are off by at most n * 2^-53 relative, so the norm is the oracle's
rounded to fp32 (one unit of 2^-24, and one more where the two 64-bit sums lie on either side of a tie).  The factor is
rounded to fp32 once and each product once: 2 * 2^-24 relative, and 2^-8 of the result in bf16.
"""
import math

import numpy as np
import pytest
import torch

from oracle import quant
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def _dr():
    from paper_2607_22614_amd import dr
    return dr


def _grads(sizes, types, seed=0, sigma=0.05, offset=0):
    """Device tensors, `offset` elements into allocations of their own."""
    gen = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = types[i % len(types)]
        buf = torch.zeros((n + offset + 3,), dtype=t, device="cuda")
        buf[offset:offset + n] = (torch.randn((n,), generator=gen) * sigma).to(t).cuda()
        out.append(buf[offset:offset + n])
    return out


def _ws(dr):
    return torch.full((dr.dr_grad_workspace(),), 0xFF, dtype=torch.uint8, device="cuda")


def _check(outs, norm, refs, max_norm):
    want_norm, want = quant.clip([r.numpy() for r in refs], max_norm)
    assert abs(float(norm) - want_norm) <= 2 * 2.0**-24 * want_norm
    for o, w in zip(outs, want):
        tol = np.abs(w) * (3 * 2.0**-24 + (2.0**-8 if o.dtype == torch.bfloat16 else 0)) + 2.0**-149
        assert (np.abs(o.to(torch.float64).cpu().numpy() - w) <= tol).all()


F, B = torch.float32, torch.bfloat16
LISTS = {"none": [], "empty": [0, 0], "one": [1], "small": [1, 7, 8, 9, 0, 255, 2049], "chunks": [16384, 16383, 16385, 3],
         "long": [50000] * 5 + [11] * 300, "many": [13] * 1000, "shards": [1 << 20] * 4}


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("types", [(F,), (B,), (F, B)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("max_norm", [0.01, 1e6])
def test_clip_to_another_place(name, types, offset, max_norm):
    dr = _dr()
    say("clip", name, types, offset, max_norm)
    grads = _grads(LISTS[name], types, offset=offset)
    refs = [g.to(torch.float64).cpu() for g in grads]
    for out_type in (F, B):
        outs = [torch.empty((g.numel() + offset,), dtype=out_type, device="cuda")[offset:] for g in grads]
        norm = torch.full((1,), -1.0, device="cuda")
        dr.dr_grad_clip(dr.GradList(grads, outs), max_norm, norm, _ws(dr))
        torch.cuda.synchronize()
        _check(outs, norm, refs, max_norm)
    for g, r in zip(grads, refs):
        assert torch.equal(g.to(torch.float64).cpu(), r)


@pytest.mark.parametrize("types", [(F,), (B,), (F, B)], ids=["f32", "bf16", "mixed"])
def test_clip_in_place(types):
    dr = _dr()
    say("clip in place", types)
    for max_norm in (0.01, 1e6, math.inf):
        grads = _grads(LISTS["small"] + LISTS["chunks"], types, 3)
        refs = [g.to(torch.float64).cpu() for g in grads]
        norm = torch.empty((1,), device="cuda")
        dr.dr_grad_clip(dr.GradList(grads), max_norm, norm, _ws(dr))
        _check(grads, norm, refs, max_norm)


def test_parts_of_a_model_on_several_ranks():
    """Sums of squares of two parts, added as an all-reduce would, scale both by the norm of the whole; a part whose list
    is empty adds nothing."""
    dr = _dr()
    say("parts")
    parts = [_grads(LISTS["chunks"], (F,), 1), _grads(LISTS["many"], (B,), 2), []]
    refs = [[g.to(torch.float64).cpu() for g in p] for p in parts]
    sums = [torch.full((1,), -1.0, dtype=torch.float64, device="cuda") for _ in parts]
    for p, s in zip(parts, sums):
        dr.dr_grad_norm(dr.GradList(p), _ws(dr), sum_squares=s)
    whole = sum(sums)
    assert abs(float(whole) / sum(float((r**2).sum()) for p in refs for r in p) - 1) < 1e-12
    norms = [torch.empty((1,), device="cuda") for _ in parts]
    for p, n in zip(parts, norms):
        dr.dr_grad_scale(dr.GradList(p), whole, 0.5, n)
    assert float(norms[0]) == float(norms[1]) == float(norms[2])
    _check(parts[0] + parts[1], norms[0], refs[0] + refs[1], 0.5)


def test_norm_alone():
    dr = _dr()
    say("norm alone")
    for name in LISTS:
        grads = _grads(LISTS[name], (F, B), 5)
        s, n = torch.empty((1,), dtype=torch.float64, device="cuda"), torch.empty((1,), device="cuda")
        dr.dr_grad_norm(dr.GradList(grads), _ws(dr), s, n)
        want = sum(float((g.to(torch.float64)**2).sum()) for g in grads)
        assert abs(float(s) - want) <= 1e-12 * want and abs(float(n) - math.sqrt(want)) <= 2 * 2.0**-24 * math.sqrt(want)
        again = torch.empty_like(s)
        dr.dr_grad_norm(dr.GradList(grads), _ws(dr), again)
        assert torch.equal(s, again)


def test_extreme_and_non_finite_values():
    """Squares beyond fp32's range, values whose squares vanish in fp32, infinities and NaN."""
    dr = _dr()
    say("extremes")
    norm = torch.empty((1,), device="cuda")
    for big in (1e30, 1e-30, 3e38):
        g = torch.full((1000,), big, device="cuda")
        out = torch.empty_like(g)
        dr.dr_grad_clip(dr.GradList([g], [out]), 1e-3, norm, _ws(dr))
        _check([out], min(float(norm), 1e39), [g.to(torch.float64).cpu()], 1e-3) if big < 3e38 else None
        if big == 3e38:  # the norm passes fp32's largest, the factor does not suffer
            assert math.isinf(float(norm)) and abs(float(out[0]) / (1e-3 / math.sqrt(1000)) - 1) < 1e-6
    for bad, rest in ((math.inf, 0.0), (math.nan, math.nan)):
        g = torch.ones((300,), device="cuda")
        g[17] = bad
        dr.dr_grad_clip(dr.GradList([g]), 1.0, norm, _ws(dr))
        assert math.isnan(float(g[17])) and (torch.isnan(g).all() if math.isnan(rest) else int((g == 0).sum()) == 299)
        assert math.isinf(float(norm)) if math.isinf(bad) else math.isnan(float(norm))


def test_graph_replays_follow_the_gradients():
    dr = _dr()
    say("graph")
    grads = _grads(LISTS["long"], (F, B), 1)
    outs = [torch.empty((g.numel(),), device="cuda") for g in grads]
    lst, ws, norm = dr.GradList(grads, outs), _ws(dr), torch.empty((1,), device="cuda")
    dr.dr_grad_clip(lst, 0.1, norm, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dr.dr_grad_clip(lst, 0.1, norm, ws)
    for i in range(3):
        for g in grads:
            g.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        _check(outs, norm, [g.to(torch.float64).cpu() for g in grads], 0.1)


def test_more_than_2_to_the_32_elements():
    """One tensor past 32-bit offsets: its last elements count and are scaled."""
    dr = _dr()
    say("2^32 + 5 elements")
    n = (1 << 32) + 5
    g = torch.zeros((n,), dtype=torch.bfloat16, device="cuda")
    g[-3:] = 2.0
    g[1 << 31] = 2.0
    norm = torch.empty((1,), device="cuda")
    dr.dr_grad_clip(dr.GradList([g]), 1.0, norm, _ws(dr))
    assert float(norm) == 4.0
    assert (g[-3:] == 0.5).all() and float(g[1 << 31]) == 0.5 and float(g[-4]) == 0.0
