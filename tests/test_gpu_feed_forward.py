"""The gated block's operators together: a training pass from x and dy to dx and the weights' gradients, a rollout pass, and
examples/eight_bit_feed_forward.py.

Tolerance of the pass.  The same roundings to 8 bits and bf16 are made in 64 bits, so that results differ by fp32 sums alone,
which take an element across a rounding's border now and then: of one in a hundred elements of every rounded matrix (a
hundred times what sums off by 1e-5 of their norm do) by a whole step, 2^-3 of the element, sqrt(0.01) * 2^-3 = 1.3 % of the matrix's norm.  dx and
the gradients depend on at most four such matrices in a row (gate and up, dh, d, or h): 5 %; 2 % is asked for.
    The example's gradients are held against the block without any rounding.  A rounding to 8 bits is off by 2^-4 of an
element at most, by 2^-4 / sqrt(3) = 3.6 % in the mean square; a gradient passes through ten (x, the fused weights, gate, up, dy,
the down weights, dh in bf16, d, and x^T or h^T), 36 % if all pulled the same way, 11 % where they do not; 25 % is allowed, and between the roles too, whose
weights are rounded to 8 bits from fp32 and from bf16.  A single token takes other kernels than a prompt, whose sums differ as
those of the pass do: 2 %.
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import gated, quant
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import eight_bit_feed_forward
    finally:
        sys.path.pop(0)
    return eight_bit_feed_forward


def _eight(x, block_rows=1):
    codes, scales = quant.quantize(x, block_rows)
    return quant.values(codes, scales, x.shape[1], block_rows)


def _bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).to(torch.float64).numpy()


def _off(got, want):
    got = got.to(torch.float64).cpu().numpy()
    return np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("m,f,hidden,kind", [(200, 688, 256, gated.SILU), (130, 384, 128, gated.GELU_TANH), (77, 345, 200, gated.SILU), (40, 130, 136, gated.GELU_TANH)])
def test_training_pass(m, f, hidden, kind):
    say("feed-forward pass", m, f, hidden, kind)
    rng = np.random.default_rng(m)
    f32 = np.float32
    w, wd = (rng.standard_normal(s).astype(f32) / np.sqrt(s[1]).astype(f32) for s in ((2 * f, hidden), (hidden, f)))
    x, dy = (torch.from_numpy(rng.standard_normal((m, hidden)).astype(f32)).to(torch.bfloat16) for _ in range(2))
    dev = [torch.from_numpy(t).cuda() for t in (w, wd)]
    grads = [torch.zeros_like(t) for t in dev]
    block = _example().TrainedBlock(*dev, *grads, m, kind)
    block.take_weights()
    y = block.forward(x.cuda(), torch.empty((m, hidden), dtype=torch.bfloat16, device="cuda"))
    dx = block.backward(dy.cuda(), torch.empty((m, hidden), dtype=torch.bfloat16, device="cuda"), first=True)
    once = [g.clone() for g in grads]
    torch.cuda.synchronize()

    x, dy = x.to(torch.float64).numpy(), dy.to(torch.float64).numpy()
    wq, wdq, xq = _eight(w.astype(np.float64), 128), _eight(wd.astype(np.float64), 128), _eight(x)
    gate_up = xq @ wq.T
    h = _eight(gated.forward(gate_up[:, :f], gate_up[:, f:], kind))
    gate, up = _eight(gate_up[:, :f]), _eight(gate_up[:, f:])
    dh = _bf16(_eight(dy) @ wdq)
    d = np.concatenate(gated.backward(dh, gate, up, kind), axis=1)
    dt, ht, dyt, xt = (_eight(np.ascontiguousarray(t.T)) for t in (d, gated.forward(gate, up, kind), dy, xq))
    assert _off(y, h @ wdq.T) <= 0.02
    assert _off(dx, _eight(d) @ wq) <= 0.02
    assert _off(once[0], dt @ xt.T) <= 0.02
    assert _off(once[1], dyt @ ht.T) <= 0.02
    # a second micro-batch on top: the same sums once more, each rounded once
    block.backward(torch.from_numpy(dy).to(torch.bfloat16).cuda(), dx, first=False)
    for g, o in zip(grads, once):
        assert torch.equal(g, 2 * o)


@pytest.mark.parametrize("tokens,act", [(200, "silu"), (77, "gelu")])
def test_example(tokens, act):
    say("example", tokens, act)
    out = _example().run(tokens=tokens, steps=3, act=act)
    assert len(out["loss"]) == 3 and all(np.isfinite(v) for v in out["loss"])
    gate_up, down = (t.to(torch.float64).cpu().requires_grad_() for t in out["weights"])
    x = out["x"].to(torch.float64).cpu().requires_grad_()
    f = down.shape[1]
    y = x @ gate_up.t()
    gelu = torch.nn.functional.gelu(y[:, :f], approximate="tanh") if act == "gelu" else torch.nn.functional.silu(y[:, :f])
    ((gelu * y[:, f:]) @ down.t()).backward(out["dy"].to(torch.float64).cpu())
    for name, want in (("dx", x.grad), ("gate_up_grad", gate_up.grad), ("down_grad", down.grad)):
        assert _off(out[name], want.numpy()) <= 0.25, name
    # both roles run the same weights, the rollout in slices and from bf16
    assert _off(out["prompt_y"], out["trained_y"].to(torch.float64).cpu().numpy()) <= 0.25
    assert _off(out["token_y"], out["prompt_y"][-1:].to(torch.float64).cpu().numpy()) <= 0.02


def test_command():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "eight_bit_feed_forward.py"), "--tokens", "64", "--steps", "1"],
                       capture_output=True, text=True, timeout=110, cwd=ROOT)
    assert r.returncode == 0, r.stderr
    assert r.stdout.startswith("step 0: loss") and "rollout against training" in r.stdout
