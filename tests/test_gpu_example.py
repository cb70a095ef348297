"""examples/eight_bit_roles.py: the 8-bit layers of both roles, the gradients' clipping and the staging between them.

Tolerances.  Codes are off by 2^-4 of an element at most, 2^-4 / sqrt(3) in the mean square, in both operands of two layers:
a logit is off by about 5 % of the logits' spread, which starts at 16 * 0.02 = 0.32 and stays of that order, so each
token's loss by about 0.02 and their mean by far less; 0.05 is allowed between the two roles.  A single token takes other
kernels than a prompt, whose sums differ by some 1e-5: now and then (0.3 %) an element of h rounds to its bf16 neighbour and
its code with it (2^-3 of an element up to 4, times weights of 0.1); 8 such elements of 256 are allowed for, 0.4.
"""
import os
import subprocess
import sys

import pytest
import torch

from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("tokens", [200, 77])
def test_both_roles(tokens):
    say("example", tokens)
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import eight_bit_roles
    finally:
        sys.path.pop(0)
    out = eight_bit_roles.run(tokens=tokens, steps=3, max_norm=0.5)
    losses = out["rollout_loss"]
    assert len(losses) == 4 and all(b < a for a, b in zip(losses, losses[1:]))
    assert all(abs(r - t) <= 0.05 for r, t in zip(losses, out["train_loss"]))
    assert max(out["token_matches"]) <= 0.4
    # the clipped gradients of the last step, each element rounded once to fp32
    total = sum(float((g.double() ** 2).sum()) for g in out["clipped"]) ** 0.5
    assert abs(total - min(0.5, out["norm"][-1])) <= 1e-5
    assert any(n > 0.5 for n in out["norm"])


def test_command():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "eight_bit_roles.py"), "--tokens", "64", "--steps", "1"],
                       capture_output=True, text=True, timeout=110, cwd=ROOT)
    assert r.returncode == 0, r.stderr
    assert r.stdout.startswith("step 0: rollout loss") and "step 1: rollout loss" in r.stdout
