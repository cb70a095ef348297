"""The oracle of the gated block: its activations against their usual forms, its gradients against differences."""
import math

import numpy as np
import pytest

from oracle import gated

G = np.concatenate([np.linspace(-12, 12, 4001), [0.0, -0.0, 1e-8, -40.0, 40.0]])


def test_activations():
    silu = np.array([g / (1 + math.exp(-g)) for g in G])
    gelu = np.array([0.5 * g * (1 + math.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g**3))) for g in G])
    assert np.allclose(gated.act(G, gated.SILU)[0], silu, rtol=1e-13, atol=1e-15)
    assert np.allclose(gated.act(G, gated.GELU_TANH)[0], gelu, rtol=1e-11, atol=1e-15)


@pytest.mark.parametrize("kind", [gated.SILU, gated.GELU_TANH])
def test_gradients_against_differences(kind):
    """Central differences are off by eps^2 / 6 times a third derivative (below 4 for both) and by 2^-52 |h| / eps."""
    rng = np.random.default_rng(kind)
    gate, up, dh = (rng.standard_normal(2000) * 3 for _ in range(3))
    eps = 1e-5
    dgate, dup = gated.backward(dh, gate, up, kind)
    by_gate = (gated.forward(gate + eps, up, kind) - gated.forward(gate - eps, up, kind)) / (2 * eps)
    by_up = (gated.forward(gate, up + eps, kind) - gated.forward(gate, up - eps, kind)) / (2 * eps)
    tol = np.abs(dh) * (eps**2 * np.abs(up) + 2.0**-50 * (1 + np.abs(gate * up)) / eps)
    assert (np.abs(dgate - dh * by_gate) <= tol).all()
    assert (np.abs(dup - dh * by_up) <= tol).all()
