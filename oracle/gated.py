"""The gated feed-forward block between its two linear layers, from its definition, in 64 bits on the CPU.

act        the activation, its slope, and the exponent z of its logistic function
forward    act(gate) * up
backward   the gradients of gate and up from the gradient of act(gate) * up
"""
from __future__ import annotations

import numpy as np

SILU, GELU_TANH = 0, 1
K = {SILU: (1.0, 0.0), GELU_TANH: (2.0 * np.sqrt(2.0 / np.pi), 2.0 * 0.044715 * np.sqrt(2.0 / np.pi))}


def act(g: np.ndarray, kind: int) -> tuple[np.ndarray, np.ndarray, np.ndarray]:
    k1, k3 = K[kind]
    z = k1 * g + k3 * g**3
    with np.errstate(over="ignore"):
        s = 1.0 / (1.0 + np.exp(-z))
        rest = 1.0 / (1.0 + np.exp(z))  # 1 - s without cancellation
    return g * s, s + g * s * rest * (k1 + 3.0 * k3 * g**2), z


def forward(gate: np.ndarray, up: np.ndarray, kind: int) -> np.ndarray:
    return act(gate, kind)[0] * up


def backward(dh: np.ndarray, gate: np.ndarray, up: np.ndarray, kind: int) -> tuple[np.ndarray, np.ndarray]:
    a, slope, _ = act(gate, kind)
    return dh * up * slope, dh * a
