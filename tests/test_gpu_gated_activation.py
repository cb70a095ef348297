"""The activation of dr_qgated by itself, on gates that the products' sums hold exactly.

A gate is -M 2^p with a whole M of 24 bits: six products by 1 of 4-bit values, three in either of two blocks of 128 columns and 8
columns apart (of 12 bits in three products where there is one block alone), and up is a single product, so that neither kind of
sums rounds anything (fast sums drop nothing but within 8 columns).  What is left is what the interface promises of the
activation, (6 + |z|) 2^-23 of itself, and the rounding of its product with up to fp32, 2^-24.  Where e^-z passes 2^126 the result may
be 0; the border is taken 2^-10 of z early.
    Half of the gates lie evenly, the others are those of a million for which z would be furthest off if it were computed in
fp32 step by step.
"""
import numpy as np
import pytest
import torch

from oracle import gated, quant
from tests.gated_helpers import check_rows, poisoned, quantized
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

SILU, GELU = gated.SILU, gated.GELU_TANH


def _dr():
    from paper_2607_22614_amd import dr
    return dr


def _gates(kind, far, f):
    """f magnitudes of negative gates, in fp32."""
    many = np.random.default_rng(f).uniform(0.5 * far, far, 1000000).astype(np.float32)
    k1, k3 = gated.K[kind]
    c = -many
    square, c = (c * c).astype(np.float64), c.astype(np.float64)
    inner = (square * np.float32(k3 * np.log2(np.e)) + np.float32(k1 * np.log2(np.e))).astype(np.float32)
    off = np.abs((c * inner).astype(np.float32) - (k1 * c + k3 * c**3) * np.log2(np.e))
    off[gated.act(c, kind)[2] < -86.0] = 0.0
    return np.concatenate([np.linspace(far, far / f, f - f // 2), many[np.argsort(off)[-(f // 2):]] if f > 1 else []])


def _weights(dr, gates, k):
    """Fused weights of -gates and of up from 1 to 3.75, whose values are exact, and what the products with ones make of them."""
    f, bits = gates.size, 24 if k > 128 else 12
    mantissa, e = np.frexp(gates)
    m, p = np.minimum(np.round(mantissa * 2.0**bits).astype(np.int64), 2**bits - 1), e - bits
    up = np.tile(np.arange(4, 16), f // 12 + 1)[:f] * 0.25 * np.where(np.arange(f) % 2, 1.0, -1.0)
    codes = np.zeros((2 * f, -(-k // 128) * 128), dtype=np.uint8)
    scales = np.full((-(-codes.shape[1] // 512), 2 * f, 4), 127, dtype=np.uint8)
    for block, part in enumerate((m >> 12, m & 4095) if bits == 24 else (m,)):
        for col, four in ((0, part // 256 * 16.0), (8, part // 16 % 16 * 1.0), (16, part % 16 / 16.0)):
            codes[:f, 128 * block + col] = quant.round_e4m3(-four)
        scales[0, :f, block] = p + 4 + (12 if bits == 24 and block == 0 else 0) + 127
    codes[f:, 24] = quant.round_e4m3(up)
    w = dr.QMatrix(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 2 * f, k, 1)
    return w, -m * 2.0**p, up


# one row, few rows, some hundred of them, tiles of either size, of one block, of a CU alone, splits and their join
SHAPES = [(1, 3001, 128), (1, 3001, 256), (1, 400, 20000), (5, 2000, 256), (16, 5000, 1000), (40, 900, 256), (100, 1000, 1000), (600, 1000, 128),
          (1157, 4100, 640), (130, 600, 8192)]


@pytest.mark.parametrize("m,f,k", SHAPES)
@pytest.mark.parametrize("kind,far", [(SILU, 95.0), (GELU, 10.2)])
@pytest.mark.parametrize("fast", [False, True])
def test_negative_gates(m, f, k, kind, far, fast):
    dr = _dr()
    say("negative gates", m, f, k, kind, fast)
    w, gate, up = _weights(dr, _gates(kind, far, f), k)
    rows = 2.0**-(np.arange(m) % 3)
    x = torch.zeros((m, k), dtype=torch.float32)
    x[:, [0, 8, 16, 24] + ([128, 136, 144] if k > 128 else [])] = torch.from_numpy(rows).float()[:, None]
    out = torch.empty((m, f), device="cuda")
    workspace = torch.full((dr.dr_qgated_workspace(m, w),), 0xFF, dtype=torch.uint8, device="cuda")
    dr.dr_qgated(x.cuda(), w, out, act=kind, fast=fast, workspace=workspace)
    got = out.to(torch.float64).cpu().numpy()
    gate, up = rows[:, None] * gate, rows[:, None] * up
    a, _, z = gated.act(gate, kind)
    want = a * up
    allowed = ((6 + np.abs(z)) * 2.0**-23 + 2.0**-24) * (1 + 2.0**-20)
    lost = -z * (1 + 2.0**-10) > 126 * np.log(2.0)
    bad = ~(np.abs(got - want) <= allowed * np.abs(want) + 2.0**-149) & ~(lost & (got == 0))
    off = np.abs(got / np.where(want == 0, 1, want) - 1) * 2.0**23
    assert not bad.any(), (int(bad.sum()), gate[bad][:4], z[bad][:4], off[bad][:4], got[bad][:4])


@pytest.mark.parametrize("m,f", [(70, 5), (70, 100), (70, 120), (70, 128), (300, 384)])
@pytest.mark.parametrize("kind", [SILU, GELU])
def test_slopes_of_far_gates(m, f, kind):
    """Gates up to fp32's ends have slopes of 1 and 0, and gradients that fp32 holds are not NaN."""
    dr = _dr()
    say("slopes of far gates", m, f, kind)
    rng = np.random.default_rng(f)
    gate, gv = quantized(dr, rng.choice([1.0, -1.0, 1.5, -1.75], (m, f)) * 2.0**rng.choice([60, 100, 113, 114, 116, 120, 126], (m, 1)))
    up, uv = quantized(dr, rng.choice([1.0, -1.0, 0.75, 0.0], (m, f)))
    dh = rng.choice([1.0, -0.5, 0.625, 0.0], (m, f)).astype(np.float32)
    made = {"d": poisoned(dr, m, 2 * f), "dt": poisoned(dr, 2 * f, m), "ht": poisoned(dr, f, m)}
    dr.dr_gated_backward(torch.from_numpy(dh).cuda(), gate, up, **{n: v[0] for n, v in made.items()}, act=kind)
    torch.cuda.synchronize()
    # slopes and logistic functions are whole here, so that nothing but dh, up and gate is multiplied: 3 roundings at most, and
    # what is 2^-100 of the factors and below may count as 0
    a, _, _ = gated.act(gv, kind)
    dv = dh.astype(np.float64)
    d, h = np.concatenate(gated.backward(dv, gv, uv, kind), 1), a * uv
    tol = 3 * 2.0**-24
    check_rows(made["d"], d, tol * np.abs(d) + 2.0**-100, "d")
    check_rows(made["dt"], d.T, (tol * np.abs(d) + 2.0**-100).T, "dt")
    check_rows(made["ht"], h.T, (tol * np.abs(h) + 2.0**-100).T, "ht")
