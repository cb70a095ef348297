"""dr_gated_backward and dr_qtranspose on the GPU, against 64 bits of the values that the codes stand for.

Tolerance of the gradients: the logistic function is off by (6 + |z|) 2^-23 of itself, and each further product or sum by
2^-24; the terms of act's slope add their own.  2^-100 of the factors
where the exponential passes 2^126; from |z| = 150 on the logistic function is 0 or 1.  Turning a matrix loses nothing.
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


def _want(dh, gate, up, kind):
    """[dgate dup], act(gate) * up, and their tolerances."""
    a, slope, z = gated.act(gate, kind)
    dgate, dup = gated.backward(dh, gate, up, kind)
    k1, k3 = gated.K[kind]
    with np.errstate(over="ignore"):
        s, rest = 1.0 / (1.0 + np.exp(-z)), 1.0 / (1.0 + np.exp(z))
    parts = s + np.abs(a) * rest * (k1 + 3 * k3 * gate**2)
    rel, cut = (12 + 3 * np.minimum(np.abs(z), 150)) * 2.0**-23, 2.0**-100
    t_gate = np.abs(dh * up) * (rel * parts + cut)
    t_up, t_h = np.abs(dh) * (rel * np.abs(a) + cut), np.abs(up) * (rel * np.abs(a) + cut)
    return np.concatenate([dgate, dup], 1), a * up, np.concatenate([t_gate, t_up], 1), t_h


def _inputs(dr, m, f, dtype, seed):
    rng = np.random.default_rng(seed)
    gate, gv = quantized(dr, rng.standard_normal((m, f)) * 2.0**rng.integers(-2, 4, (m, 1)), 1, 16)
    up, uv = quantized(dr, rng.standard_normal((m, f)) * 2.0**rng.integers(-20, 9, (m, 1)), 1, 32)
    dh = (rng.standard_normal((m, f)) * 2.0**rng.integers(-24, 1, (m, 1))).astype(np.float32)
    if m > 3:
        dh[m // 3] = 0.0
    dh = torch.from_numpy(dh).to(dtype)
    return gate, up, dh, gv, uv, dh.to(torch.float64).numpy()


SHAPES = [(1, 1), (1, 128), (3, 5), (2, 129), (128, 128), (129, 256), (200, 344), (77, 130), (300, 127), (130, 384), (257, 1001)]


@pytest.mark.parametrize("m,f", SHAPES)
@pytest.mark.parametrize("kind,dtype", [(SILU, torch.bfloat16), (GELU, torch.float32)])
def test_gradients(m, f, kind, dtype):
    dr = _dr()
    gate, up, dh, gv, uv, dv = _inputs(dr, m, f, dtype, m * 1000 + f)
    d, h, t_d, t_h = _want(dv, gv, uv, kind)
    for which in ("d dt ht", "d", "dt", "ht", "d ht", "dt ht", "d dt"):
        say("backward", m, f, kind, dtype, which)
        made = {"d": poisoned(dr, m, 2 * f), "dt": poisoned(dr, 2 * f, m), "ht": poisoned(dr, f, m)}
        dr.dr_gated_backward(dh.cuda(), gate, up, **{n: made[n][0] for n in which.split()}, act=kind)
        torch.cuda.synchronize()
        for name in which.split():
            want, tol = {"d": (d, t_d), "dt": (d.T, t_d.T), "ht": (h.T, t_h.T)}[name]
            check_rows(made[name], want, tol, name)


@pytest.mark.parametrize("f", [128, 130])
@pytest.mark.parametrize("offset,stride", [(1, 301), (8, 304), (3, 512)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_at_any_element(f, offset, stride, dtype):
    dr = _dr()
    say("backward at", f, offset, stride, dtype)
    m = 70
    gate, up, dh, gv, uv, dv = _inputs(dr, m, f, dtype, 5)
    buf = torch.full((offset + m * stride,), float("nan"), dtype=dtype, device="cuda")
    src = buf[offset:].view(m, stride)[:, :f]
    src.copy_(dh)
    made = {"d": poisoned(dr, m, 2 * f), "dt": poisoned(dr, 2 * f, m)}
    dr.dr_gated_backward(src, gate, up, made["d"][0], made["dt"][0])
    torch.cuda.synchronize()
    d, _, t_d, _ = _want(dv, gv, uv, SILU)
    check_rows(made["d"], d, t_d, "d")
    check_rows(made["dt"], d.T, t_d.T, "dt")


def test_rows_far_apart():
    """Rows of dh 2^24 bytes and more apart, beyond the offsets of the kernel for whole tiles."""
    dr = _dr()
    say("backward, rows far apart")
    m, f, stride = 3, 256, (1 << 23) + 8
    gate, up, dh, gv, uv, dv = _inputs(dr, m, f, torch.bfloat16, 6)
    buf = torch.zeros((m - 1) * stride + f, dtype=torch.bfloat16, device="cuda")
    src = buf.as_strided((m, f), (stride, 1))
    src.copy_(dh)
    made = {"d": poisoned(dr, m, 2 * f), "dt": poisoned(dr, 2 * f, m), "ht": poisoned(dr, f, m)}
    dr.dr_gated_backward(src, gate, up, **{n: v[0] for n, v in made.items()})
    torch.cuda.synchronize()
    d, h, t_d, t_h = _want(dv, gv, uv, SILU)
    check_rows(made["d"], d, t_d, "d")
    check_rows(made["dt"], d.T, t_d.T, "dt")
    check_rows(made["ht"], h.T, t_h.T, "ht")


# more tiles than the CUs hold three times, bands of sixteen tiles that are cut off, inputs that are streamed
@pytest.mark.parametrize("m,f,dtype", [(2200, 1408, torch.bfloat16), (1700, 1500, torch.float32), (4100, 4224, torch.float32), (900, 2051, torch.bfloat16)])
def test_large(m, f, dtype):
    dr = _dr()
    say("large backward", m, f, dtype)
    gen = torch.Generator(device="cuda").manual_seed(m)
    gate, up = dr.QMatrix.empty(m, f), dr.QMatrix.empty(m, f)
    for q in (gate, up):
        dr.dr_quantize(torch.randn((m, f), generator=gen, device="cuda") * torch.exp2(torch.randn((m, 1), generator=gen, device="cuda")), q)
    gv, uv = (quant.values(q.data.cpu().numpy(), q.scales.cpu().numpy(), f, 1) for q in (gate, up))
    dh = (torch.randn((m, f), generator=gen, device="cuda") * 1e-3).to(dtype)
    made = {"d": poisoned(dr, m, 2 * f), "dt": poisoned(dr, 2 * f, m), "ht": poisoned(dr, f, m)}
    dr.dr_gated_backward(dh, gate, up, **{n: v[0] for n, v in made.items()}, act=GELU)
    torch.cuda.synchronize()
    d, h, t_d, t_h = _want(dh.to(torch.float64).cpu().numpy(), gv, uv, GELU)
    check_rows(made["d"], d, t_d, "d")
    check_rows(made["dt"], d.T, t_d.T, "dt")
    check_rows(made["ht"], h.T, t_h.T, "ht")


@pytest.mark.parametrize("m,f", [(33000, 131072), (131072, 33003)])
def test_matrices_of_more_than_4_gib(m, f):
    """Elements at the beginning, around 2^32 bytes and at the end of every matrix."""
    dr = _dr()
    say("large matrices", m, f)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def random(rows, cols):
        q = dr.QMatrix.empty(rows, cols)
        q.data.random_(0, 100, generator=gen)
        q.data[:, cols:] = 0
        q.scales.random_(118, 124, generator=gen)
        return q

    def values(q, rows, cols):
        per = q.scales[cols[0] // 512:(cols[-1]) // 512 + 1, rows].permute(1, 0, 2).reshape(len(rows), -1).cpu().numpy()
        per = per[:, (cols // 128) - cols[0] // 512 * 4]
        scale = 2.0**(per - 127.0)
        return quant.E4M3[q.data[rows][:, cols].cpu().numpy()] * scale, scale

    gate, up = random(m, f), random(m, f)
    dh = torch.randn((m, f), generator=gen, device="cuda", dtype=torch.bfloat16)
    d, dt, ht, gt = dr.QMatrix.empty(m, 2 * f), dr.QMatrix.empty(2 * f, m), dr.QMatrix.empty(f, m), dr.QMatrix.empty(f, m)
    dr.dr_gated_backward(dh, gate, up, d, dt, ht)
    dr.dr_qtranspose(gate, gt)
    torch.cuda.synchronize()
    for r0 in (0, (1 << 32) // f // 128 * 128, (m - 1) // 128 * 128):
        for c0 in (0, (1 << 32) // m // 128 * 128, (f - 1) // 128 * 128):
            rows, cols = np.arange(r0, min(r0 + 128, m)), np.arange(c0, min(c0 + 128, f))
            gv, uv = values(gate, rows, cols)[0], values(up, rows, cols)[0]
            want, h, t_d, t_h = _want(dh[rows][:, cols].to(torch.float64).cpu().numpy(), gv, uv, SILU)
            n = len(cols)
            for q, i, j, w, t in ((d, rows, cols, want[:, :n], t_d[:, :n]), (d, rows, cols + f, want[:, n:], t_d[:, n:]),
                                  (dt, cols, rows, want[:, :n].T, t_d[:, :n].T), (dt, cols + f, rows, want[:, n:].T, t_d[:, n:].T),
                                  (ht, cols, rows, h.T, t_h.T), (gt, cols, rows, gv.T, 0.0)):
                got, scale = values(q, i, j)
                assert (np.abs(got - w) <= np.maximum(2.0**-4 * np.abs(w), 2.0**-10 * scale) * (1 + 2.0**-20) + 2 * t).all()


@pytest.mark.parametrize("f", [128, 100])
@pytest.mark.parametrize("kind", [SILU, GELU])
def test_far_and_not_finite(f, kind):
    """Gates from -2^40 to 2^40 give slopes of 1 and 0; what is not finite becomes NaN and leaves its block's scale alone."""
    dr = _dr()
    say("backward, far", f, kind)
    m = 40
    rng = np.random.default_rng(1)
    gate, gv = quantized(dr, rng.choice([0.0, -0.0, 1.0, -1.0, 30.0, -30.0, 100.0, -100.0, 150.0, -150.0, 2.0**14, -2.0**14, 2.0**40, -2.0**40], (m, f)))
    up, uv = quantized(dr, rng.choice([1.0, -2.0, 0.0, 0.75], (m, f)))
    dh = rng.standard_normal((m, f)).astype(np.float32)
    made = {"d": poisoned(dr, m, 2 * f), "dt": poisoned(dr, 2 * f, m), "ht": poisoned(dr, f, m)}
    args = {n: v[0] for n, v in made.items()}
    dr.dr_gated_backward(torch.from_numpy(dh).cuda(), gate, up, **args, act=kind)
    d, h, t_d, t_h = _want(dh.astype(np.float64), gv, uv, kind)
    check_rows(made["d"], d, t_d, "d")
    check_rows(made["dt"], d.T, t_d.T, "dt")
    check_rows(made["ht"], h.T, t_h.T, "ht")
    gate.data[7, 3] = 0x7F
    up.data[9, 4] = 0xFF
    dh[11, 5], dh[12, 6] = np.inf, np.nan
    gv[7, 3] = uv[9, 4] = np.nan
    dr.dr_gated_backward(torch.from_numpy(dh).cuda(), gate, up, **args, act=kind)
    d, h, t_d, t_h = _want(dh.astype(np.float64), gv, uv, kind)
    # inf times a zero of the slope or of up is NaN, which is no number either
    d[11, [5, 5 + f]] = np.nan
    check_rows(made["d"], d, t_d, "d")
    check_rows(made["dt"], d.T, t_d.T, "dt")
    check_rows(made["ht"], h.T, t_h.T, "ht")


@pytest.mark.parametrize("f", [128, 90])
@pytest.mark.parametrize("kind", [SILU, GELU])
def test_ends_of_fp32(f, kind):
    """Gradients among fp32's subnormals, where a scale is no less than 2^-127 and a product is off by up to 2^-149 each time; and
    such that pass its largest number, which become NaN."""
    dr = _dr()
    say("backward, ends of fp32", f, kind)
    m = 24
    rng = np.random.default_rng(4)
    gate, gv = quantized(dr, rng.standard_normal((m, f)))
    up, uv = quantized(dr, rng.choice([1.0, -0.5, 0.25, 2.0], (m, f)) * np.where(np.arange(m) < 16, 1.0, 2.0**60)[:, None])
    dh = rng.choice([1.0, -1.5, 1.25, -1.75], (m, f)) * 2.0**np.concatenate([rng.integers(-148, -100, 16), rng.integers(80, 100, 8)])[:, None]
    dh = dh.astype(np.float32)
    made = {"d": poisoned(dr, m, 2 * f), "dt": poisoned(dr, 2 * f, m), "ht": poisoned(dr, f, m)}
    dr.dr_gated_backward(torch.from_numpy(dh).cuda(), gate, up, **{n: v[0] for n, v in made.items()}, act=kind)
    torch.cuda.synchronize()
    d, h, t_d, t_h = _want(dh.astype(np.float64), gv, uv, kind)
    step = 2.0**-148
    dv = dh.astype(np.float64)
    t_d = t_d + step * (2 + np.abs(np.concatenate([uv, dv], 1)))
    # dh * up is formed first; where it passes fp32, dgate does
    over = np.concatenate([np.abs(dv * uv) >= 2.0**128, np.zeros_like(dv, dtype=bool)], 1) | (np.abs(d) >= 2.0**128)
    d = np.where(over, np.nan, d)
    check_rows(made["d"], d, t_d, "d")
    check_rows(made["dt"], d.T, t_d.T, "dt")
    check_rows(made["ht"], h.T, t_h.T, "ht")


def _check_turned(made, values):
    q, wide, scales = made
    codes, sc = quant.quantize(values.T, 1)
    rows, padded = codes.shape
    got = wide.cpu().numpy()
    both_nan = ((codes & 0x7F) == 0x7F) & ((got[:rows, :padded] & 0x7F) == 0x7F)
    assert np.array_equal(np.where(both_nan, codes, got[:rows, :padded]), codes)
    assert (got[rows:] == 0xA5).all() and (got[:, padded:] == 0xA5).all(), "written outside the matrix"
    got = scales.cpu().numpy()
    assert np.array_equal(got[:sc.size], sc.reshape(-1)) and (got[sc.size:] == 0xA5).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (2, 129), (5, 8), (128, 128), (129, 127), (333, 344), (40, 1100), (300, 512), (257, 513)])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_turned(rows, cols, block_rows):
    dr = _dr()
    say("qtranspose", rows, cols, block_rows)
    rng = np.random.default_rng(rows + cols)
    x = rng.standard_normal((rows, cols)) * 2.0**rng.integers(-12, 12, (rows, 1))
    x[rows // 2] = 0.0
    src, values = quantized(dr, x, block_rows, 16)
    if rows > 4:
        src.data[1, 0] = 0x7F
        values[1, 0] = np.nan
    made = poisoned(dr, cols, rows)
    dr.dr_qtranspose(src, made[0])
    torch.cuda.synchronize()
    _check_turned(made, values)


def test_every_code_and_scale():
    """All codes in rows of every scale; elements below 2^-133 count as zero and those from 2^128 on as NaN."""
    dr = _dr()
    say("qtranspose, every code")
    rows, cols = 255, 256
    src = dr.QMatrix.empty(rows, cols)
    src.data.copy_(torch.arange(256, dtype=torch.uint8).repeat(rows, 1))
    src.scales.fill_(127)
    src.scales[0, :, :2] = torch.arange(255, dtype=torch.uint8)[:, None]
    values = quant.values(src.data.cpu().numpy(), src.scales.cpu().numpy(), cols, 1)
    with np.errstate(invalid="ignore"):
        values = np.where(np.abs(values) >= 2.0**128, np.nan, np.where(np.abs(values) < 2.0**-133, values * 0.0, values))
    made = poisoned(dr, cols, rows)
    dr.dr_qtranspose(src, made[0])
    torch.cuda.synchronize()
    _check_turned(made, values)


def test_empty():
    dr = _dr()
    say("empty")
    for m, f in ((0, 5), (5, 0), (0, 0)):
        dr.dr_gated_backward(torch.empty((m, f), device="cuda"), dr.QMatrix.empty(m, f), dr.QMatrix.empty(m, f), dr.QMatrix.empty(m, 2 * f),
                             dr.QMatrix.empty(2 * f, m), dr.QMatrix.empty(f, m))
        dr.dr_qtranspose(dr.QMatrix.empty(m, f), dr.QMatrix.empty(f, m))
    torch.cuda.synchronize()


@pytest.mark.parametrize("f", [256, 333])
def test_replayed_graph_on_another_stream(f):
    dr = _dr()
    say("graph", f)
    m = 300
    gate, up, dh, _, _, _ = _inputs(dr, m, f, torch.bfloat16, 2)
    dhs = dh.cuda()
    out = [dr.QMatrix.empty(m, 2 * f), dr.QMatrix.empty(2 * f, m), dr.QMatrix.empty(f, m), dr.QMatrix.empty(f, m)]

    def step():
        dr.dr_gated_backward(dhs, gate, up, *out[:3])
        dr.dr_qtranspose(gate, out[3])

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    for seed in range(3):
        dhs.copy_(torch.randn((m, f), generator=torch.Generator().manual_seed(seed)))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for q in out for t in (q.data, q.scales)]
        for q in out:
            q.data.fill_(1), q.scales.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [t for q in out for t in (q.data, q.scales)]))
