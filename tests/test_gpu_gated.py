"""dr_qgated and dr_qgated_save on the GPU against the block in 64 bits of the values that the codes stand for.

Tolerance.  The sums of gate and up are off by at most D = (K padded to 128, and 64) * 2^-23 * sum |x||w| each (as the
products' are), or with fast sums by 2^-10 of the sum over groups of 8 columns of the largest |x||w| besides.  act has a
slope of at most 1.13, is itself off by (8 + |z|) 2^-23 of its value with the product's rounding, and by 2^-117 (up's
magnitude times) where its exponential passes 2^126; from |z| = 150 on the logistic function is 0 or 1.  bf16 adds 2^-8 of the result.
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


def _groups(a, b):
    """sum over groups of 8 adjacent columns of the largest |a||b| of the group."""
    k = -a.shape[1] % 8
    a, b = (np.abs(np.pad(v, ((0, 0), (0, k)))).reshape(v.shape[0], -1, 8) for v in (a, b))
    return sum((a[:, None, g] * b[None, :, g]).max(axis=2) for g in range(a.shape[1]))


def _want(xv, wv, kind, fast=False):
    """(gate, up, h) and their tolerances, before any rounding of a result."""
    f = wv.shape[0] // 2
    y, size = quant.product(xv, wv)
    d = (-(-xv.shape[1] // 128) * 128 + 64) * 2.0**-23 * size + (2.0**-10 * _groups(xv, wv) if fast else 0.0)
    gate, up, dg, du = y[:, :f], y[:, f:], d[:, :f], d[:, f:]
    a, _, z = gated.act(gate, kind)
    h = a * up
    tol = 1.13 * dg * (np.abs(up) + du) + np.abs(a) * du + (8 + np.minimum(np.abs(z), 150)) * 2.0**-23 * np.abs(h) + 2.0**-117 * (np.abs(up) + du)
    return (gate, up, h), (dg, du, tol)


def _inputs(dr, m, f, k, x_type, seed, block_rows=128, extra=0):
    """x, w, and their values; gates of a few units, some rows far larger and one of zeros."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((m, k)) * 2.0**rng.integers(-2, 3, (m, 1))
    if m > 2:
        x[m // 3] *= 64.0
        x[m // 2] = 0.0
    x = torch.from_numpy(x.astype(np.float32)).to(x_type)
    w, wv = quantized(dr, rng.standard_normal((2 * f, k)) * 2.0 / np.sqrt(k), block_rows, extra)
    xq = quant.quantize(x.to(torch.float64).numpy(), 1)
    return x, w, quant.values(*xq, k, 1), wv


def _space(dr, m, w, save=False):
    need = (dr.dr_qgated_save_workspace if save else dr.dr_qgated_workspace)(m, w)
    return torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN wherever it is read before it is written


def _close(got, want, tol, bf16):
    got = got.to(torch.float64).cpu().numpy()
    bad = ~(np.abs(got - want) <= tol + (2.0**-8 * (np.abs(want) + tol) if bf16 else 0.0))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


ROWS = [1, 2, 15, 16, 17, 33, 64, 129, 300]
SIZES = [(1, 1), (8, 128), (7, 200), (33, 344), (128, 1000), (344, 256), (555, 130), (260, 2176)]


@pytest.mark.parametrize("m", ROWS)
@pytest.mark.parametrize("f,k", SIZES)
@pytest.mark.parametrize("kind,x_type", [(SILU, torch.bfloat16), (GELU, torch.float32)])
def test_rows_in_rows_out(m, f, k, kind, x_type):
    dr = _dr()
    x, w, xv, wv = _inputs(dr, m, f, k, x_type, m + f + k, extra=16)
    ws = _space(dr, m, w)
    for out_type, fast in ((torch.bfloat16, True), (torch.bfloat16, False), (torch.float32, False)):
        say("gated", m, f, k, kind, x_type, out_type, fast)
        (_, _, h), (_, _, tol) = _want(xv, wv, kind, fast)
        out = torch.full((m + 1, f), 7.0, dtype=out_type, device="cuda")
        dr.dr_qgated(x.cuda(), w, out[:m], act=kind, fast=fast, workspace=ws)
        torch.cuda.synchronize()
        _close(out[:m], h, tol, out_type == torch.bfloat16)
        assert (out[m] == 7.0).all()


@pytest.mark.parametrize("m", [1, 40, 128, 200, 300])
@pytest.mark.parametrize("f,k", [(1, 1), (128, 128), (130, 200), (344, 256), (640, 1000), (100, 2176)])
@pytest.mark.parametrize("kind", [SILU, GELU])
def test_save(m, f, k, kind):
    dr = _dr()
    x, w, _, wv = _inputs(dr, m, f, k, torch.float32, m + f + k, extra=32)
    xq, xv = quantized(dr, x.to(torch.float64).numpy(), 1, 16)
    ws = _space(dr, m, w, save=True)
    for fast in (True, False):
        say("save", m, f, k, kind, fast)
        (gate, up, h), tols = _want(xv, wv, kind, fast)
        made = [poisoned(dr, m, f) for _ in range(3)]
        dr.dr_qgated_save(xq, w, *(q for q, _, _ in made), act=kind, fast=fast, workspace=ws)
        torch.cuda.synchronize()
        for one, want, tol, name in zip(made, (h, gate, up), (tols[2], tols[0], tols[1]), ("h", "gate", "up")):
            check_rows(one, want, tol, name)
        alone = poisoned(dr, m, f, 0)
        dr.dr_qgated_save(xq, w, alone[0], act=kind, fast=fast, workspace=ws)
        assert torch.equal(alone[0].data, made[0][0].data[:, :alone[0].data.shape[1]]) and torch.equal(alone[0].scales, made[0][0].scales)


@pytest.mark.parametrize("blocks", [(1, 1), (128, 1), (128, 128)])
def test_save_blocks_of_either_kind(blocks):
    """x and w in blocks of 1 x 128 or 128 x 128; up's first row lies inside a square block of w."""
    dr = _dr()
    say("save blocks", blocks)
    m, f, k = 150, 200, 300
    rng = np.random.default_rng(3)
    x, xv = quantized(dr, rng.standard_normal((m, k)) * 2.0**rng.integers(-4, 4, (m, 1)), blocks[0])
    w, wv = quantized(dr, rng.standard_normal((2 * f, k)) * 2.0**rng.integers(-5, -1, (2 * f, 1)), blocks[1])
    (gate, up, h), tols = _want(xv, wv, SILU)
    made = [poisoned(dr, m, f) for _ in range(3)]
    dr.dr_qgated_save(x, w, *(q for q, _, _ in made), workspace=_space(dr, m, w, save=True))
    torch.cuda.synchronize()
    for one, want, tol, name in zip(made, (h, gate, up), (tols[2], tols[0], tols[1]), ("h", "gate", "up")):
        check_rows(one, want, tol, name)


@pytest.mark.parametrize("m,f,k", [(5, 50, 300), (130, 75, 300), (300, 145, 150)])
@pytest.mark.parametrize("offset,stride", [(1, 1), (4, 8), (2, 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_at_any_element(m, f, k, offset, stride, dtype):
    """Rows of x and of h at odd places: nothing beside them is read as a value or written."""
    dr = _dr()
    say("gated at", offset, stride, m, f, k, dtype)
    x, w, xv, wv = _inputs(dr, m, f, k, dtype, 1)
    wide = torch.full((offset + m * (k + stride) + 8,), float("nan"), dtype=dtype, device="cuda")
    xs = wide[offset:offset + m * (k + stride)].view(m, k + stride)[:, :k]
    xs.copy_(x)
    step = f + stride
    buf = torch.full((offset + m * step + 8,), -3.0, dtype=dtype, device="cuda")
    out = buf[offset:offset + m * step].view(m, step)[:, :f]
    dr.dr_qgated(xs, w, out, workspace=_space(dr, m, w))
    torch.cuda.synchronize()
    (_, _, h), (_, _, tol) = _want(xv, wv, SILU)
    _close(out, h, tol, dtype == torch.bfloat16)
    out.fill_(-3.0)
    assert (buf == -3.0).all()


@pytest.mark.parametrize("m", [1, 20, 300])
@pytest.mark.parametrize("kind", [SILU, GELU])
def test_far_gates(m, kind):
    """Gates from -2^60 to 2^60: act is g, or 0, and never NaN; a NaN in x makes its row NaN and no other."""
    dr = _dr()
    say("far gates", m, kind)
    f, k = 40, 128
    gates = np.array([0.0, 1.0, -1.0, 20.0, -20.0, 88.0, -88.0, 104.0, -104.0, 128.0, -128.0, 448.0, -448.0, 2.0**15, -2.0**15, 2.0**60, -2.0**60, 3.5, -3.5, 0.5])
    gates = np.tile(gates, 2)
    w = np.zeros((2 * f, k))
    w[:f, 0] = gates
    w[f:, 1] = np.linspace(-2, 2, f)
    w, wv = quantized(dr, w, 1)
    x = np.zeros((m, k), dtype=np.float32)
    x[:, 0] = x[:, 1] = 1.0
    xv = x.astype(np.float64)
    (gate, up, h), (dg, du, tol) = _want(xv, wv, kind)
    ws = _space(dr, m, w)
    out = torch.empty((m, f), device="cuda")
    dr.dr_qgated(torch.from_numpy(x).cuda(), w, out, act=kind, workspace=ws)
    _close(out, h, tol, False)
    made = [poisoned(dr, m, f) for _ in range(3)]
    xq, _ = quantized(dr, xv)
    dr.dr_qgated_save(xq, w, *(q for q, _, _ in made), act=kind, workspace=_space(dr, m, w, save=True))
    for one, want, t, name in zip(made, (h, gate, up), (tol, dg, du), ("h", "gate", "up")):
        check_rows(one, want, t, name)
    x[m // 2, 5] = np.nan
    dr.dr_qgated(torch.from_numpy(x).cuda(), w, out, act=kind, workspace=ws)
    nan = torch.isnan(out).cpu().numpy()
    assert nan[m // 2].all() and int(nan.sum()) == f


def test_empty():
    dr = _dr()
    say("empty")
    w = dr.QMatrix.empty(8, 200, 128)
    dr.dr_qgated(torch.empty((0, 200), device="cuda"), w, torch.empty((0, 4), device="cuda"))
    dr.dr_qgated(torch.empty((3, 200), device="cuda"), dr.QMatrix.empty(0, 200, 128), torch.empty((3, 0), device="cuda"))
    dr.dr_qgated_save(dr.QMatrix.empty(0, 200), w, dr.QMatrix.empty(0, 4))
    # no columns: gate and up are 0, and so is h
    none = dr.QMatrix.empty(8, 0, 128)
    for m in (3, 40):
        out = torch.full((m, 4), 5.0, device="cuda")
        dr.dr_qgated(torch.empty((m, 0), device="cuda"), none, out, workspace=_space(dr, m, none))
        assert (out == 0.0).all()
        made = [poisoned(dr, m, 4) for _ in range(3)]
        dr.dr_qgated_save(dr.QMatrix.empty(m, 0), none, *(q for q, _, _ in made), workspace=_space(dr, m, none, save=True))
        for one in made:
            check_rows(one, np.zeros((m, 4)), np.zeros((m, 4)), "no columns")


@pytest.mark.parametrize("m", [1, 200])
def test_replayed_graph_on_another_stream(m):
    """Captured once and replayed on new inputs, with other work of the process in between."""
    dr = _dr()
    say("graph", m)
    f, k = 300, 512
    x, w, _, _ = _inputs(dr, m, f, k, torch.bfloat16, 9)
    xs, ws, ws2 = x.cuda(), _space(dr, m, w), _space(dr, m, w, save=True)
    out, xq = torch.empty((m, f), dtype=torch.bfloat16, device="cuda"), dr.QMatrix.empty(m, k)
    saved = [dr.QMatrix.empty(m, f) for _ in range(3)]

    def block():
        dr.dr_qgated(xs, w, out, fast=True, workspace=ws)
        dr.dr_quantize(xs, xq)
        dr.dr_qgated_save(xq, w, *saved, fast=True, workspace=ws2)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        block()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            block()
    for seed in range(4):
        fresh = torch.randn((m, k), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)
        xs.copy_(fresh)
        block()
        torch.cuda.synchronize()
        want = [out.clone()] + [t.clone() for q in saved for t in (q.data, q.scales)]
        out.fill_(3.0)
        for q in saved:
            q.data.fill_(1), q.scales.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, [out] + [t for q in saved for t in (q.data, q.scales)]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def _want_large(xv, wv, kind, fast):
    """_want with the products on the GPU, in 64 bits.  Fast sums lose 2^-10 of sum |x||w| at most."""
    xg, wg = torch.from_numpy(xv).cuda(), torch.from_numpy(wv).cuda()
    y, size = (xg @ wg.t()).cpu().numpy(), (xg.abs() @ wg.abs().t()).cpu().numpy()
    f = wv.shape[0] // 2
    d = ((-(-xv.shape[1] // 128) * 128 + 64) * 2.0**-23 + (2.0**-10 if fast else 0.0)) * size
    gate, up, dg, du = y[:, :f], y[:, f:], d[:, :f], d[:, f:]
    a, _, z = gated.act(gate, kind)
    h = a * up
    tol = 1.13 * dg * (np.abs(up) + du) + np.abs(a) * du + (8 + np.minimum(np.abs(z), 150)) * 2.0**-23 * np.abs(h) + 2.0**-117 * (np.abs(up) + du)
    return (gate, up, h), (dg, du, tol)


def _large_inputs(dr, m, f, k, seed, block_rows):
    """Quantized on the GPU (dr_quantize is tested apart), and what the codes stand for."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((m, k), generator=gen, device="cuda") * torch.exp2(torch.randint(-2, 3, (m, 1), generator=gen, device="cuda").float())
    w = torch.randn((2 * f, k), generator=gen, device="cuda") * (2.0 / k**0.5)
    xq, wq = dr.QMatrix.empty(m, k), dr.QMatrix.empty(2 * f, k, block_rows)
    dr.dr_quantize(x, xq), dr.dr_quantize(w, wq)
    values = [quant.values(q.data.cpu().numpy(), q.scales.cpu().numpy(), k, b) for q, b in ((xq, 1), (wq, block_rows))]
    return x, xq, wq, *values


# tiles of 256 rows and of 128, last rounds of them cut in two or four, tiles alone on their CU, and splits; columns that
# are no multiple of a tile or of 16 bytes
LARGE = [(1157, 8100, 300), (2050, 8200, 640), (520, 4104, 1000), (1000, 700, 2176), (3000, 3456, 256), (130, 2000, 2000), (257, 6001, 129), (700, 9000, 128)]


@pytest.mark.parametrize("m,f,k", LARGE)
@pytest.mark.parametrize("fast", [True, False])
@pytest.mark.parametrize("block_rows", [128, 1])
def test_large(m, f, k, fast, block_rows):
    dr = _dr()
    kind = GELU if fast else SILU
    x, xq, wq, xv, wv = _large_inputs(dr, m, f, k, m + f, block_rows)
    (gate, up, h), (dg, du, tol) = _want_large(xv, wv, kind, fast)
    say("large gated", m, f, k, fast, block_rows)
    for out_type in (torch.bfloat16, torch.float32):
        out = torch.full((m + 1, f), 7.0, dtype=out_type, device="cuda")
        dr.dr_qgated(x, wq, out[:m], act=kind, fast=fast, workspace=_space(dr, m, wq))
        torch.cuda.synchronize()
        _close(out[:m], h, tol, out_type == torch.bfloat16)
        assert (out[m] == 7.0).all()
    say("large save", m, f, k, fast, block_rows)
    made = [poisoned(dr, m, f) for _ in range(3)]
    dr.dr_qgated_save(xq, wq, *(q for q, _, _ in made), act=kind, fast=fast, workspace=_space(dr, m, wq, save=True))
    torch.cuda.synchronize()
    for one, want, t, name in zip(made, (h, gate, up), (tol, dg, du), ("h", "gate", "up")):
        check_rows(one, want, t, name)


def test_large_not_finite():
    """A row of x that is not finite, and gates past fp32's range, in the tiles of a long batch."""
    dr = _dr()
    say("large, not finite")
    m, f, k = 600, 4200, 512
    x, xq, wq, xv, wv = _large_inputs(dr, m, f, k, 1, 128)
    xq.data[77, 5] = 0x7F
    xv[77] = np.nan
    xq.scales[:, 300] = 254  # 2^127 times the codes: infinite sums of either sign
    (gate, up, h), (dg, du, tol) = _want_large(xv, wv, SILU, False)
    skip = np.zeros(m, dtype=bool)
    skip[300] = True
    made = [poisoned(dr, m, f) for _ in range(3)]
    dr.dr_qgated_save(xq, wq, *(q for q, _, _ in made), workspace=_space(dr, m, wq, save=True))
    torch.cuda.synchronize()
    codes = [q.data[300, :f].cpu().numpy() & 0x7F for q, _, _ in made]
    assert all((c == 0x7F).mean() > 0.9 for c in codes[1:])  # nearly all sums are infinite
    for one, want, t, name in zip(made, (h, gate, up), (tol, dg, du), ("h", "gate", "up")):
        q, wide, scales = one
        q.data[300] = q.data[299]
        q.scales[:, 300] = q.scales[:, 299]
        want[300], t[300] = want[299], t[299]
        check_rows(one, want, np.where(np.isnan(t), 0.0, t), name)


@pytest.mark.parametrize("f,k", [(3, 16384), (9, 16385), (20, 20000), (4200, 300)])
@pytest.mark.parametrize("x_type", [torch.bfloat16, torch.float32])
def test_one_row(f, k, x_type):
    """One row at the ends of what its own kernel's LDS holds, and beyond."""
    dr = _dr()
    say("one row", f, k, x_type)
    x, w, xv, wv = _inputs(dr, 1, f, k, x_type, k, extra=16)
    (_, _, h), (_, _, tol) = _want(xv, wv, GELU)
    out = torch.full((2, f), 7.0, device="cuda")
    dr.dr_qgated(x.cuda(), w, out[:1], act=GELU, workspace=_space(dr, 1, w))
    _close(out[:1], h, tol, False)
    assert (out[1] == 7.0).all()


@pytest.mark.parametrize("m", [1, 5, 40, 300])
def test_weights_of_more_than_4_gib(m):
    """up's rows, and gate's last ones, begin beyond 2^32 bytes."""
    dr = _dr()
    say("large weights", m)
    f, k = 300001, 8192
    gen = torch.Generator(device="cuda").manual_seed(m)
    codes = torch.randint(0, 120, (2 * f, k), generator=gen, device="cuda", dtype=torch.uint8) | torch.randint(0, 2, (2 * f, 1), generator=gen, device="cuda", dtype=torch.uint8) << 7
    w = dr.QMatrix(codes, torch.full((k // 512, -(-2 * f // 128), 4), 114, dtype=torch.uint8, device="cuda"), 2 * f, k, 128)
    x = torch.randn((m, k), generator=gen, device="cuda") * 0.01
    at = torch.tensor([0, 1, 4097, 131071, 131072, 262143, 262144, 299999, f - 1], device="cuda")
    wv = quant.E4M3[torch.cat([codes[at], codes[at + f]]).cpu().numpy()] * 2.0**(114 - 127)
    xv = quant.values(*quant.quantize(x.to(torch.float64).cpu().numpy(), 1), k, 1)
    (gate, up, h), (dg, du, tol) = _want(xv, wv, SILU)
    out = torch.empty((m, f), device="cuda")
    dr.dr_qgated(x, w, out, workspace=_space(dr, m, w))
    _close(out[:, at], h, tol, False)
    if m < 40:
        return
    xq, made = dr.QMatrix.empty(m, k), [dr.QMatrix.empty(m, f) for _ in range(3)]
    dr.dr_quantize(x, xq)
    dr.dr_qgated_save(xq, w, *made, workspace=_space(dr, m, w, save=True))
    for q, want, t in zip(made, (h, gate, up), (tol, dg, du)):
        per = q.scales.permute(1, 0, 2).reshape(m, -1)[:, at // 128].cpu().numpy()
        got = quant.E4M3[q.data[:, at].cpu().numpy()] * 2.0**(per - 127.0)
        assert (np.abs(got - want) <= np.maximum(2.0**-4 * np.abs(want), 2.0**(per - 137.0)) * (1 + 2.0**-20) + 2 * t).all()


def test_two_streams_at_once():
    """Calls on two streams with workspaces of their own, and what each gives alone."""
    dr = _dr()
    say("two streams")
    jobs = []
    for i, (m, f, k) in enumerate([(200, 700, 512), (1, 3000, 1024), (90, 1500, 2048), (600, 1300, 256)]):
        x, w, _, _ = _inputs(dr, m, f, k, torch.bfloat16, i)
        xq, h, out = dr.QMatrix.empty(m, k), dr.QMatrix.empty(m, f), torch.empty((m, f), dtype=torch.bfloat16, device="cuda")
        xs = x.cuda()
        dr.dr_quantize(xs, xq)
        jobs.append((xs, xq, w, h, out, _space(dr, m, w), _space(dr, m, w, save=True)))

    def run(job, stream=None):
        xs, xq, w, h, out, ws, ws2 = job
        dr.dr_qgated(xs, w, out, fast=True, workspace=ws, stream=stream)
        dr.dr_qgated_save(xq, w, h, fast=True, workspace=ws2, stream=stream)

    alone = []
    for job in jobs:
        run(job)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in (job[3].data, job[3].scales, job[4])])
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(5):
        for job, stream in zip(jobs, streams):
            run(job, stream)
    torch.cuda.synchronize()
    for job, want in zip(jobs, alone):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip((job[3].data, job[3].scales, job[4]), want))


def test_another_device_is_refused(monkeypatch):
    dr = _dr()
    w, x, h = dr.QMatrix.empty(8, 128, 128), torch.empty((3, 128), device="cuda"), torch.empty((3, 4), device="cuda")
    q, g, t = dr.QMatrix.empty(3, 128), dr.QMatrix.empty(3, 4), dr.QMatrix.empty(128, 3)
    monkeypatch.setattr(dr, "_device", lambda: 1)
    for call in (lambda: dr.dr_qgated(x, w, h), lambda: dr.dr_qgated_save(q, w, g), lambda: dr.dr_qtranspose(q, t),
                 lambda: dr.dr_gated_backward(h, g, g, dr.QMatrix.empty(3, 8))):
        with pytest.raises(ValueError, match="current device"):
            call()
