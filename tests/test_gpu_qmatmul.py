"""dr_qmatmul and dr_qlinear on the GPU against products in 64 bits of the values that the codes stand for.

Tolerance.  A product of two e4m3 values is exact in fp32, as are the powers of two; what is left are the roundings of
the sum of K products, in whatever order.  With S = sum |a||b| an fp32 sum of n terms is off by at most n * 2^-24 * S
(2^-23 where an adder truncates); n is K padded to 128, and a few more to join partial sums.  A bf16 result adds
2^-8 of itself for its own rounding.
"""
import numpy as np
import pytest
import torch

from oracle import quant
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def _dr():
    from paper_2607_22614_amd import dr
    return dr


def _matrix(dr, rows, cols, block_rows, seed, spread=8, extra=0):
    """Random codes (all but NaN) and scales, on the device, and their values in 64 bits."""
    rng = np.random.default_rng(seed)
    m = dr.QMatrix.empty(rows, cols, block_rows)
    padded = m.data.shape[1]
    codes = rng.integers(0, 255, (rows, padded)).astype(np.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x3A
    codes[:, cols:] = 0
    scales = rng.integers(127 - spread, 127 + spread + 1, tuple(m.scales.shape)).astype(np.uint8)
    wide = torch.full((rows, padded + extra), 0x7F, dtype=torch.uint8, device="cuda")  # NaN behind each row
    wide[:, :padded] = torch.from_numpy(codes).cuda()
    q = dr.QMatrix(wide, torch.from_numpy(scales).cuda(), rows, cols, block_rows)
    return q, quant.values(codes, scales, cols, block_rows)


def _close(got, want, size, k, bf16):
    tol = (-(-k // 128) * 128 + 64) * 2.0**-23 * size + (np.abs(want) * 2.0**-8 if bf16 else 0)
    got = got.to(torch.float64).cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


def _workspace(dr, m, n, k):
    return torch.empty((dr.dr_qmatmul_workspace(m, n, k),), dtype=torch.uint8, device="cuda")


SHAPES = [(1, 1, 1), (1, 16, 128), (3, 17, 129), (16, 16, 256), (17, 33, 640), (64, 64, 128), (65, 130, 344), (128, 128, 512),
          (200, 688, 256), (129, 257, 1000), (255, 255, 2048), (256, 256, 384), (300, 520, 136), (513, 300, 896), (1000, 77, 128),
          (31, 1025, 3000), (700, 1300, 200)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("blocks", [(1, 128), (1, 1), (128, 128)])
def test_product(m, n, k, blocks):
    dr = _dr()
    a, av = _matrix(dr, m, k, blocks[0], m + k, extra=16)
    b, bv = _matrix(dr, n, k, blocks[1], n + k + 1, extra=48)
    want, size = quant.product(av, bv)
    ws = _workspace(dr, m, n, k)
    for dtype in (torch.float32, torch.bfloat16):
        say("product", m, n, k, blocks, dtype)
        out = torch.full((m + 1, n), 7.0, dtype=dtype, device="cuda")
        dr.dr_qmatmul(a, b, out[:m], workspace=ws)
        torch.cuda.synchronize()
        _close(out[:m], want, size, k, dtype == torch.bfloat16)
        assert (out[m] == 7.0).all()
    start = torch.from_numpy(np.random.default_rng(5).standard_normal((m, n)).astype(np.float32) * float(np.abs(want).mean() + 1))
    out = start.cuda()
    dr.dr_qmatmul(a, b, out, accumulate=True, workspace=ws)
    torch.cuda.synchronize()
    s = start.to(torch.float64).numpy()
    _close(out, want + s, size + np.abs(s), k, False)


def _groups(a, b):
    """sum over groups of 8 adjacent columns of the largest |a||b| of the group."""
    k = -a.shape[1] % 8
    a, b = (np.abs(np.pad(v, ((0, 0), (0, k)))).reshape(v.shape[0], -1, 8) for v in (a, b))
    return sum((a[:, None, g] * b[None, :, g]).max(axis=2) for g in range(a.shape[1]))


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("blocks", [(1, 128), (1, 1), (128, 128)])
def test_fast_sums(m, n, k, blocks):
    """Each product of 8 adjacent columns may lose what lies below 2^-13 of the largest one's power of two, so at most
    2^-13 of the largest product: 8 * 2^-13 of it per group, beside the tolerance of the exact sums."""
    dr = _dr()
    a, av = _matrix(dr, m, k, blocks[0], m + k, extra=16)
    b, bv = _matrix(dr, n, k, blocks[1], n + k + 1, extra=48)
    want, size = quant.product(av, bv)
    tol = 2.0**-10 * _groups(av, bv) + (-(-k // 128) * 128 + 64) * 2.0**-23 * size
    ws = _workspace(dr, m, n, k)
    start = torch.from_numpy(np.random.default_rng(5).standard_normal((m, n)).astype(np.float32) * float(np.abs(want).mean() + 1))
    for dtype, accumulate in ((torch.float32, False), (torch.bfloat16, False), (torch.float32, True)):
        say("fast", m, n, k, blocks, dtype, accumulate)
        out = torch.full((m + 1, n), 7.0, dtype=dtype, device="cuda")
        add = start.to(torch.float64).numpy() if accumulate else 0.0
        if accumulate:
            out[:m] = start.cuda()
        dr.dr_qmatmul(a, b, out[:m], accumulate=accumulate, fast=True, workspace=ws)
        torch.cuda.synchronize()
        got = out[:m].to(torch.float64).cpu().numpy()
        bound = tol + (np.abs(want) * 2.0**-8 if dtype == torch.bfloat16 else 2.0**-22 * np.abs(add))
        assert (np.abs(got - want - add) <= bound).all()
        assert (out[m] == 7.0).all()


def test_fast_sums_of_normal_values():
    """Normally distributed values: a group's 8 products lose less than 2^-13 of its largest each, with signs of their own,
    so of the norm at most sqrt(8 * 2^-26 * E[largest^2] / (8 * E[product^2])) <= 2^-13 * sqrt(8)."""
    dr = _dr()
    say("fast, normal values")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w = torch.randn((300, 4096), generator=gen, device="cuda"), torch.randn((520, 4096), generator=gen, device="cuda")
    a, b = dr.QMatrix.empty(300, 4096, 1), dr.QMatrix.empty(520, 4096, 128)
    dr.dr_quantize(x, a), dr.dr_quantize(w, b)
    out = torch.empty((300, 520), device="cuda")
    dr.dr_qmatmul(a, b, out, fast=True, workspace=_workspace(dr, 300, 520, 4096))
    av = quant.values(a.data.cpu().numpy(), a.scales.cpu().numpy(), 4096, 1)
    bv = quant.values(b.data.cpu().numpy(), b.scales.cpu().numpy(), 4096, 128)
    want = av @ bv.T
    assert np.linalg.norm(out.cpu().numpy() - want) <= 2.0**-13 * np.sqrt(8) * np.linalg.norm(want)


@pytest.mark.parametrize("m,n,k", [(5, 50, 300), (130, 150, 300), (300, 290, 150)])
@pytest.mark.parametrize("offset,stride", [(1, 1), (4, 8), (2, 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_output_at_any_element(m, n, k, offset, stride, dtype):
    """Rows of c at odd places: nothing beside them is written."""
    dr = _dr()
    say("output at", offset, stride, m, n, k, dtype)
    a, av = _matrix(dr, m, k, 1, 1)
    b, bv = _matrix(dr, n, k, 128, 2)
    step = n + stride
    buf = torch.full((offset + m * step + 8,), -3.0, dtype=dtype, device="cuda")
    out = buf[offset:offset + m * step].view(m, step)[:, :n]
    dr.dr_qmatmul(a, b, out, workspace=_workspace(dr, m, n, k))
    torch.cuda.synchronize()
    _close(out, *quant.product(av, bv), k, dtype == torch.bfloat16)
    out.fill_(-3.0)
    assert (buf == -3.0).all()


@pytest.mark.parametrize("m", [1, 20, 300])
def test_extreme_scales_and_nan(m):
    """Scales from 2^-127 on, products that leave fp32's range, NaN codes: as the values say."""
    dr = _dr()
    say("extreme scales", m)
    n, k = 40, 512
    a, b = dr.QMatrix.empty(m, k, 1), dr.QMatrix.empty(n, k, 1)
    a.data.fill_(0x38), b.data.fill_(0x38)  # 1.0
    for ea, eb, want in ((0, 254, 512.0), (127, 127, 512.0), (0, 127, 2.0**-118), (247, 7, 512.0), (254, 254, float("inf"))):
        a.scales.fill_(ea), b.scales.fill_(eb)
        out = torch.empty((m, n), device="cuda")
        dr.dr_qmatmul(a, b, out, workspace=_workspace(dr, m, n, k))
        assert (out == want).all(), (ea, eb, out.flatten()[0].item())
    a.scales.fill_(127), b.scales.fill_(127)
    a.data[0, 300] = 0x7F
    b.data[3, 5] = 0xFF
    out = torch.empty((m, n), device="cuda")
    dr.dr_qmatmul(a, b, out, workspace=_workspace(dr, m, n, k))
    nan = torch.isnan(out)
    assert nan[0].all() and nan[:, 3].all() and int(nan.sum()) == m + n - 1


def test_empty_products():
    dr = _dr()
    out = torch.full((3, 4), 5.0, device="cuda")
    a, b = dr.QMatrix.empty(3, 0, 1), dr.QMatrix.empty(4, 0, 128)
    dr.dr_qmatmul(a, b, out, accumulate=True)
    assert (out == 5.0).all()
    dr.dr_qmatmul(a, b, out)
    assert (out == 0.0).all()
    dr.dr_qmatmul(dr.QMatrix.empty(0, 200, 1), dr.QMatrix.empty(4, 200, 128), torch.empty((0, 4), device="cuda"))
    dr.dr_qmatmul(dr.QMatrix.empty(3, 200, 1), dr.QMatrix.empty(0, 200, 128), torch.empty((3, 0), device="cuda"))
    y = torch.full((3, 4), 5.0, device="cuda")
    dr.dr_qlinear(torch.empty((3, 0), device="cuda"), dr.QMatrix.empty(4, 0, 128), y)
    assert (y == 0.0).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 33, 64, 100, 129, 300])
@pytest.mark.parametrize("n,k", [(16, 128), (70, 344), (256, 1000), (1111, 130), (520, 2176)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_linear(m, n, k, dtype):
    dr = _dr()
    say("linear", m, n, k, dtype)
    rng = np.random.default_rng(m + n + k)
    x = torch.from_numpy((rng.standard_normal((m, k)) * 2.0**rng.integers(-9, 9, (m, 1))).astype(np.float32)).to(dtype)
    x[m // 2, :k // 2] = 0
    w, wv = _matrix(dr, n, k, 128, n, spread=3)
    xv = quant.values(*quant.quantize(x.to(torch.float64).numpy(), 1), k, 1)
    want, size = quant.product(xv, wv)
    ws = torch.empty((dr.dr_qlinear_workspace(m, w),), dtype=torch.uint8, device="cuda")
    for out_type in (torch.bfloat16, torch.float32):
        y = torch.empty((m, n), dtype=out_type, device="cuda")
        dr.dr_qlinear(x.cuda(), w, y, workspace=ws)
        torch.cuda.synchronize()
        _close(y, want, size, k, out_type == torch.bfloat16)


@pytest.mark.parametrize("m,n,k", [(4100, 4360, 256), (4100, 4360, 300), (4352, 4096, 520), (3000, 3001, 256), (3001, 2999, 384), (5000, 2600, 1030),
                                   (8200, 2050, 100), (8200, 2051, 128), (300, 16400, 640), (40, 70000, 300)])
@pytest.mark.parametrize("fast", [False, True])
def test_more_tiles_than_workgroups(m, n, k, fast):
    """Workgroups that go from tile to tile, of two blocks and more and of a single one, at the edges of c and inside."""
    dr = _dr()
    a, av = _matrix(dr, m, k, 1, m + k, spread=3)
    b, bv = _matrix(dr, n, k, 128, n + k, spread=3)
    av, bv = torch.from_numpy(av).cuda(), torch.from_numpy(bv).cuda()
    want, size = av @ bv.t(), av.abs() @ bv.abs().t()
    n_sum = -(-k // 128) * 128 + 64
    tol = (n_sum * 2.0**-23 + (2.0**-10 if fast else 0)) * size
    ws = _workspace(dr, m, n, k)
    for dtype, accumulate in ((torch.bfloat16, False), (torch.float32, False), (torch.float32, True)):
        say("many tiles", m, n, k, fast, dtype, accumulate)
        out = torch.full((m, n), 3.0, dtype=dtype, device="cuda")
        dr.dr_qmatmul(a, b, out, accumulate=accumulate, fast=fast, workspace=ws)
        off = (out.to(torch.float64) - want - (3.0 if accumulate else 0.0)).abs()
        assert (off <= tol + (want.abs() * 2.0**-8 if dtype == torch.bfloat16 else 2.0**-20)).all()


@pytest.mark.parametrize("m", [1, 16, 20, 32])
@pytest.mark.parametrize("n,k", [(4097, 264), (16385, 130), (20001, 1160)])
@pytest.mark.parametrize("fast", [False, True])
def test_few_rows_of_wide_weights(m, n, k, fast):
    dr = _dr()
    say("few rows, wide", m, n, k, fast)
    gen = torch.Generator().manual_seed(m + n)
    w, wv = _matrix(dr, n, k, 128, n, spread=3)
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.randn((m, k), generator=gen).to(dtype)
        xv = quant.values(*quant.quantize(x.to(torch.float64).numpy(), 1), k, 1)
        want, size = quant.product(xv, wv)
        y = torch.empty((m, n), device="cuda")
        dr.dr_qlinear(x.cuda(), w, y, fast=fast, workspace=torch.empty((dr.dr_qlinear_workspace(m, w),), dtype=torch.uint8, device="cuda"))
        if fast:  # 2^-10 of each group's largest product, at most of the sum of magnitudes
            size = size * (1 + 2.0**-10 / ((-(-k // 128) * 128 + 64) * 2.0**-23))
        _close(y, want, size, k, False)


@pytest.mark.parametrize("m", [3, 40])
def test_linear_rows_at_any_element_and_not_finite(m):
    dr = _dr()
    say("linear strided", m)
    n, k = 50, 300
    w, wv = _matrix(dr, n, k, 128, 3)
    for offset, stride in ((1, 301), (8, 304)):
        x = torch.randn((m, k), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
        buf = torch.full((offset + m * stride,), float("nan"), dtype=torch.bfloat16, device="cuda")
        src = buf[offset:].view(m, stride)[:, :k]
        src.copy_(x)
        ws = torch.empty((dr.dr_qlinear_workspace(m, w),), dtype=torch.uint8, device="cuda")
        y = torch.empty((m, n), device="cuda")
        dr.dr_qlinear(src, w, y, workspace=ws)
        xv = quant.values(*quant.quantize(x.to(torch.float64).numpy(), 1), k, 1)
        _close(y, *quant.product(xv, wv), k, False)
        src[1, 7] = float("inf")
        dr.dr_qlinear(src, w, y, workspace=ws)
        nan = torch.isnan(y)
        assert nan[1].all() and int(nan.sum()) == n
    torch.cuda.synchronize()


def test_backward_is_the_gradient_of_the_forward():
    """Integers that e4m3 holds exactly: the three products are exact, and the gradients equal central differences of
    sum(y * dy) in the inputs."""
    dr = _dr()
    say("gradients by differences")
    m, n, k = 150, 200, 136
    gen = torch.Generator().manual_seed(3)
    x, w, dy = (torch.randint(-3, 4, s, generator=gen).to(torch.bfloat16) for s in ((m, k), (n, k), (m, n)))
    mats = {}
    for name, t, br in (("x", x, 1), ("w", w, 128), ("dy", dy, 1)):
        mats[name], mats[name + "t"] = dr.QMatrix.empty(*t.shape, br), dr.QMatrix.empty(t.shape[1], t.shape[0], br)
        dr.dr_quantize(t.cuda(), mats[name], mats[name + "t"])
    ws = torch.empty((max(dr.dr_qmatmul_workspace(*p) for p in ((m, n, k), (m, k, n), (n, k, m))),), dtype=torch.uint8, device="cuda")

    def forward(x_, w_):
        return x_.to(torch.float64) @ w_.to(torch.float64).t()

    y, dx, dw = torch.empty((m, n), device="cuda"), torch.empty((m, k), device="cuda"), torch.zeros((n, k), device="cuda")
    dr.dr_qmatmul(mats["x"], mats["w"], y, workspace=ws)
    dr.dr_qmatmul(mats["dy"], mats["wt"], dx, workspace=ws)
    dr.dr_qmatmul(mats["dyt"], mats["xt"], dw, accumulate=True, workspace=ws)
    assert torch.equal(y.cpu().to(torch.float64), forward(x, w))
    d64 = dy.to(torch.float64)
    loss = lambda x_, w_: float((forward(x_, w_) * d64).sum())  # noqa: E731
    for t, grad in ((x, dx), (w, dw)):
        for i, j in ((0, 0), (3, 135), (149, 71), (77, 128)):
            up, down = t.clone(), t.clone()
            up[i, j] += 1
            down[i, j] -= 1
            diff = (loss(up, w) - loss(down, w)) / 2 if t is x else (loss(x, up) - loss(x, down)) / 2
            assert float(grad[i, j]) == diff


def test_on_another_stream_and_in_a_graph():
    """A side stream's own order holds, and a replayed graph follows its inputs."""
    dr = _dr()
    say("streams and graphs")
    side = torch.cuda.Stream()
    for m in (4, 70, 400):
        n, k = 300, 520
        w, wv = _matrix(dr, n, k, 128, 9)
        x = torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
        y = torch.empty((m, n), device="cuda")
        ws = torch.empty((dr.dr_qlinear_workspace(m, w),), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            x.normal_()
            dr.dr_qlinear(x, w, y, workspace=ws)
        side.synchronize()
        ref = lambda: quant.product(quant.values(*quant.quantize(x.to(torch.float64).cpu().numpy(), 1), k, 1), wv)  # noqa: E731
        _close(y, *ref(), k, False)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dr.dr_qlinear(x, w, y, workspace=ws)
        for _ in range(3):
            x.normal_()
            y.fill_(-1)
            graph.replay()
            torch.cuda.synchronize()
            _close(y, *ref(), k, False)


@pytest.mark.parametrize("m,n,k", [(4100, 4360, 5120), (5000, 7000, 3000), (4352, 4104, 4000)])
@pytest.mark.parametrize("fast", [False, True])
def test_last_tiles_in_quarters(m, n, k, fast):
    """Somewhat more large tiles than a round of workgroups takes: the others leave as quarters, some of them outside of c."""
    dr = _dr()
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    x, w = torch.randn((m, k), generator=gen, device="cuda"), torch.randn((n, k), generator=gen, device="cuda")
    a, b = dr.QMatrix.empty(m, k, 1), dr.QMatrix.empty(n, k, 128)
    dr.dr_quantize(x, a), dr.dr_quantize(w, b)
    av = torch.from_numpy(quant.values(a.data.cpu().numpy(), a.scales.cpu().numpy(), k, 1)).cuda()
    bv = torch.from_numpy(quant.values(b.data.cpu().numpy(), b.scales.cpu().numpy(), k, 128)).cuda()
    want, size = av @ bv.t(), av.abs() @ bv.abs().t()
    tol = ((-(-k // 128) * 128 + 64) * 2.0**-23 + (2.0**-10 if fast else 0)) * size
    ws = _workspace(dr, m, n, k)
    for dtype, accumulate in ((torch.bfloat16, False), (torch.float32, False), (torch.float32, True)):
        say("quarters", m, n, k, fast, dtype, accumulate)
        buf = torch.full((m + 1, n + 16), 3.0, dtype=dtype, device="cuda")
        dr.dr_qmatmul(a, b, buf[:m, :n], accumulate=accumulate, fast=fast, workspace=ws)
        off = (buf[:m, :n].to(torch.float64) - want - (3.0 if accumulate else 0.0)).abs()
        assert (off <= tol + (want.abs() * 2.0**-8 if dtype == torch.bfloat16 else 2.0**-20)).all()
        assert (buf[m] == 3.0).all() and (buf[:, n:] == 3.0).all()


@pytest.mark.parametrize("m,n,k", [(509, 2008, 1990), (509, 2003, 512), (1200, 2000, 2000), (130, 6903, 5100), (517, 905, 4900), (260, 2600, 640), (2000, 1999, 385)])
@pytest.mark.parametrize("blocks", [(1, 128), (1, 1), (128, 128)])
def test_workgroups_with_a_cu_to_themselves(m, n, k, blocks):
    """Up to 256 tiles, whole or split along K, of four blocks and more: at the edges of c, with every kind of scales."""
    dr = _dr()
    a, av = _matrix(dr, m, k, blocks[0], m + k, spread=5, extra=16)
    b, bv = _matrix(dr, n, k, blocks[1], n + k + 1, spread=5, extra=48)
    av, bv = torch.from_numpy(av).cuda(), torch.from_numpy(bv).cuda()
    want, size = av @ bv.t(), av.abs() @ bv.abs().t()
    ws = _workspace(dr, m, n, k)
    for fast in (True, False):
        tol = ((-(-k // 128) * 128 + 64) * 2.0**-23 + (2.0**-10 if fast else 0)) * size
        for dtype, accumulate in ((torch.bfloat16, False), (torch.float32, False), (torch.float32, True)):
            say("alone on a CU", m, n, k, blocks, fast, dtype, accumulate)
            buf = torch.full((m + 1, n), 3.0, dtype=dtype, device="cuda")
            dr.dr_qmatmul(a, b, buf[:m], accumulate=accumulate, fast=fast, workspace=ws)
            off = (buf[:m].to(torch.float64) - want - (3.0 if accumulate else 0.0)).abs()
            assert (off <= tol + (want.abs() * 2.0**-8 if dtype == torch.bfloat16 else 2.0**-20)).all()
            assert (buf[m] == 3.0).all()


@pytest.mark.parametrize("m,n", [(700, 2000), (700, 2001), (4100, 4360)])
@pytest.mark.parametrize("fast", [False, True])
def test_extreme_scales_and_nan_in_tiles(m, n, fast):
    dr = _dr()
    say("extreme scales in tiles", m, n, fast)
    k = 640
    a, b = dr.QMatrix.empty(m, k, 1), dr.QMatrix.empty(n, k, 1)
    a.data.fill_(0x38), b.data.fill_(0x38)  # 1.0
    ws = _workspace(dr, m, n, k)
    out = torch.empty((m, n), device="cuda")
    for ea, eb, want in ((0, 254, 640.0), (127, 127, 640.0), (0, 127, 640 * 2.0**-127), (247, 7, 640.0), (254, 254, float("inf"))):
        a.scales.fill_(ea), b.scales.fill_(eb)
        dr.dr_qmatmul(a, b, out, fast=fast, workspace=ws)
        assert (out == want).all(), (ea, eb, out.flatten()[0].item())
    a.scales.fill_(127), b.scales.fill_(127)
    a.data[m - 1, 300] = 0x7F
    b.data[n - 1, 5] = 0xFF
    dr.dr_qmatmul(a, b, out, fast=fast, workspace=ws)
    nan = torch.isnan(out)
    assert nan[m - 1].all() and nan[:, n - 1].all() and int(nan.sum()) == m + n - 1


@pytest.mark.parametrize("m", [33, 47, 63, 64, 130])
@pytest.mark.parametrize("n,k", [(1000, 130), (4097, 264), (9217, 900), (200, 3000)])
@pytest.mark.parametrize("fast", [False, True])
def test_small_products(m, n, k, fast):
    """Two, three and four times 16 rows a workgroup."""
    dr = _dr()
    a, av = _matrix(dr, m, k, 1, m + k, spread=5)
    b, bv = _matrix(dr, n, k, 128, n + k + 1, spread=5)
    want, size = quant.product(av, bv)
    ws = _workspace(dr, m, n, k)
    for dtype in (torch.float32, torch.bfloat16):
        say("small", m, n, k, fast, dtype)
        out = torch.full((m + 1, n), 7.0, dtype=dtype, device="cuda")
        dr.dr_qmatmul(a, b, out[:m], fast=fast, workspace=ws)
        torch.cuda.synchronize()
        if fast:  # 2^-10 of each group's largest product, at most of the sum of magnitudes
            _close(out[:m], want, size * (1 + 2.0**-10 / ((-(-k // 128) * 128 + 64) * 2.0**-23)), k, dtype == torch.bfloat16)
        else:
            _close(out[:m], want, size, k, dtype == torch.bfloat16)
        assert (out[m] == 7.0).all()
