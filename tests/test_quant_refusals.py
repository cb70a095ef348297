"""Arguments that the 8-bit and gradient calls refuse: each is refused before any HIP call, so this needs no GPU."""
import ctypes
import math

import pytest

from paper_2607_22614_amd import dr

P = 1 << 20  # an aligned address that nothing may touch


def _q(rows=4, cols=200, block_rows=1, **kw):
    f = {"data": P, "scales": P, "rows": rows, "cols": cols, "stride": -(-cols // 128) * 128, "block_rows": block_rows, "reserved": 0, **kw}
    return dr.dr_qmatrix(*[f[n] for n, _ in dr.dr_qmatrix._fields_])


def _refused(rc, text):
    assert rc == dr.DR_EINVAL
    assert text in dr.dr_last_error(), dr.dr_last_error()


BAD = [({"rows": -1}, "rows are below"), ({"rows": 1 << 26}, "rows are below"), ({"cols": (1 << 23) + 1}, "columns at most"),
       ({"block_rows": 64}, "blocks of 64"), ({"stride": 128}, "stride"), ({"stride": 264}, "stride"), ({"stride": 1 << 24}, "stride"),
       ({"data": 0}, "null or misaligned"), ({"data": P + 8}, "null or misaligned"), ({"scales": 0}, "null or misaligned"),
       ({"scales": P + 2}, "null or misaligned"), ({"reserved": 1}, "reserved")]


@pytest.mark.parametrize("bad,text", BAD, ids=[str(b) for b, _ in BAD])
def test_matrices(bad, text):
    good, q = _q(), _q(**bad)
    lib = dr._lib
    _refused(lib.dr_qmatmul(q, good, P, 0, 1 << 30, 0, None, 0, None), text)
    _refused(lib.dr_qmatmul(good, q, P, 0, 1 << 30, 0, None, 0, None), text)
    _refused(lib.dr_quantize(P, 0, q.rows, q.cols, max(q.cols, 1), q, None, None), text)
    _refused(lib.dr_qlinear(P, 0, 1, q.cols, q, P, 0, 1 << 30, 0, None, 0, None), text)


def test_quantize():
    lib = dr._lib
    _refused(lib.dr_quantize(P, 0, 4, 200, 200, None, None, None), "neither")
    _refused(lib.dr_quantize(P, 0, 5, 200, 200, _q(), None, None), "q is not")
    _refused(lib.dr_quantize(P, 0, 4, 200, 200, None, _q(), None), "qt is not")
    _refused(lib.dr_quantize(P, 0, 4, 200, 200, _q(), _q(200, 4, 128), None), "differ in block_rows")
    _refused(lib.dr_quantize(P, 2, 4, 200, 200, _q(), None, None), "unknown type")
    _refused(lib.dr_quantize(P, 0, 4, 200, 199, _q(), None, None), "row stride")
    _refused(lib.dr_quantize(0, 0, 4, 200, 200, _q(), None, None), "null or misaligned")
    _refused(lib.dr_quantize(P + 2, 0, 4, 200, 200, _q(), None, None), "null or misaligned")
    _refused(lib.dr_quantize(P + 1, 1, 4, 200, 200, _q(), None, None), "null or misaligned")
    big = _q((1 << 26) - 1, 1 << 23)
    _refused(lib.dr_quantize(P, 0, big.rows, big.cols, big.cols, big, None, None), "2^24 tiles")


def test_products():
    lib = dr._lib
    a, b = _q(), _q(7, 200, 128)
    _refused(lib.dr_qmatmul(None, b, P, 0, 7, 0, None, 0, None), "a is null")
    _refused(lib.dr_qmatmul(a, _q(7, 201), P, 0, 7, 0, None, 0, None), "columns")
    _refused(lib.dr_qmatmul(a, b, P, 3, 7, 0, None, 0, None), "unknown type")
    _refused(lib.dr_qmatmul(a, b, P, 0, 6, 0, None, 0, None), "row stride")
    _refused(lib.dr_qmatmul(a, b, 0, 0, 7, 0, None, 0, None), "null or misaligned")
    _refused(lib.dr_qmatmul(a, b, P + 2, 0, 7, 0, None, 0, None), "null or misaligned")
    _refused(lib.dr_qmatmul(a, b, P, 1, 7, 1, None, 0, None), "ACCUMULATE")
    _refused(lib.dr_qmatmul(a, b, P, 0, 7, 4, None, 0, None), "unknown flags")
    n = ctypes.c_uint64()
    _refused(lib.dr_qmatmul_workspace(-1, 2, 3, n), "rows are below")
    _refused(lib.dr_qmatmul_workspace(1, 2, 3, None), "null")


def test_linear():
    lib = dr._lib
    w = _q(7, 200, 128)
    need = dr._bytes(lib.dr_qlinear_workspace, "", 100, 7, 200)
    assert need > 0 and dr._bytes(lib.dr_qlinear_workspace, "", 1, 7, 200) == 0
    _refused(lib.dr_qlinear(P, 0, 100, 200, w, P, 0, 7, 0, P, need - 1, None), "workspace")
    _refused(lib.dr_qlinear(P, 0, 100, 200, w, P, 0, 7, 0, None, need, None), "workspace")
    _refused(lib.dr_qlinear(P, 0, 100, 200, w, P, 0, 7, 0, P + 8, need, None), "workspace")
    _refused(lib.dr_qlinear(P, 0, 1, 199, w, P, 0, 7, 0, None, 0, None), "row stride")
    _refused(lib.dr_qlinear(P, 5, 1, 200, w, P, 0, 7, 0, None, 0, None), "unknown type")
    _refused(lib.dr_qlinear(P, 0, 1, 200, w, P, 5, 7, 0, None, 0, None), "unknown type")
    _refused(lib.dr_qlinear(P, 0, -1, 200, w, P, 0, 7, 0, None, 0, None), "rows are below")
    _refused(lib.dr_qlinear(P, 0, 1, 200, w, P, 0, 7, 1, None, 0, None), "unknown flags")
    _refused(lib.dr_qlinear(P, 0, 1, 200, None, P, 0, 7, 0, None, 0, None), "w is null")


def test_sizes():
    assert dr.dr_qmatrix_sizes(5, 129, 1) == {"stride": 256, "data_bytes": 1280, "scale_bytes": 20}
    assert dr.dr_qmatrix_sizes(129, 513, 128) == {"stride": 640, "data_bytes": 129 * 640, "scale_bytes": 16}
    assert dr.dr_qmatrix_sizes(0, 0, 1) == {"stride": 0, "data_bytes": 0, "scale_bytes": 0}
    with pytest.raises(dr.DrError):
        dr.dr_qmatrix_sizes(1, 1, 2)


def _g(**kw):
    f = {"grad": P, "out": P, "numel": 10, "grad_type": 0, "out_type": 0, **kw}
    return (dr.dr_grad * 1)(dr.dr_grad(*[f[n] for n, _ in dr.dr_grad._fields_]))


def test_gradients():
    lib = dr._lib
    for bad, text in (({"grad": 0}, "null or misaligned"), ({"grad": P + 2}, "null or misaligned"), ({"grad_type": 2}, "unknown type"),
                      ({"numel": -1}, "elements"), ({"numel": (1 << 45) + 1}, "elements")):
        _refused(lib.dr_grad_norm(_g(**bad), 1, P, None, P, None), text)
        _refused(lib.dr_grad_scale(_g(**bad), 1, P, 1.0, None, None), text)
        _refused(lib.dr_grad_clip(_g(**bad), 1, 1.0, P, None, None), text)
    for bad, text in (({"out": 0}, "null or misaligned"), ({"out": P + 1, "out_type": 1}, "null or misaligned"), ({"out_type": 7}, "unknown type"),
                      ({"out_type": 1}, "in place to another type")):
        _refused(lib.dr_grad_scale(_g(**bad), 1, P, 1.0, None, None), text)
        _refused(lib.dr_grad_clip(_g(**bad), 1, 1.0, P, None, None), text)
    for bad in (-1.0, math.nan):
        _refused(lib.dr_grad_scale(_g(), 1, P, bad, None, None), "max_norm")
        _refused(lib.dr_grad_clip(_g(), 1, bad, P, None, None), "max_norm")
    _refused(lib.dr_grad_norm(None, 1, P, None, None, None), "null")
    _refused(lib.dr_grad_norm(_g(), -1, P, None, None, None), "list of -1")
    _refused(lib.dr_grad_norm(_g(), 1, 0, None, None, None), "workspace")
    _refused(lib.dr_grad_norm(_g(), 1, P, P + 4, None, None), "misaligned result")
    _refused(lib.dr_grad_scale(_g(), 1, 0, 1.0, None, None), "sum_squares")
    _refused(lib.dr_grad_clip(_g(), 1, 1.0, P + 4, None, None), "workspace")
