"""Arguments that the gated block's calls refuse: each is refused before any HIP call, so this needs no GPU."""
import ctypes

import pytest

from paper_2607_22614_amd import dr

P = 1 << 20  # an aligned address that nothing may touch
LOTS = 1 << 40


def _q(rows=4, cols=200, block_rows=1, **kw):
    f = {"data": P, "scales": P, "rows": rows, "cols": cols, "stride": -(-cols // 128) * 128, "block_rows": block_rows, "reserved": 0, **kw}
    return dr.dr_qmatrix(*[f[n] for n, _ in dr.dr_qmatrix._fields_])


def _refused(rc, text):
    assert rc == dr.DR_EINVAL
    assert text in dr.dr_last_error(), dr.dr_last_error()


BAD = [({"rows": -2}, "rows are below"), ({"rows": 1 << 26}, "rows are below"), ({"cols": (1 << 23) + 1}, "columns at most"),
       ({"block_rows": 64}, "blocks of 64"), ({"stride": 128}, "stride"), ({"stride": 264}, "stride"), ({"stride": 1 << 24}, "stride"),
       ({"data": 0}, "null or misaligned"), ({"data": P + 8}, "null or misaligned"), ({"scales": 0}, "null or misaligned"),
       ({"scales": P + 2}, "null or misaligned"), ({"reserved": 1}, "reserved")]


@pytest.mark.parametrize("bad,text", BAD, ids=[str(b) for b, _ in BAD])
def test_matrices(bad, text):
    good, q, lib = _q(), _q(**bad), dr._lib
    _refused(lib.dr_qgated(P, 0, 1, 200, q, 0, P, 0, 1 << 30, 0, P, LOTS, None), text)
    _refused(lib.dr_qgated_save(q, good, 0, _q(4, 2), None, None, 0, P, LOTS, None), text)
    _refused(lib.dr_qgated_save(good, q, 0, _q(4, 2), None, None, 0, P, LOTS, None), text)
    _refused(lib.dr_qgated_save(good, good, 0, q, None, None, 0, P, LOTS, None), text)
    _refused(lib.dr_gated_backward(P, 0, 1 << 30, q, good, 0, _q(4, 400), None, None, None), text)
    _refused(lib.dr_gated_backward(P, 0, 1 << 30, good, q, 0, _q(4, 400), None, None, None), text)
    _refused(lib.dr_gated_backward(P, 0, 200, good, good, 0, q, None, None, None), text)
    _refused(lib.dr_gated_backward(P, 0, 200, good, good, 0, None, q, None, None), text)
    _refused(lib.dr_gated_backward(P, 0, 200, good, good, 0, None, None, q, None), text)
    _refused(lib.dr_qtranspose(q, _q(200, 4), None), text)
    _refused(lib.dr_qtranspose(good, q, None), text)


def test_gated():
    lib, w = dr._lib, _q(4000, 2000, 128)
    need = dr._bytes(lib.dr_qgated_workspace, "", 300, 2000, 2000)

    def call(x=P, x_type=0, m=300, x_stride=2000, w=w, act=0, h=P, h_type=0, h_stride=2000, flags=0, ws=P, have=need):
        return lib.dr_qgated(x, x_type, m, x_stride, w, act, h, h_type, h_stride, flags, ws, have, None)

    _refused(call(w=None), "w is null")
    _refused(call(w=_q(13, 200, 128)), "13 rows")
    _refused(call(act=2), "unknown activation")
    _refused(call(act=-1), "unknown activation")
    _refused(call(m=-1), "rows are below")
    _refused(call(m=1 << 26), "rows are below")
    _refused(call(x=0), "x is null or misaligned")
    _refused(call(x=P + 2), "x is null or misaligned")
    _refused(call(x_type=2), "unknown type")
    _refused(call(x_stride=1999), "row stride")
    _refused(call(h=0), "h is null or misaligned")
    _refused(call(h=P + 1, h_type=1), "h is null or misaligned")
    _refused(call(h_type=5), "unknown type")
    _refused(call(h_stride=1999), "row stride")
    _refused(call(flags=1), "unknown flags")
    _refused(call(flags=4), "unknown flags")
    assert need > 0
    _refused(call(have=300 * 2048), "workspace")
    _refused(call(ws=None), "workspace")
    _refused(call(ws=P + 8), "workspace")
    big = _q((1 << 26) - 2, 128, 128)
    _refused(call(m=1 << 25, w=big, x_stride=200, h_stride=1 << 30, have=LOTS), "inner columns")
    wide = _q(1 << 24, 128, 128)
    _refused(call(m=1 << 15, w=wide, h_stride=1 << 30, have=LOTS), "results")


def test_save():
    lib = dr._lib
    x, w, h, c = _q(100, 200), _q(14, 200, 128), _q(100, 7), _q(100, 7)
    need = dr._bytes(lib.dr_qgated_save_workspace, "", 100, 7, 200)

    def call(x=x, w=w, act=0, h=h, gate=c, up=c, flags=0, ws=P, have=need):
        return lib.dr_qgated_save(x, w, act, h, gate, up, flags, ws, have, None)

    _refused(call(x=None), "x is null")
    _refused(call(w=None), "w is null")
    _refused(call(h=None), "h is null")
    _refused(call(x=_q(100, 201)), "columns")
    _refused(call(w=_q(13, 200, 128)), "13 rows")
    _refused(call(act=2), "unknown activation")
    _refused(call(h=_q(99, 7)), "h is 99 x 7")
    _refused(call(h=_q(100, 14)), "h is 100 x 14")
    _refused(call(h=_q(100, 7, 128)), "blocks of 128")
    _refused(call(gate=None), "without the other")
    _refused(call(up=None), "without the other")
    _refused(call(gate=_q(100, 8)), "gate is 100 x 8")
    _refused(call(up=_q(101, 7)), "up is 101 x 7")
    _refused(call(up=_q(100, 7, 128)), "blocks of 128")
    _refused(call(flags=1), "unknown flags")
    if need:
        _refused(call(have=need - 1), "workspace")
        _refused(call(ws=None), "workspace")
        _refused(call(ws=P + 8), "workspace")


def test_backward():
    lib = dr._lib
    c = _q(100, 7)

    def call(dh=P, kind=0, stride=7, gate=c, up=c, act=0, d=None, dt=None, ht=None):
        return lib.dr_gated_backward(dh, kind, stride, gate, up, act, d, dt, ht, None)

    d, dt, ht = _q(100, 14), _q(14, 100), _q(7, 100)
    _refused(call(), "none of")
    _refused(call(gate=None, d=d), "gate is null")
    _refused(call(up=None, d=d), "up is null")
    _refused(call(gate=_q(100, 7, 128), d=d), "blocks of 128")
    _refused(call(up=_q(100, 7, 128), d=d), "blocks of 128")
    _refused(call(up=_q(100, 8), d=d), "up is 100 x 8")
    _refused(call(act=7, d=d), "unknown activation")
    _refused(call(dh=0, d=d), "dh is null or misaligned")
    _refused(call(dh=P + 2, d=d), "dh is null or misaligned")
    _refused(call(kind=3, d=d), "unknown type")
    _refused(call(stride=6, d=d), "row stride")
    _refused(call(d=_q(100, 7)), "d is 100 x 7")
    _refused(call(d=d, dt=_q(100, 14)), "dt is 100 x 14")
    _refused(call(dt=dt, ht=dt), "ht is 14 x 100")
    _refused(call(d=_q(100, 14, 128)), "blocks of 128")
    _refused(call(dt=_q(14, 100, 128)), "blocks of 128")
    _refused(call(ht=_q(7, 100, 128)), "blocks of 128")
    # two columns of up past half of the limit; more tiles than a launch holds
    _refused(call(gate=_q(4, (1 << 22) + 1), up=_q(4, (1 << 22) + 1), stride=1 << 23, d=_q(4, (1 << 23) + 2)), "columns at most")
    many = _q((1 << 26) - 1, 1 << 22)
    _refused(call(gate=many, up=many, stride=1 << 22, d=_q((1 << 26) - 1, 1 << 23)), "tiles")


def test_turned():
    lib = dr._lib
    _refused(lib.dr_qtranspose(None, _q(200, 4), None), "src is null")
    _refused(lib.dr_qtranspose(_q(), None, None), "qt is null")
    _refused(lib.dr_qtranspose(_q(), _q(), None), "qt is 4 x 200")
    _refused(lib.dr_qtranspose(_q(), _q(200, 4, 128), None), "blocks of 128")
    _refused(lib.dr_qtranspose(_q((1 << 23), 1 << 23), _q(1 << 23, 1 << 23), None), "tiles")


def test_workspaces():
    n = ctypes.c_uint64()
    for call in (dr._lib.dr_qgated_workspace, dr._lib.dr_qgated_save_workspace):
        _refused(call(1, 2, 3, None), "null")
        _refused(call(-1, 2, 3, n), "rows are below")
        _refused(call(1, -2, 3, n), "inner columns")
        _refused(call(1, (1 << 23) + 1, 3, n), "inner columns")
        _refused(call(1, 2, -3, n), "columns at most")
        _refused(call(1 << 25, 1 << 23, 3, n), "results")
        assert call(0, 5, 5, n) == 0 and n.value == 0
        assert call(5, 0, 5, n) == 0 and n.value == 0
