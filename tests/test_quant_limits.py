"""Sizes that dr_quantize refuses because a launch cannot hold them: before any HIP call, so this needs no GPU."""
import pytest

from paper_2607_22614_amd import dr

P = 1 << 20  # an aligned address that nothing may touch


def _q(rows, cols, block_rows):
    return dr.dr_qmatrix(P, P, rows, cols, -(-cols // 128) * 128, block_rows, 0)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,text", [(1 << 24, 1 << 13, "2^23 or more tiles"), ((1 << 23) - 127, (1 << 14) - 127, "2^23 or more tiles"),
                                            (1 << 18, (1 << 21) + 1, "more than 2^24 tiles")])
def test_more_lanes_than_a_launch_holds(rows, cols, text, block_rows):
    """A tile of 128 x 128 is a workgroup of 512 lanes, and a launch holds 2^32 - 1 of them."""
    q = _q(rows, cols, block_rows)
    for qt in (None, _q(cols, rows, block_rows) if rows <= 1 << 23 else None):
        rc = dr._lib.dr_quantize(P, 1, rows, cols, cols, q, qt, None)
        assert rc == dr.DR_EINVAL and text in dr.dr_last_error(), (rc, dr.dr_last_error())
