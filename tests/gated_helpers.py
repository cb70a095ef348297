"""Matrices and tolerances of the gated block's tests.

What a kernel computes in fp32 and quantizes may differ from the value in 64 bits by a tolerance, so a block's largest
magnitude may too: its scale has to be the one of a maximum within the tolerance, and each element within half a step of
e4m3 (2^-4 of itself, 2^-10 of the scale below the scale's 2^-6) of the value, beside the tolerance.
"""
import numpy as np
import torch

from oracle import quant

POISON = 0xA5


def poisoned(dr, rows, cols, extra=16, block_rows=1):
    """(matrix, its data with `extra` bytes behind each row and a row more, its scales with 16 bytes more), all filled."""
    m = dr.QMatrix.empty(rows, cols, block_rows)
    wide = torch.full((rows + 1, m.data.shape[1] + extra), POISON, dtype=torch.uint8, device="cuda")
    scales = torch.full((m.scales.numel() + 16,), POISON, dtype=torch.uint8, device="cuda")
    q = dr.QMatrix(wide[:rows], scales[:m.scales.numel()].view(m.scales.shape), rows, cols, block_rows)
    return q, wide, scales


def quantized(dr, x, block_rows=1, extra=0):
    """x (numpy) in 8 bits on the device, NaN codes behind each row, and what it stands for."""
    codes, scales = quant.quantize(x, block_rows)
    wide = torch.full((x.shape[0], codes.shape[1] + extra), 0x7F, dtype=torch.uint8, device="cuda")
    wide[:, :codes.shape[1]] = torch.from_numpy(codes).cuda()
    return dr.QMatrix(wide, torch.from_numpy(scales).cuda(), *x.shape, block_rows), quant.values(codes, scales, x.shape[1], block_rows)


def check_rows(made, want, tol, name):
    """`made` (of poisoned()) holds `want` within `tol` (both [rows, cols]; NaN where NaN is due), and nothing else is touched."""
    q, wide, scales = made
    rows, cols = want.shape
    padded = -(-cols // 128) * 128
    data, sc = wide.cpu().numpy(), scales.cpu().numpy()
    assert (data[rows:] == POISON).all() and (data[:, padded:] == POISON).all(), f"{name}: written outside the matrix"
    assert (data[:rows, cols:padded] == 0).all(), f"{name}: columns behind the last are not 0"
    used = q.scales.numel()
    assert (sc[used:] == POISON).all(), f"{name}: scales written outside"
    laid = sc[:used].reshape(tuple(q.scales.shape)).transpose(1, 0, 2).reshape(rows, -1)
    assert (laid[:, padded // 128:] == 127).all(), f"{name}: unused scales are not 127"
    code = laid[:, :padded // 128].astype(np.int64)
    fine = np.isfinite(want)
    pad = ((0, 0), (0, padded - cols))
    mag = np.pad(np.where(fine, np.abs(want), 0.0), pad).reshape(rows, -1, 128)
    off = np.pad(np.where(fine, tol, 0.0), pad).reshape(rows, -1, 128)

    def scale_of(amax):
        with np.errstate(divide="ignore"):
            m, e = np.frexp(amax / 448.0)
        return np.where(amax == 0, 127, np.maximum(np.where(m == 0.5, e - 1, e), -127) + 127)

    lo, hi = scale_of(np.maximum(mag - off, 0).max(axis=2)), scale_of((mag + off).max(axis=2))
    surely = np.maximum(mag - off, 0).max(axis=2) > 0  # else the block may count as one of zeros
    ok = (code == 127) & ~surely | (code >= np.where(surely, lo, 0)) & (code <= hi)
    assert ok.all(), (name, np.argwhere(~ok)[:4].tolist(), code[~ok][:4], lo[~ok][:4], hi[~ok][:4])
    scale = np.repeat(2.0**(code - 127.0), 128, axis=1)[:, :cols]
    got = quant.E4M3[data[:rows, :cols]] * scale
    assert np.array_equal(np.isnan(got), ~fine), f"{name}: NaN in other places"
    bound = np.maximum(np.abs(want) * 2.0**-4, scale * 2.0**-10) * (1 + 2.0**-20) + 2 * tol
    bad = fine & ~(np.abs(np.where(fine, got - want, 0.0)) <= np.where(fine, bound, 0.0))
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])
