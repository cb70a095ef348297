"""The 8-bit matrices, their products and gradient clipping, from their definitions, in 64 bits on the CPU.

quantize     codes and scales of a matrix: e4m3 (1 sign, 4 exponent, 3 mantissa bits, bias 7, largest 448, no
             infinity, NaN 0x7F) and one power of two per block of block_rows x 128 elements
values       what codes and scales stand for
product      a b^T of two 8-bit matrices
clip         the global norm of gradients and what clipping makes of them
"""
from __future__ import annotations

import numpy as np

BLOCK = 128


def _table() -> np.ndarray:
    """Value of each of the 256 e4m3 codes."""
    code = np.arange(256)
    e, m = (code >> 3) & 15, (code & 7).astype(np.float64)
    v = np.where(e == 0, m / 8 * 2.0**-6, (1 + m / 8) * 2.0**(e - 7.0))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(code >= 128, -v, v)


E4M3 = _table()


def round_e4m3(x: np.ndarray) -> np.ndarray:
    """Codes of the nearest values of x (|x| <= 448 or not finite), ties to the even code; NaN for what is not finite."""
    mag = E4M3[:127]  # 0 .. 448, in order
    a = np.abs(x)
    finite = np.isfinite(x)
    a = np.where(finite, a, 0.0)
    hi = np.searchsorted(mag, a)  # first value >= a
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = a - mag[lo], mag[hi] - a
    take_lo = (below < above) | ((below == above) & (lo % 2 == 0))
    code = np.where(finite, np.where(take_lo, lo, hi), 127)
    return (code | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def quantize(x: np.ndarray, block_rows: int) -> tuple[np.ndarray, np.ndarray]:
    """(codes [rows, cols padded to 128], scale codes [column blocks / 4, row blocks, 4])."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // BLOCK)
    codes = np.zeros((rows, nc * BLOCK), dtype=np.uint8)
    scales = np.full((-(-nc // 4), nr, 4), 127, dtype=np.uint8)
    for i in range(nr):
        for j in range(nc):
            block = x[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK]
            fine = np.abs(block[np.isfinite(block)])
            amax = fine.max() if fine.size else 0.0
            e = 0
            if amax > 0:
                e = -127
                while amax > 448.0 * 2.0**e:
                    e += 1
            codes[i * block_rows:(i + 1) * block_rows, j * BLOCK:j * BLOCK + block.shape[1]] = round_e4m3(block * 2.0**-e)
            scales[j // 4, i, j % 4] = e + 127
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray, cols: int, block_rows: int) -> np.ndarray:
    per = 2.0**(scales.transpose(1, 0, 2).reshape(scales.shape[1], -1).astype(np.float64) - 127)
    per = np.repeat(np.repeat(per, block_rows, axis=0)[:codes.shape[0]], BLOCK, axis=1)
    return E4M3[codes][:, :cols] * per[:, :cols]


def product(a: np.ndarray, b: np.ndarray) -> tuple[np.ndarray, np.ndarray]:
    """a b^T of values, and the sum of the products' magnitudes (what rounding errors are measured by)."""
    return a @ b.T, np.abs(a) @ np.abs(b).T


def clip(grads, max_norm: float) -> tuple[float, list[np.ndarray]]:
    norm = float(np.sqrt(sum(np.sum(np.square(np.asarray(g, dtype=np.float64))) for g in grads)))
    factor = 1.0 if max_norm == np.inf or norm < max_norm - 1e-6 else max_norm / (norm + 1e-6)
    return norm, [np.asarray(g, dtype=np.float64) * min(1.0, factor) for g in grads]
