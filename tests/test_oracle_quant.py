"""The oracle of the 8-bit matrices against independent statements of the format and of its own definition."""
import numpy as np
import pytest
import torch

from oracle import quant


def test_codes_are_the_format():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(quant.E4M3, want, equal_nan=True)
    assert quant.E4M3[0x7E] == 448.0 and quant.E4M3[1] == 2.0**-9 and np.isnan(quant.E4M3[0x7F])


def test_rounding_is_nearest_even():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 2.0**rng.uniform(-12, 8, 20000)])
    mid = (quant.E4M3[:126] + quant.E4M3[1:127]) / 2  # ties
    x = np.clip(np.concatenate([x, mid, -mid, [0.0, -0.0, 448.0, -448.0]]), -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(quant.round_e4m3(x.astype(np.float64)), want)
    assert (quant.round_e4m3(np.array([np.nan, np.inf])) == 0x7F).all()


@pytest.mark.parametrize("block_rows", [1, 128])
def test_scales_are_the_smallest_that_fit(block_rows):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((130, 300)) * 2.0**rng.integers(-40, 40, (130, 1))
    x[5] = 0
    codes, scales = quant.quantize(x, block_rows)
    assert codes.shape == (130, 384) and scales.shape == (1, -(-130 // block_rows), 4)
    assert (codes[:, 300:] == 0).all() and (scales[:, :, 3] == 127).all()
    per = scales.transpose(1, 0, 2).reshape(scales.shape[1], -1).astype(np.float64) - 127
    for i in range(per.shape[0]):
        for j in range(3):
            top = np.abs(x[i * block_rows:(i + 1) * block_rows, j * 128:(j + 1) * 128]).max()
            assert (top == 0 and per[i, j] == 0) or 224 < top / 2.0**per[i, j] <= 448
    v = quant.values(codes, scales, 300, block_rows)
    # 4 significant bits, or half a step of 2^-9 below 2^-6
    full = np.repeat(np.repeat(2.0**per, block_rows, 0)[:130], 128, 1)[:, :300]
    assert (np.abs(v - x) <= np.maximum(np.abs(x) / 16, full * 2.0**-10)).all()


def test_square_blocks_quantize_the_transpose_alike():
    x = np.random.default_rng(2).standard_normal((200, 300))
    a, sa = quant.quantize(x, 128)
    b, sb = quant.quantize(x.T, 128)
    assert np.array_equal(quant.values(a, sa, 300, 128), quant.values(b, sb, 200, 128).T)


def test_clip():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    norm, out = quant.clip(g, 1.0)
    assert norm == 5.0 and np.allclose(out[0], [3 / (5 + 1e-6), 0])
    assert np.array_equal(quant.clip(g, 6.0)[1][1], g[1]) and np.array_equal(quant.clip(g, np.inf)[1][0], g[0])
