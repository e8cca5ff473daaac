"""Pins of the 8-bit oracle: format tables, scales, rounding."""
import numpy as np
import pytest
import torch

from oracle import fp8 as O

TORCH = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_code_values(fmt):
    theirs = torch.arange(256, dtype=torch.uint8).view(TORCH[fmt]).double().numpy()
    assert np.array_equal(O.code_values(fmt), theirs, equal_nan=True)
    assert np.nanmax(np.where(np.isinf(theirs), np.nan, theirs)) == O.FORMATS[fmt][2]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("tile", [False, True])
def test_rounding_and_scale(fmt, tile):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((150, 300)) * np.exp(3 * rng.standard_normal((150, 300)))
    codes, scales = O.quantize(x, fmt, tile)
    assert codes.shape == (150, 384) and scales.shape == (150, 3) and not codes[:, 300:].any()
    v = O.values(codes, scales, fmt, 300)
    s = np.repeat(2.0 ** (scales.astype(float) - 127.0), 128, axis=1)[:, :300]
    top, frac, low = O.FORMATS[fmt][2], O.FORMATS[fmt][0], 1 - O.FORMATS[fmt][1]
    # at most half a step, and within the format although a scale of half the size would not do
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.abs(x) / s)), low) - frac)
    assert (np.abs(v - x) <= 0.5 * step * s).all()
    assert (np.abs(x) <= top * s).all()
    blocks = np.add.reduceat((np.abs(x) > top * s / 2).astype(int), [0, 128, 256], axis=1)
    if tile:
        blocks = np.add.reduceat(blocks, [0, 128], axis=0)
    assert (blocks > 0).all()
    r = torch.tensor((x / s).astype(np.float32)).to(TORCH[fmt]).view(torch.uint8).numpy()
    same32 = (x / s).astype(np.float32).astype(np.float64) == x / s
    assert (r == codes[:, :300])[same32].all()


def test_ties_zeros_and_specials():
    x = np.zeros((4, 128))
    x[0, :6] = [448.0, 1.0625, 1.1875, -1.0625, 2.0 ** -10, 3 * 2.0 ** -10]   # between two values each
    x[1, 5] = np.nan
    x[2, 7] = -np.inf
    codes, scales = O.quantize(x, "e4m3")
    assert O.values(codes, scales, "e4m3", 128)[0, :6].tolist() == [448.0, 1.0, 1.25, -1.0, 0.0, 2.0 ** -8]
    assert scales[:, 0].tolist() == [127, 255, 255, 0]
    assert (codes[1:3] == O.NAN_CODE).all() and not codes[3].any()
    assert np.isnan(O.values(codes, scales, "e4m3", 128)[1:3]).all()


def test_scale_bytes_are_packed_by_four_blocks():
    s = np.arange(3 * 6, dtype=np.uint8).reshape(3, 6) + 1
    p = O.pack_scales(s)
    assert p.size == 4 * 3 * 2
    for r in range(3):
        for j in range(8):
            assert p[((j // 4) * 3 + r) * 4 + j % 4] == (s[r, j] if j < 6 else 0)
