"""Matrices in 8-bit floating point with a power-of-two scale for each block of 128, in 64 bits.

A block's scale is 2^(e - 127), e >= 0 the smallest whole number for which the block's largest magnitude is at
most the format's largest value times the scale; a code stands for the value of the format nearest to x / scale,
of two equally near ones for the one with the even fraction.  e = 255 marks a block with a NaN or an infinity.
"""
import numpy as np

BLOCK = 128
# fraction bits, exponent bias, largest value
FORMATS = {"e4m3": (3, 7, 448.0), "e5m2": (2, 15, 57344.0)}
NAN_CODE = 0x7F


def code_values(fmt):
    """The value of each of the 256 codes."""
    frac, bias, _ = FORMATS[fmt]
    c = np.arange(256)
    e, f = (c & 0x7F) >> frac, c & ((1 << frac) - 1)
    v = np.where(e == 0, f * 2.0 ** (1 - bias - frac), (1.0 + f / 2.0 ** frac) * 2.0 ** (e.astype(float) - bias))
    if fmt == "e4m3":
        v[(c & 0x7F) == 0x7F] = np.nan
    else:
        v[e == 31] = np.where(f[e == 31] == 0, np.inf, np.nan)
    return np.where(c & 0x80, -v, v)


def _nearest(v, fmt):
    """Codes of the values nearest to v (|v| at most the largest value): by search among the format's values."""
    values = code_values(fmt)[:0x80]
    values = values[np.isfinite(values)]                    # non-negative, ascending: code = index
    a = np.abs(v)
    hi = np.clip(np.searchsorted(values, a), 1, len(values) - 1)
    lo = hi - 1
    below, above = a - values[lo], values[hi] - a           # exact: few bits apart
    code = np.where(below < above, lo, np.where(below > above, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def _pad(x, rows, cols):
    p = np.zeros((rows, cols))
    p[:x.shape[0], :x.shape[1]] = x
    return p


def quantize(x, fmt, tile=False):
    """(codes (rows, padded cols) uint8, scale bytes (rows, blocks) uint8) of a float64 matrix."""
    rows, cols = x.shape
    tall = BLOCK if tile else 1
    R, C = -(-rows // tall) * tall, -(-cols // BLOCK) * BLOCK
    b = _pad(x, R, C).reshape(R // tall, tall, C // BLOCK, BLOCK)
    amax = np.abs(b).max(axis=(1, 3))
    bad = ~np.isfinite(amax)
    top = FORMATS[fmt][2]
    e = np.zeros(amax.shape, dtype=np.int64)
    for i in np.ndindex(amax.shape):
        while not bad[i] and amax[i] > top * 2.0 ** (e[i] - 127.0):
            e[i] += 1 if e[i] > 100 else 50 if amax[i] > top * 2.0 ** (e[i] - 77.0) else 1
    e[bad] = 255
    scale = np.where(bad, 1.0, 2.0 ** (e - 127.0))[:, None, :, None]
    with np.errstate(invalid="ignore"):
        codes = np.where(bad[:, None, :, None], NAN_CODE, _nearest(np.where(bad[:, None, :, None], 0.0, b) / scale, fmt))
    scales = np.repeat(e, tall, axis=0)[:rows]
    return codes.reshape(R, C)[:rows].astype(np.uint8), scales.astype(np.uint8)


def pack_scales(scales):
    """Byte of (row r, block j) at ((j // 4) * rows + r) * 4 + j % 4, zeros behind the last block."""
    rows, blocks = scales.shape
    out = np.zeros((-(-blocks // 4), rows, 4), dtype=np.uint8)
    for j in range(blocks):
        out[j // 4, :, j % 4] = scales[:, j]
    return out.reshape(-1)


def values(codes, scales, fmt, cols):
    """The values that codes (rows, padded) and scale bytes (rows, blocks) stand for."""
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(float) - 127.0))
    return (code_values(fmt)[codes] * np.repeat(s, BLOCK, axis=1))[:, :cols]
