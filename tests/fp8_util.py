"""8-bit floating-point blocks on the CPU, in 64 bits, written from the formats'
definitions: a table of every code's value, and the nearest one by its midpoints."""
from __future__ import annotations

import numpy as np

BLOCK = 128
# bits of the fraction, exponent bias, codes 0 .. top (of one sign) that are finite
FORMATS = {"e4m3": (3, 7, 0x7E), "e5m2": (2, 15, 0x7B)}


def table(fmt):
    """The values of codes 0 .. top, ascending."""
    frac, bias, top = FORMATS[fmt]
    code = np.arange(top + 1)
    e, f = code >> frac, code & ((1 << frac) - 1)
    return np.where(e == 0, f * 2.0 ** (1 - bias - frac), (1.0 + f / (1 << frac)) * 2.0 ** (e.astype(float) - bias))


def quantize(x, fmt):
    """(codes uint8 [rows, len], scale bytes uint8 [rows, blocks]) of FP32 x; NaN codes are
    0x7F or 0xFF, or any NaN's in e5m2."""
    x = np.asarray(x, np.float32)
    rows, n = x.shape
    blocks = -(-n // BLOCK)
    values = table(fmt)
    bad = ~np.isfinite(x)
    v = np.where(np.abs(x) < np.float32(2.0 ** -126), np.float32(0), x).astype(np.float64)  # (subnormals: zero)
    mag = np.where(bad, 0.0, np.abs(v))
    pad = np.zeros((rows, blocks * BLOCK))
    pad[:, :n] = mag
    top = pad.reshape(rows, blocks, BLOCK).max(axis=2) if blocks else np.zeros((rows, 0))
    byte = np.zeros(top.shape, np.int64)  # the least power of two with top <= largest * 2^p
    for p in range(-127, 129):
        byte[top > values[-1] * 2.0 ** (p - 1)] = p + 127
    byte[top <= values[-1] * 2.0 ** -127] = 0
    unit = np.repeat(2.0 ** (byte - 127.0), BLOCK, axis=1)[:, :n]
    q = mag / unit  # (exact)
    mid = (values[1:] + values[:-1]) / 2
    lo, hi = np.searchsorted(mid, q, side="left"), np.searchsorted(mid, q, side="right")
    code = np.where(lo == hi, lo, np.where(lo % 2 == 0, lo, hi))  # (a tie: the even code)
    code = np.where(bad, 0x7F, code) | np.where(np.signbit(x), 0x80, 0)
    return code.astype(np.uint8), byte.astype(np.uint8)


def values(codes, byte, fmt):
    """The values of codes [rows, len] with scale bytes [rows, blocks] (NaN's aside)."""
    t = table(fmt)
    v = t[np.minimum(codes & 0x7F, len(t) - 1)] * np.where(codes & 0x80, -1.0, 1.0)
    v = np.where((codes & 0x7F) >= len(t), np.nan, v)
    return v * np.repeat(2.0 ** (byte.astype(np.float64) - 127.0), BLOCK, axis=1)[:, :codes.shape[1]]


def is_nan_code(codes, fmt):
    return (codes & 0x7F) == 0x7F if fmt == "e4m3" else (codes & 0x7F) > 0x7C


def check_tensor(t, x, fmt):
    """t (FP8Tensor) holds the conversion of x [rows, len] bit for bit, zeros behind it."""
    import torch
    rows, n = x.shape
    codes, byte = quantize(x, fmt)
    data = t.data.view(torch.uint8).cpu().numpy()
    scales = t.scales.cpu().numpy()
    blocks = -(-n // BLOCK)
    assert data.shape == (rows, blocks * BLOCK) and scales.shape == (rows, -(-blocks // 4) * 4)
    assert np.array_equal(scales[:, :blocks], byte)
    got = data[:, :n]
    nan = is_nan_code(codes, fmt)
    assert np.array_equal(is_nan_code(got, fmt), nan)
    assert np.array_equal(got[~nan], codes[~nan])
    assert not data[:, n:].any() and not scales[:, blocks:].any()
