"""Floating point of 4 bits in numpy, 64 bits, from the definitions: e2m1 codes, e8m0 and e4m3 block scales, matrices and a
cache quantised and read back.  Every value, scale and border is a double exactly, so every decision is that of exact arithmetic
(but for the quotient m / 6, whose 53 bits lie on the right side of every border of e4m3)."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# e4m3: 1 sign bit, 4 exponent bits (bias 7), 3 mantissa bits; byte 127 is NaN, 126 is 448
E4M3 = np.array([(b & 7) * 2.0 ** -9 if b < 8 else (8 + (b & 7)) * 2.0 ** ((b >> 3) - 10) for b in range(127)])


def nearest(x, table):
    """Index of the nearest entry of an ascending table for x >= 0; the even index at a tie, the last one beyond the end."""
    x = np.asarray(x, np.float64)
    mid = (table[1:] + table[:-1]) / 2
    i = np.searchsorted(mid, x, side="left")   # a tie stays below
    tie = (i < len(mid)) & (x == mid[np.minimum(i, len(mid) - 1)])
    return np.where(tie & (i % 2 == 1), i + 1, i)


def codes_of(x, unit):
    """e2m1 codes of x in units of `unit` (0: code 0)."""
    x, unit = np.broadcast_arrays(np.asarray(x, np.float64), np.asarray(unit, np.float64))
    with np.errstate(all="ignore"):
        idx = np.zeros(x.shape, np.int64)
        for i in range(7):  # borders times the unit are exact, a quotient would not be
            border = (GRID[i] + GRID[i + 1]) / 2 * unit
            idx += (np.abs(x) >= border) if i % 2 else (np.abs(x) > border)
    return np.where(unit > 0, idx + 8 * ((x < 0) & (idx > 0)), 0).astype(np.uint8)


def values_of(codes):
    return np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]


def quantise(x, block):
    """x [rows, k] -> (codes [rows, k], scale bytes [rows, k / block], row_scale [rows])."""
    x = np.asarray(x, np.float64)
    b = x.reshape(len(x), -1, block)
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(b).all(-1)
    top = np.where(bad, 0.0, top)
    row = np.ones(len(x))
    if block == 32:
        e = np.where(top > 0, np.floor(np.log2(np.where(top > 0, top, 1.0))), -127.0).astype(int)
        e = np.where(np.ldexp(1.0, e) > top, e - 1, np.where(np.ldexp(1.0, e + 1) <= top, e + 1, e))
        e = np.where(top > 0, np.maximum(e - 2, -127), -127)
        scale, unit = (e + 127).astype(np.uint8), np.where(top > 0, np.ldexp(1.0, e), 0.0)
        scale = np.where(bad, 255, scale).astype(np.uint8)
    else:
        for r, m in enumerate(top.max(-1)):
            if m > 0:
                p = -126
                while m > 2688 * 2.0 ** p:
                    p += 1
                row[r] = 2.0 ** p
        scale = nearest(top / row[:, None] / 6, E4M3).astype(np.uint8)
        unit = E4M3[scale] * row[:, None]
        scale = np.where(bad, 127, scale).astype(np.uint8)
    codes = codes_of(np.where(bad[..., None], 0.0, b), unit[..., None])
    return codes.reshape(x.shape), scale, row


def dequantise(codes, scale, row, block):
    """The values of codes [rows, k]."""
    if block == 32:
        unit = np.where(scale == 255, np.nan, np.ldexp(1.0, np.minimum(scale.astype(int), 254) - 127))
    else:
        unit = np.where(scale == 127, np.nan, E4M3[np.minimum(scale & 127, 126)]) * np.asarray(row, np.float64)[:, None]
    v = values_of(codes).reshape(len(codes), -1, block) * unit[..., None]
    return v.reshape(codes.shape)


def cache_quantise(x, exponent):
    """x [..., dim] by blocks of 16 under 2^exponent: (codes [..., dim], scale bytes [..., dim / 16])."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, 16)
    bad = ~np.isfinite(b).all(-1)
    top = np.where(bad, 0.0, np.abs(b).max(-1))
    scale = nearest(np.minimum(top / 2.0 ** exponent / 6, 448.0), E4M3).astype(np.uint8)
    codes = codes_of(np.where(bad[..., None], 0.0, b), (E4M3[scale] * 2.0 ** exponent)[..., None])
    return codes.reshape(x.shape), np.where(bad, 127, scale).astype(np.uint8)


def cache_values(codes, scale, exponent):
    unit = np.where(scale == 127, np.nan, E4M3[np.minimum(scale & 127, 126)]) * 2.0 ** exponent
    return (values_of(codes).reshape(*codes.shape[:-1], -1, 16) * unit[..., None]).reshape(codes.shape)


def pack(codes):
    """Two codes a byte, the even column in the low half."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(packed):
    return np.stack([packed & 15, packed >> 4], -1).reshape(*packed.shape[:-1], -1)


def linear(xq, wq, bias=None):
    """(X W^T + bias, sum |x w|) of values in 64 bits."""
    y = xq @ wq.T
    return (y if bias is None else y + np.asarray(bias, np.float64)), np.abs(xq) @ np.abs(wq).T
