"""The 4-bit store of keys and values, float64.

Every 32 elements of a head share a power of two: the smallest s with
max |x| <= 7 s, kept in [2^-123, 2^125] and stored as the byte log2(s) + 127;
each element becomes the nearest of +-{0, .5, 1, 1.5, 2, 3, 4, 6} * s, ties to
the even code (the position in that list), at most 6 s.  A group that holds a
NaN or an infinity gets the byte 255 and zero codes, and reads as NaN.  Element
2i is the low half of byte i of a row, element 2i + 1 the high half.

Test infrastructure only; shares no code with the HIP path.
"""
from __future__ import annotations

import math

import numpy as np

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def group_exponent(amax: float) -> int:
    """log2 of the scale of a group whose largest magnitude is amax."""
    e = -123
    while e < 125 and amax > 7.0 * math.ldexp(1.0, e):
        e += 1
    return e


def nearest_code(x: float, s: float) -> int:
    """Code of x at scale s: nearest grid point, ties to the even position, the sign in bit 3."""
    a = abs(x) / s
    best = min(range(8), key=lambda c: (abs(min(a, 6.0) - GRID[c]), c % 2))
    return best | (8 if math.copysign(1.0, x) < 0 else 0)


def encode(x: np.ndarray):
    """x [n, heads, d] float64 -> (codes uint8 [n, heads, d/2], scales uint8 [n, heads, d/32])."""
    n, h, d = x.shape
    codes = np.zeros((n, h, d // 2), dtype=np.uint8)
    scales = np.zeros((n, h, d // 32), dtype=np.uint8)
    for i in range(n):
        for k in range(h):
            for g in range(d // 32):
                v = x[i, k, 32 * g:32 * g + 32]
                if not np.all(np.isfinite(v)):
                    scales[i, k, g] = 255
                    continue
                e = group_exponent(float(np.max(np.abs(v))))
                scales[i, k, g] = e + 127
                c = [nearest_code(float(y), math.ldexp(1.0, e)) for y in v]
                codes[i, k, 16 * g:16 * g + 16] = [c[2 * m] | c[2 * m + 1] << 4 for m in range(16)]
    return codes, scales


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The values that codes and scales stand for, float64 [n, heads, d]."""
    n, h, half = codes.shape
    c = np.zeros((n, h, 2 * half), dtype=np.int64)
    c[..., 0::2], c[..., 1::2] = codes & 15, codes >> 4
    v = np.array(GRID)[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return v * np.repeat(s, 32, axis=-1)
