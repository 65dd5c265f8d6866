"""The cache in 8 bits, stated in 64 bits with numpy -- TEST INFRASTRUCTURE, not part of the product.

A block of rows of one matrix has one scale s; a value is code * s.  Written from the definition: a = the largest finite
magnitude of the rows that enter the block at once; INT8: s = a / 127 rounded to fp32, codes are integers; E4M3: s = the smallest
power of two with a <= 448 s, codes are floating values of 4 significant bits, down to multiples of 2^-9.  No scale but zero is below 2^-126.
Imports nothing from the CUDA package.
"""
from __future__ import annotations

import numpy as np

INT8, E4M3 = "int8", "e4m3"


def scale(largest: float, kind: str) -> float:
    """The scale of a block whose largest finite magnitude is given."""
    if largest == 0:
        return 0.0
    if kind == INT8:
        s = float(np.float32(float(largest) / 127.0))
    else:
        s = 2.0 ** -200
        while largest > 448.0 * s:
            s *= 2.0
    return max(s, 2.0 ** -126)


def codes(x, s: float, kind: str) -> np.ndarray:
    """Codes, as the numbers they are, of values x under scale s (s = 0 counts as 1: only infinities and NaN are not zero there)."""
    x = np.asarray(x, dtype=np.float64)
    most = 127.0 if kind == INT8 else 448.0
    with np.errstate(all="ignore"):
        t = np.clip(x / (s if s > 0 else 1.0), -most, most)
        if kind == INT8:
            return np.rint(np.nan_to_num(t, nan=0.0))
        mag = np.abs(t)
        exponent = np.floor(np.log2(np.where(mag >= 2.0 ** -6, mag, 2.0 ** -6)))
        step = 2.0 ** (exponent - 3)
        return np.clip(np.rint(t / step) * step, -most, most)


def append(matrix_codes, scales, rows, length: int, kind: str, block: int):
    """Rows enter behind the first `length` rows of one matrix: (codes [capacity, d], scales [blocks]) afterwards, copies."""
    c, s = np.array(matrix_codes, dtype=np.float64), np.array(scales, dtype=np.float64)
    rows = np.asarray(rows, dtype=np.float64)
    end = length + len(rows)
    for i in range(length // block, -(-end // block)):
        lo, hi = max(length, i * block), min(end, (i + 1) * block)
        new = rows[lo - length:hi - length]
        finite = np.abs(new[np.isfinite(new)])
        want = scale(float(finite.max()) if finite.size else 0.0, kind)
        if lo > i * block:                      # rows that are there already
            had = s[i]
            s[i] = max(had, want)
            if s[i] > had:
                c[i * block:lo] = codes(c[i * block:lo] * had, s[i], kind)
        else:
            s[i] = want
        c[lo:hi] = codes(new, s[i], kind)
    return c, s


def values(matrix_codes, scales, block: int) -> np.ndarray:
    """code * scale of every row."""
    c = np.asarray(matrix_codes, dtype=np.float64)
    return c * np.repeat(np.asarray(scales, dtype=np.float64), block)[: len(c), None]
