"""8-bit integers with a scale per row, exactly.

TEST INFRASTRUCTURE (see the package docstring): never called by the product path.

A row's scale is its largest magnitude / 127, and its integers are 127 x / that magnitude to the nearest, ties to
even. bf16 values are integers times powers of two, so the quotient is a ratio of two integers and is rounded by
integer arithmetic, without any floating-point rounding. Products are int64 sums times the two scales in float64.
"""
from __future__ import annotations

import numpy as np


def _parts(bits):
    """bf16 bit patterns as integers: x = m * 2^e, m signed, e the exponent of the last place."""
    b = np.asarray(bits, dtype=np.uint16).astype(np.int64)
    e = (b >> 7) & 0xff
    m = np.where(e == 0, b & 0x7f, (b & 0x7f) | 0x80)
    return np.where(b >> 15, -m, m), np.maximum(e, 1) - 134


def quantise(bits):
    """bf16 bits [R, H] -> (int8 [R, H], scale float64 [R]); rows below 2^-110 are zero, rows with an infinity or a
    NaN have a NaN scale and zeros."""
    bits = np.asarray(bits, dtype=np.uint16)
    m, e = _parts(bits)
    mag = bits & 0x7fff
    top = mag.max(axis=1)
    q = np.zeros(bits.shape, dtype=np.int8)
    scale = np.zeros(len(bits), dtype=np.float64)
    for r in range(len(bits)):
        if top[r] >= 0x7f80:
            scale[r] = np.nan
            continue
        if top[r] < (127 - 110) << 7:
            continue
        i = int(mag[r].argmax())
        tm, te = abs(int(m[r, i])), int(e[r, i])
        scale[r] = tm * 2.0 ** te / 127.0
        # |127 m / (tm 2^(te - e))|, in halves: floor and remainder of integers; from 2^20 below the top on it is 0
        shift = np.minimum(te - e[r], 20)
        num, den = 127 * np.abs(m[r]), tm << shift
        fl, rem = num // den, num % den
        up = (2 * rem > den) | ((2 * rem == den) & (fl % 2 == 1))
        q[r] = np.sign(m[r]) * (fl + up)
    return q, scale


def product(x, sx, w, sw):
    """(x sx) (w sw)^T in float64, the integer sums exact."""
    s = np.asarray(x, dtype=np.int64) @ np.asarray(w, dtype=np.int64).T
    return s * np.asarray(sx, dtype=np.float64)[:, None] * np.asarray(sw, dtype=np.float64)
