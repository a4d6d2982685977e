"""Rotary positions in their general form, in 64 bits.

TEST INFRASTRUCTURE (see the package docstring): never called by the product path.

A head's pair j turns by p * w_j and is multiplied by a magnitude; which features make a pair depends on the layout,
and w_j on the scaling for long contexts. Written as complex products, frequency by frequency, from the formulas:

  none    theta^(-2j/R)
  linear  that / factor
  base    with theta replaced by theta * factor^(R/(R-2)), so that the last pair ends at 1/factor of its frequency
  bands   by wavelength: short waves (at least `high` turns over the original length) keep their frequency, long ones
          (at most `low` turns) get it / factor, and between them it is interpolated by the number of turns
  ramp    by pair number, between the pairs that make `high` and `low` turns over the original length
"""
from __future__ import annotations

import math

import numpy as np


def frequency(j: int, rotary_dim: int, theta: float, scaling: str = "none", factor: float = 1.0,
              original_len: int = 0, low: float = 0.0, high: float = 0.0) -> float:
    R = rotary_dim
    w = math.exp(-(2.0 * j / R) * math.log(theta))
    if scaling == "linear":
        return w / factor
    if scaling == "base":
        # the factor enters as factor^(-2j/(R-2)): 1 for the first pair, 1/factor for the last
        return w if R == 2 else w * math.exp(-2.0 * j / (R - 2) * math.log(factor))
    if scaling == "bands":
        wavelength = 2.0 * math.pi / w
        if wavelength <= original_len / high:
            return w
        if wavelength >= original_len / low:
            return w / factor
        s = (original_len / wavelength - low) / (high - low)
        return s * w + (1.0 - s) * w / factor
    if scaling == "ramp":
        def pair(turns):
            return R * math.log(original_len / (turns * 2.0 * math.pi)) / (2.0 * math.log(theta))
        first, last = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), R - 1)
        if j <= first:
            return w
        if j >= last:
            return w / factor
        t = (j - first) / (last - first)
        return (1.0 - t) * w + t * w / factor
    assert scaling == "none", scaling
    return w


def pairs_of(layout: str, rotary_dim: int):
    """Index arrays of the two features of every pair."""
    j = np.arange(rotary_dim // 2)
    return (j, j + rotary_dim // 2) if layout == "half" else (2 * j, 2 * j + 1)


def turn(x, positions, layout: str, rotary_dim: int, theta: float, magnitude: float = 1.0, transposed: bool = False,
         **scaling) -> np.ndarray:
    """x [rows, heads, D] float64 turned by the rows' positions; features from rotary_dim on as they are."""
    y = np.array(x, dtype=np.float64)
    a, b = pairs_of(layout, rotary_dim)
    w = np.array([frequency(j, rotary_dim, theta, **scaling) for j in range(rotary_dim // 2)])
    ang = np.asarray(positions, dtype=np.float64)[:, None, None] * w
    z = (y[..., a] + 1j * y[..., b]) * np.exp(1j * (-ang if transposed else ang)) * magnitude
    y[..., a], y[..., b] = z.real, z.imag
    return y
