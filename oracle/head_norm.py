"""Norms of heads, in 64 bits.

TEST INFRASTRUCTURE (see the package docstring): never called by the product path.

A head x becomes (x - mu) / sqrt(mean((x - mu)^2) + eps) * (offset + weight), mu its mean in the centred form and 0
otherwise. Written from the formula, with Python's exact sums where numbers of very different size meet.
"""
from __future__ import annotations

import math

import numpy as np


def norm(x, weight=None, eps: float = 1e-6, offset: float = 0.0, center: bool = False) -> np.ndarray:
    """x [..., D] float64; weight [D], or one of x's last two axes, or None."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    flat = x.reshape(-1, d)
    out = np.empty_like(flat)
    for i, row in enumerate(flat):
        mu = math.fsum(row) / d if center else 0.0
        row = row - mu
        out[i] = row / math.sqrt(math.fsum(row * row) / d + eps)
    out = out.reshape(x.shape)
    return out if weight is None else out * (offset + np.asarray(weight, dtype=np.float64))


def scale(x, eps: float = 1e-6, center: bool = False) -> np.ndarray:
    """1 / sqrt(var + eps) of each head, [..., 1]: what an error of its mean is multiplied by."""
    x = np.asarray(x, dtype=np.float64)
    if center:
        x = x - x.mean(-1, keepdims=True)
    return 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
