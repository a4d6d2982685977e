"""Low-rank adapters beside a projection, in 64 bits.

TEST INFRASTRUCTURE (see the package docstring): never called by the product path.

Row t with adapter a becomes y[t] + s_a (x[t] A_a^T) B_a^T, a row without one stays y[t]; with the activation the halves
g and u of that become g / (1 + e^-g) * u. Row by row, from the formula.
"""
from __future__ import annotations

import numpy as np


def share(x, a, b, scale, row_adapter) -> np.ndarray:
    """The adapters' part alone: x [T, H], a [n, r, H], b [n, N, r], scale [n] or None, row_adapter [T]."""
    out = np.zeros((x.shape[0], b.shape[1]))
    for t, k in enumerate(np.asarray(row_adapter).tolist()):
        if 0 <= k < a.shape[0]:
            out[t] = (1.0 if scale is None else scale[k]) * (b[k] @ (a[k] @ x[t]))
    return out


def silu_gate(z) -> np.ndarray:
    g, u = np.split(np.asarray(z, dtype=np.float64), 2, axis=1)
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-g)) * u


def order(row_adapter, n: int):
    """The rows of each adapter, ascending, and at the end those of none."""
    row_adapter = np.asarray(row_adapter)
    groups = [np.flatnonzero(row_adapter == a) for a in range(n)]
    return groups + [np.flatnonzero((row_adapter < 0) | (row_adapter >= n))]
