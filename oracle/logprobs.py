"""Log probabilities of logit rows, in 64 bits.

TEST INFRASTRUCTURE (see the package docstring): never called by the product path.

For logits x of a row and l = scale x: log p_i = l_i - ln sum e^l, the entropy -sum p ln p, and the order of tokens by
larger logit, then lower number, in which a token's rank is its place. Rows without a distribution (a NaN, +infinity, or
nothing but -infinity) give NaN and -1, tokens that are masked (-infinity) are listed nowhere and have no rank.
"""
from __future__ import annotations

import math

import numpy as np


def row(x, scale: float = 1.0, token: int = -1, top: int = 0) -> dict:
    """x: the row's logits (float64). Everything that is asked of one row."""
    x = np.asarray(x, dtype=np.float64)
    out = {"logprob": math.nan, "rank": -1, "entropy": math.nan, "top_ids": [-1] * top, "top_logprobs": [math.nan] * top}
    live = np.flatnonzero(x != -np.inf)
    if len(live) == 0 or not np.isfinite(x[live]).all():
        return out
    with np.errstate(over="ignore"):
        l = (x - x[live].max()) * scale       # the largest is 0
    p = np.exp(l)
    total = math.fsum(p)
    lse = math.log(total)
    out["entropy"] = max(0.0, lse - math.fsum(p[live] * np.where(p[live] > 0, l[live], 0.0)) / total)
    order = live[np.lexsort((live, -x[live]))]
    if 0 <= token < len(x):
        out["logprob"] = l[token] - lse
        if x[token] != -np.inf:
            out["rank"] = int(np.flatnonzero(order == token)[0])
    n = min(top, len(order))
    out["top_ids"] = [int(i) for i in order[:n]] + [-1] * (top - n)
    out["top_logprobs"] = [l[i] - lse for i in order[:n]] + [-math.inf] * (top - n)
    return out
