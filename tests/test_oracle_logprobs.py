"""Pins of the 64-bit log probabilities: closed forms, ties, masks."""
import math

import numpy as np
import pytest

import oracle.logprobs as L


def test_closed_forms():
    r = L.row(np.log([1.0, 2.0, 5.0]), token=1, top=3)
    assert math.isclose(r["logprob"], math.log(0.25), rel_tol=1e-14) and r["rank"] == 1
    assert math.isclose(r["entropy"], -(math.log(1 / 8) / 8 + math.log(1 / 4) / 4 + 5 * math.log(5 / 8) / 8), rel_tol=1e-14)
    assert r["top_ids"] == [2, 1, 0]
    np.testing.assert_allclose(r["top_logprobs"], np.log([5 / 8, 1 / 4, 1 / 8]), rtol=1e-14)
    u = L.row(np.full(1000, -3.0), token=17, top=2)
    assert math.isclose(u["entropy"], math.log(1000), rel_tol=1e-14) and u["rank"] == 17 and u["top_ids"] == [0, 1]


def test_scale_and_shift():
    x = np.random.default_rng(1).normal(size=50)
    a, b = L.row(3.0 * x + 7.0, 1.0, 5, 4), L.row(x, 3.0, 5, 4)
    np.testing.assert_allclose([a["logprob"], a["entropy"], *a["top_logprobs"]], [b["logprob"], b["entropy"], *b["top_logprobs"]],
                               rtol=1e-12)
    assert a["top_ids"] == b["top_ids"] and a["rank"] == b["rank"]


def test_masks():
    x = np.array([-np.inf, 1.0, -np.inf, 1.0])
    r = L.row(x, token=0, top=3)
    assert r["logprob"] == -np.inf and r["rank"] == -1 and r["top_ids"] == [1, 3, -1] and r["top_logprobs"][2] == -np.inf
    assert math.isclose(r["entropy"], math.log(2))
    assert L.row(x, token=3)["rank"] == 1 and L.row([5.0])["entropy"] == 0.0


@pytest.mark.parametrize("bad", [[-np.inf] * 3, [1.0, np.nan, 0.0], [1.0, np.inf, -np.inf]])
def test_no_distribution(bad):
    r = L.row(bad, token=0, top=2)
    assert math.isnan(r["logprob"]) and math.isnan(r["entropy"]) and r["rank"] == -1 and r["top_ids"] == [-1, -1]
