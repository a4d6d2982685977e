"""Pins of the 64-bit norm of heads: closed forms and invariants."""
import numpy as np
import pytest

import oracle.head_norm as N


def test_closed_forms():
    np.testing.assert_allclose(N.norm([3.0, -3.0, 3.0, 3.0], eps=0.0), [1, -1, 1, 1], rtol=1e-15)
    np.testing.assert_allclose(N.norm([1.0, 3.0], eps=0.0, center=True), [-1, 1], rtol=1e-15)
    np.testing.assert_allclose(N.norm([3.0, 4.0], [1.0, 2.0], eps=3.5, offset=1.0), [1.5, 3.0], rtol=1e-15)   # sqrt(12.5 + 3.5) = 4
    assert np.array_equal(N.norm(np.zeros((2, 4)), eps=1e-6), np.zeros((2, 4)))
    assert np.array_equal(N.norm(np.full((2, 4), 7.0), center=True), np.zeros((2, 4)))


@pytest.mark.parametrize("center", [False, True])
def test_invariants(center):
    x = np.random.default_rng(1).normal(size=(5, 3, 48))
    z = N.norm(x, eps=0.0, center=center)
    np.testing.assert_allclose((z * z).mean(-1), 1.0, rtol=1e-13)
    np.testing.assert_allclose(N.norm(1e150 * x, eps=0.0, center=center), z, rtol=1e-11, atol=1e-14)
    np.testing.assert_allclose(x * N.scale(x, 0.0) if not center else (x - x.mean(-1, keepdims=True)) * N.scale(x, 0.0, True), z,
                               rtol=1e-12, atol=1e-14)
    if center:
        np.testing.assert_allclose(N.norm(x + 5.0, eps=0.0, center=True), z, rtol=1e-10, atol=1e-12)
        assert np.abs(z.mean(-1)).max() < 1e-14


def test_weights_by_head():
    x, w = np.random.default_rng(2).normal(size=(4, 3, 16)), np.random.default_rng(3).normal(size=(3, 16))
    z = N.norm(x, w, offset=1.0)
    for h in range(3):
        np.testing.assert_array_equal(z[:, h], N.norm(x[:, h], w[h], offset=1.0))
