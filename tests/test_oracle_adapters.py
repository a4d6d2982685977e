"""Pins of the 64-bit adapters."""
import numpy as np

import oracle.adapters as A


def test_share():
    g = np.random.default_rng(1)
    x, a, b, s = g.normal(size=(5, 7)), g.normal(size=(3, 2, 7)), g.normal(size=(3, 4, 2)), g.normal(size=3)
    rows = [2, -1, 0, 2, 9]
    got = A.share(x, a, b, s, rows)
    for t, k in enumerate(rows):
        want = s[k] * np.einsum("nr,rh,h->n", b[k], a[k], x[t]) if 0 <= k < 3 else np.zeros(4)
        np.testing.assert_allclose(got[t], want, rtol=1e-13)
    np.testing.assert_allclose(A.share(x, a, b, None, rows)[0] * s[2], got[0], rtol=1e-13)
    # an adapter is the low-rank matrix that it stands for, added to the projection's
    np.testing.assert_allclose(x[0] @ (s[2] * b[2] @ a[2]).T, got[0], rtol=1e-12)


def test_silu_gate():
    np.testing.assert_allclose(A.silu_gate([[0.0, 1.0, 3.0, 2.0]]), [[0.0, 2.0 / (1.0 + np.exp(-1.0))]], rtol=1e-15)
    assert A.silu_gate([[-1e4, 5.0]])[0, 0] == 0.0


def test_order():
    got = A.order([3, 0, -1, 3, 1, 7], 4)
    assert [r.tolist() for r in got] == [[1], [4], [], [0, 3], [2, 5]]
