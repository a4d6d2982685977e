"""Pins of oracle/int8.py: hand-worked rows and a rational brute force."""
from fractions import Fraction

import numpy as np

import oracle.int8 as Q
from paper_2608_15171_amd import inputs as I


def bits(*v):
    return I.f32_to_bf16_bits(np.array([v], dtype=np.float32))


def test_hand_worked_rows():
    q, s = Q.quantise(bits(127.0, -127.0, 1.0, 0.0))
    assert q.tolist() == [[127, -127, 1, 0]] and s.tolist() == [1.0]
    q, s = Q.quantise(bits(254.0, 1.0, 3.0, -5.0, 127.0))      # halves go to the even integer
    assert q.tolist() == [[127, 0, 2, -2, 64]] and s.tolist() == [2.0]
    q, s = Q.quantise(bits(0.0, 0.0))
    assert q.tolist() == [[0, 0]] and s.tolist() == [0.0]
    q, s = Q.quantise(bits(1.0, np.inf))
    assert q.tolist() == [[0, 0]] and np.isnan(s).all()
    q, s = Q.quantise(bits(2.0 ** -111, 0.0))
    assert q.tolist() == [[0, 0]] and s.tolist() == [0.0]


def test_rational_brute_force():
    b = I.normal_bf16(I.rng(3, 1), (40, 33))
    q, s = Q.quantise(b)
    v = (b.astype(np.uint32) << 16).view(np.float32)
    for r in range(40):
        top = max(Fraction(float(abs(x))) for x in v[r])
        assert abs(Fraction(s[r]) * 127 / top - 1) < Fraction(1, 2 ** 51)
        for x, got in zip(v[r], q[r]):
            assert int(got) == round(Fraction(float(x)) * 127 / top)     # ties to even


def test_product_is_exact():
    g = np.random.default_rng(5)
    x, w = g.integers(-128, 128, (3, 50), dtype=np.int8), g.integers(-128, 128, (4, 50), dtype=np.int8)
    y = Q.product(x, np.array([1.0, 0.5, 2.0]), w, np.array([1.0, 4.0, -1.0, 0.0]))
    for i in range(3):
        for j in range(4):
            assert y[i, j] == sum(int(a) * int(b) for a, b in zip(x[i], w[j])) * [1, .5, 2][i] * [1, 4, -1, 0][j]
