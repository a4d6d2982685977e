"""Pins of oracle/rope_forms.py: closed forms of the frequencies, and the turn against the rotate-half oracle."""
import math

import numpy as np
import pytest

import oracle.rope as R
import oracle.rope_forms as F

W = dict(theta=1e6, rotary_dim=128)


def test_plain_form_is_the_rotate_half_oracle():
    g = np.random.default_rng(0)
    x, pos = g.standard_normal((5, 3, 128)), np.array([0, 1, 7, 4096, 99999])
    np.testing.assert_allclose(F.turn(x, pos, "half", 128, 1e6), R.rotate(x, pos, 1e6), atol=1e-9)


def test_interleaved_is_a_permutation_of_half():
    g = np.random.default_rng(1)
    x, pos = g.standard_normal((4, 2, 96)), np.array([3, 5, 1000, 12])
    a, b = F.pairs_of("interleaved", 64)
    order = np.concatenate([a, b, np.arange(64, 96)])
    y = F.turn(x, pos, "interleaved", 64, 1e4)
    np.testing.assert_allclose(y[..., order], F.turn(x[..., order], pos, "half", 64, 1e4), atol=1e-12)
    assert np.array_equal(y[..., 64:], x[..., 64:])


def test_transposed_inverts_and_magnitude_scales():
    g = np.random.default_rng(2)
    x, pos = g.standard_normal((3, 2, 128)), np.array([11, -5, 800])
    y = F.turn(x, pos, "half", 128, 1e6, magnitude=1.5)
    np.testing.assert_allclose(F.turn(y, pos, "half", 128, 1e6, magnitude=1 / 1.5, transposed=True), x, atol=1e-12)
    np.testing.assert_allclose(np.linalg.norm(y, axis=-1), 1.5 * np.linalg.norm(x, axis=-1))


def test_scaled_frequencies_closed_forms():
    base = [F.frequency(j, **W) for j in range(64)]
    assert base[0] == 1.0 and math.isclose(base[32], 1e-3) and math.isclose(base[63], 1e6 ** (-126 / 128))
    assert all(math.isclose(F.frequency(j, scaling="linear", factor=4.0, **W) * 4, base[j]) for j in range(64))
    big = [F.frequency(j, scaling="base", factor=4.0, **W) for j in range(64)]
    assert big[0] == 1.0 and math.isclose(big[63] * 4, base[63])
    assert all(math.isclose(big[j], (1e6 * 4 ** (128 / 126)) ** (-2 * j / 128)) for j in range(64))
    kw = dict(factor=8.0, original_len=8192, low=1.0, high=4.0)
    bands = [F.frequency(j, scaling="bands", **kw, **W) for j in range(64)]
    for j, (w, b) in enumerate(zip(base, bands)):
        turns = 8192 * w / (2 * math.pi)
        want = b if 1 < turns < 4 else w if turns >= 4 else w / 8
        assert math.isclose(b, want) and w / 8 <= b <= w, j
    # the pair of 2.5 turns of a made-up theta is half way between the ends
    th = (8192 / (2 * math.pi * 2.5)) ** 2
    w = F.frequency(1, rotary_dim=4, theta=th)
    assert math.isclose(F.frequency(1, rotary_dim=4, theta=th, scaling="bands", **kw), (w + w / 8) / 2)
    ramp = [F.frequency(j, scaling="ramp", factor=4.0, original_len=8192, low=1.0, high=32.0, **W) for j in range(64)]
    first, last = 17, 34       # 128 ln(8192 / (2 pi b)) / (2 ln 1e6): 17.17 for 32 turns, 33.23 for one
    assert ramp[:first + 1] == base[:first + 1] and all(math.isclose(4 * r, w) for r, w in zip(ramp[last:], base[last:]))
    assert math.isclose(ramp[25], base[25] * (1 - 8 / 17 * 0.75))


@pytest.mark.parametrize("scaling", ["linear", "base", "bands", "ramp"])
def test_factor_one_changes_nothing(scaling):
    for j in range(64):
        assert math.isclose(F.frequency(j, scaling=scaling, factor=1.0, original_len=4096, low=1.0, high=32.0, **W),
                            F.frequency(j, **W))
