"""The centred norm of heads whose features are nearly, or quite, equal: what is left of them is their difference from the
mean, so that the mean's own rounding shows.

Features within a factor of two of each other are whole multiples of one bf16 step, of up to 2^8 of them each, so that
the sum of 256 has 17 bits: exact in fp32, in any order. The mean is the sum over D, kept as a division's result and its
remainder, and a feature's difference from the first is exact (Sterbenz); taking the remainder away rounds once, by u = 2^-24
of the difference, the remainder itself by less than 2^-46 of the mean. What the mean of squares, the root and the weight
add to a difference is at most 20 u of the result, and of the turn 1e-6 m (|a| + |b|) for a pair:
    |gpu - exact| <= 2^-8 |exact| + sum over the pair 2.5e-6 |z|  (+ 2^-46 s |g| |x|)  + 2^-133.
"""
import numpy as np
import pytest

import oracle.head_norm as N
import oracle.rope as R
import oracle.rope_forms as F
from paper_2608_15171_amd import inputs as I

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas, step
    return ppas, step, torch


def run(lib, x, w, layout, rotary, eps):
    """x: bits [rows, heads, D], w: bits [D] or None."""
    ppas, step, torch = lib
    dev = lambda b: torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).cuda().view(torch.bfloat16)   # noqa: E731
    norm = ppas.head_norm(None if w is None else dev(w), eps, 0.0, True)
    y = torch.full(x.shape, -1, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    pos = torch.arange(len(x), dtype=torch.int32, device="cuda") * 17
    ppas.norm_rope_rows(norm, ppas.rope(layout, rotary), dev(x), pos, y)
    torch.cuda.synchronize()
    return R.bf16_bits_to_f64(step.bits_of(y)), pos.cpu().numpy()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("eps", [1e-6, 2.0 ** -100])
def test_equal_features_have_no_variance(lib, layout, eps):
    """Every even size; values of every magnitude, among them those whose sums and squares pass fp32."""
    g = I.rng(31)
    values = np.concatenate(([0x44e0, 0x4660, 0x7f7f, 0xff7f, 0x7200, 0x0001, 0x0080], g.integers(0, 0x7f80, 250))).astype(np.uint16)
    values[20::2] |= 0x8000
    for dim in range(2, 257, 2):
        x = np.repeat(values[:, None, None], dim, 2)
        got, _ = run(lib, x, None, layout, dim if dim % 16 else dim // 2, eps)
        bad = (got != 0).any(axis=(1, 2))
        assert not bad.any(), (dim, [hex(v) for v in values[bad][:5]], np.abs(got[bad]).max())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rotary", [(14, 14), (56, 48), (112, 112), (120, 64), (126, 100), (128, 128), (224, 192), (252, 252)])
@pytest.mark.parametrize("size", [0x3f80, 0x4600, 0x7200])
def test_small_differences_of_large_features(lib, layout, dim, rotary, size):
    """Features some bf16 steps apart, in one head a single one that differs."""
    g = I.rng(32, dim, size)
    x = (size + g.integers(0, 4, (12, 3, dim))).astype(np.uint16)
    x[0] = size + 64
    x[0, :, 3] += 1
    x[1] = size + 127
    x[1, :, dim - 1] -= 1
    w = R.f64_to_bf16_bits(1.0 + 0.2 * g.normal(size=dim))
    eps = 2.0 ** -100
    got, pos = run(lib, x, w, layout, rotary, eps)
    x64, w64 = R.bf16_bits_to_f64(x), R.bf16_bits_to_f64(w)
    z = N.norm(x64, w64, eps, 0.0, True)
    exact = F.turn(z, pos, layout, rotary, 1e6, 1.0, False)
    part = 2.5e-6 * np.abs(z) + 2.0 ** -46 * N.scale(x64, eps, True) * np.abs(w64) * np.abs(x64)
    a, b = F.pairs_of(layout, rotary)
    both = part[..., a] + part[..., b]
    part[..., a], part[..., b] = both, both
    tol = 2.0 ** -8 * np.abs(exact) + part + 2.0 ** -133
    err = np.abs(got - exact)
    print(f"mean {layout} dim={dim} size={size:#x}: worst/tol={float((err / tol).max()):.3f}", flush=True)
    assert (err <= tol).all()
