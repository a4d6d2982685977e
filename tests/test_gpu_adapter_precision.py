"""What the adapters' results keep beyond bf16, on inputs whose exact values are known to the last bit. u = 2^-24."""
import numpy as np
import pytest

import oracle.adapters as A
import oracle.rope as R
from paper_2608_15171_amd import inputs as I

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas, step
    return ppas, step, torch


def run(lib, x, a, b, scale, y, rows, out, act):
    """Bit patterns in (x, a, b, y), the result in 64 bits out."""
    ppas, step, torch = lib
    dev = lambda bits: torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)   # noqa: E731
    n, rank, hidden = a.shape
    T = len(rows)
    s = ppas.adapters(dev(a), dev(b), torch.from_numpy(scale).cuda())
    order = ppas.AdapterRows(T, n)
    order.sort(torch.from_numpy(np.asarray(rows, np.int32)).cuda())
    ws = torch.empty(max(16, ppas.adapter_workspace_bytes(T, hidden, rank, n)), dtype=torch.uint8, device="cuda")
    got = torch.empty(T, out, dtype=torch.bfloat16, device="cuda")
    (ppas.adapter_act if act else ppas.adapter_add)(s, dev(x), dev(y), got, order, ws)
    torch.cuda.synchronize()
    return R.bf16_bits_to_f64(step.bits_of(got))


def bits(x):
    return I.f32_to_bf16_bits(np.asarray(x, dtype=np.float32))


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("rank", [2, 16, 17, 40, 64, 128])
@pytest.mark.parametrize("T,n", [(96, 12), (256, 4)])
def test_the_share_keeps_fp32(lib, act, rank, T, n):
    """Row t takes one number f = s a, fp32, through two ranks: B's columns are 1 and a small b, and y is f's rounding to
    bf16, negative, so that f - bf16(f) + f b is left. Some column's b takes nearly all of f's next eight bits away: what
    is left then is at the place of f's last ones. Only the three products of f with 1 round visibly, by at most 4 u |f| each,
    and those with b, y's sum and the oracle's f b by another 4 u |f|:
        |gpu - exact| <= 2^-8 |exact| + 16 u |f|,
    where f without its last eight bits is off by up to 64 u |f|. With the activation, silu(16) (taken within 8 u) is a
    factor of it."""
    H, N = 64, 256
    g = I.rng(1, T, rank)
    rows = np.arange(T) % n
    x = np.zeros((T, H))
    at = (np.arange(T) * 7) % H
    x[np.arange(T), at] = 1.0
    a = np.zeros((n, rank, H), np.uint16)
    a[:, 0] = a[:, 1] = bits(0.5 + g.random((n, H)))
    scale = (0.5 + g.random(n)).astype(np.float32)
    f = scale[rows] * R.bf16_bits_to_f64(a[rows, 0, at]).astype(np.float32)    # one rounding, the kernel's own
    assert f.dtype == np.float32
    small = bits((np.arange(N) - N // 2) * 2.0 ** -16)
    b = np.zeros((n, N, rank), np.uint16)
    b[:, :, 0], b[:, :, 1] = bits(1.0), small
    top = R.bf16_bits_to_f64(bits(f))
    y = np.repeat(bits(-top)[:, None], N, 1)
    exact = (f.astype(np.float64) - top)[:, None] + f.astype(np.float64)[:, None] * R.bf16_bits_to_f64(small)
    tol = 2.0 ** -8 * np.abs(exact) + 16 * U * np.abs(f)[:, None]
    if act:
        y = np.concatenate((np.full((T, N), bits(16.0)), y), 1)
        b = np.concatenate((np.zeros_like(b), b), 1)
        factor = float(A.silu_gate(np.array([[16.0, 1.0]]))[0, 0])
        exact = exact * factor
        tol = tol * factor + 9 * U * np.abs(exact)
    print(f"share in fp32: T={T} n={n} rank={rank} act={act}", flush=True)
    got = run(lib, bits(x), a, b, scale, y, rows, N, act)
    err = np.abs(got - exact)
    print(f"  worst/tol={float((err / tol).max()):.3f}", flush=True)
    assert (err <= tol).all()


@pytest.mark.parametrize("T", [16, 80])
def test_the_activation_of_every_gate(lib, T):
    """Rows without an adapter: g and u are y's, exact. silu(g) is within 7 u of its value (its exponent's rounding 1 u of
    the result, the exponential 2 u, 1 + t 1 u, the reciprocal 2 u and the last product 1 u), the product with u rounds once
    more, and then bf16's grid decides: a result is off by half of its step at most, and by 8 u of the value beside that.
    Below 2^-126 fp32's own grid adds to it: e^-|g| is off by up to 2^-150, which |g| < 2^7 and u < 2 bring to 2^-142, and
    two products' roundings are 2^-150 times u and 2^-150."""
    gate = np.arange(0x10000, dtype=np.uint16)
    gate = gate[(gate & 0x7fff) < 0x7f80]                                      # every finite one
    N = len(gate)
    u = (0x3f80 + np.arange(T) * (128 // 16) % 128 + np.arange(T) // 16).astype(np.uint16)   # in [1, 2): many roundings of each
    y = np.concatenate((np.tile(gate, (T, 1)), np.repeat(u[:, None], N, 1)), 1)
    z = np.zeros
    print(f"every gate: T={T}", flush=True)
    got = run(lib, z((T, 8), np.uint16), z((1, 8, 8), np.uint16), z((1, 2 * N, 8), np.uint16), np.ones(1, np.float32), y,
              np.full(T, -1), N, True)
    exact = A.silu_gate(R.bf16_bits_to_f64(y))
    assert np.isfinite(exact).all()
    big = np.abs(exact) >= 2.0 ** 128 * (1 - 2.0 ** -9)                        # rounds to an infinity
    assert (np.abs(got[big]) == np.inf).all() and (np.sign(got[big]) == np.sign(exact[big])).all()
    step = 2.0 ** (np.maximum(np.frexp(exact)[1] - 1, -126) - 7)               # between bf16 numbers at that size
    lim = step / 2 + 8 * U * np.abs(exact) + 2.0 ** -141
    err = np.where(big, 0.0, np.abs(np.where(big, 0.0, got) - np.where(big, 0.0, exact)))
    print(f"  beyond half a step, in u of the value: {float(((err - step / 2) / (U * np.abs(exact) + 2.0 ** -144)).max()):.2f}", flush=True)
    assert (err <= lim).all(), int((err > lim).sum())
