"""GPU parity of the adapters (ppas_adapter_rows, ppas_adapter_add, ppas_adapter_act) against the 64-bit oracle.

Bound, with u = 2^-24: v = x A^T has exact products; its sum is taken by instructions of 32 features, of which a wave makes at
most H / 128 one after the other (four waves share hidden) and which round at most 4 u of the magnitudes |x| |A| each, then by
8 more additions over waves and splits: (H / 32 + 40) u sum |x| |A|. s v rounds once and is taken on with an error of 2^-17;
the second product has up to 8 instructions for either part, 64 u, and y is added: of w = sum_r |s| |v_r| |B_r| it loses
(2^-17 + 66 u) w and u of the result, which is rounded to bf16 once:
    |gpu - exact| <= 2^-8 |exact| + (2^-17 + 66 u) w + (H / 32 + 40) u sum_r |s| |B_r| sum |x| |A_r| =: 2^-8 |exact| + d.
With the activation, g and u are off by their d; silu's slope is at most 1.1 and silu(g) is within 6 u of its value:
    |gpu - exact| <= 2^-8 |exact| + 1.1 d_g |u| + (|silu(g)| + 1.1 d_g) d_u + 8 u |exact|.
2^-133 is added: half of bf16's smallest step.
"""
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


def bf16(g, shape, scale=1.0):
    """Rounded normal values: their bits and themselves in 64 bits."""
    bits = I.f32_to_bf16_bits((scale * g.standard_normal(shape)).astype(np.float32))
    return bits, R.bf16_bits_to_f64(bits)


def placed(lib, bits, pad=0, shift=0):
    """Rows on the GPU, `pad` elements apart, `shift` into a buffer of ones; the buffer and the rows."""
    ppas, step, torch = lib
    rows, cols = bits.shape
    buf = torch.full((shift + rows * (cols + pad) + 16,), -1, dtype=torch.int16, device="cuda")
    view = buf.as_strided((rows, cols), (cols + pad, 1), shift)
    view.copy_(torch.from_numpy(bits.view(np.int16)))
    return buf, view.view(torch.bfloat16)


def bounds(x, a, b, scale, rows, z):
    """w-like terms of every output, [T, N]."""
    s = np.ones(len(a)) if scale is None else np.abs(scale)
    first = A.share(np.abs(x), np.abs(a), np.abs(b), s, rows)      # sum |s| |B| sum |x| |A|
    second = np.zeros_like(first)
    for t, k in enumerate(np.asarray(rows).tolist()):
        if 0 <= k < len(a):
            second[t] = s[k] * (np.abs(b[k]) @ np.abs(a[k] @ x[t]))
    return (x.shape[1] / 32 + 40) * U * first + (2.0 ** -17 + 66 * U) * second + U * np.abs(z)


def case(lib, rows, hidden, out, rank, n, act=False, pad=0, shift=0, in_place=False, with_scale=True, seed=0, y=None, unaligned=False,
         n_real=None):
    """rows: the adapter of each row."""
    ppas, step, torch = lib
    rows = np.asarray(rows, dtype=np.int32)
    T, wide = len(rows), out * (2 if act else 1)
    g = I.rng(seed, T, hidden, out, rank)
    xb, x = bf16(g, (T, hidden))
    ab, a = bf16(g, (n, rank, hidden), hidden ** -0.5)
    bb, b = bf16(g, (n, wide, rank), rank ** -0.5)
    yb, y64 = bf16(g, (T, wide)) if y is None else y(x, a, b, rows)
    scale = (0.5 + g.random(n)).astype(np.float32) if with_scale else None
    print(f"adapters T={T} {hidden}->{out} rank={rank} n={n} act={act} pad={pad} shift={shift} in_place={in_place}", flush=True)
    off = 1 if unaligned else 0
    _, av = placed(lib, ab.reshape(1, -1), 0, off)
    _, bv = placed(lib, bb.reshape(1, -1), 0, off)
    s = ppas.adapters(av.view(n, rank, hidden), bv.view(n, wide, rank), None if scale is None else torch.from_numpy(scale).cuda())
    _, xv = placed(lib, xb, pad, shift)
    ybuf, yv = placed(lib, yb, pad, shift)
    obuf, ov = (ybuf, yv) if in_place else placed(lib, np.full((T, out), 0xffff, np.uint16), pad, shift)
    order = ppas.AdapterRows(T, n)
    order.sort(torch.from_numpy(rows).cuda())
    ws = torch.full((max(16, ppas.adapter_workspace_bytes(T, hidden, rank, n)),), 0xff, dtype=torch.uint8, device="cuda")
    (ppas.adapter_act if act else ppas.adapter_add)(s, xv, yv, ov, order, ws)
    torch.cuda.synchronize()
    got = R.bf16_bits_to_f64(step.bits_of(ov))
    z = y64 + A.share(x, a, b, scale, rows)
    d = bounds(x, a, b, scale, rows, z)
    if act:
        want = A.silu_gate(z)
        zg, zu = np.split(z, 2, 1)
        dg, du = np.split(d, 2, 1)
        tol = 2.0 ** -8 * np.abs(want) + 1.1 * dg * np.abs(zu) + (np.abs(A.silu_gate(np.concatenate((zg, np.ones_like(zg)), 1))) +
                                                                1.1 * dg) * du + 8 * U * np.abs(want)
    else:
        want, tol = z, 2.0 ** -8 * np.abs(z) + d
    err, tol = np.abs(got - want), tol + 2.0 ** -133
    print(f"  worst/tol={float((err / tol).max()) if err.size else 0:.3f}", flush=True)
    assert np.isfinite(got).all() and (err <= tol).all()
    # rows without an adapter are the projection's, bit for bit
    if not act:
        none = (rows < 0) | (rows >= n)
        assert np.array_equal(step.bits_of(ov)[none], yb[none])
    if not in_place:
        assert np.array_equal(step.bits_of(yv), yb)
    assert np.array_equal(step.bits_of(xv), xb)
    around = torch.ones(obuf.numel(), dtype=torch.bool, device="cuda")
    around.as_strided((T, out), (out + pad, 1), shift).fill_(False)
    assert bool((obuf[around] == -1).all()), "wrote outside its rows"
    return step.bits_of(ov)


def mixed(T, n, seed, loose=0.2):
    g = I.rng(seed, T, n)
    r = g.integers(0, n, T)
    r[g.random(T) < loose] = -1
    return r


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("rank", [1, 2, 7, 8, 12, 16, 17, 24, 31, 32, 33, 40, 64, 65, 96, 127, 128])
@pytest.mark.parametrize("T,n", [(37, 5), (200, 2)])
def test_ranks(lib, act, rank, T, n):
    case(lib, mixed(T, n, 1), 192, 104, rank, n, act)


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("hidden,out", [(1, 1), (8, 8), (33, 7), (64, 64), (256, 40), (257, 255), (520, 33), (1000, 513), (2048, 256),
                                        (5504, 72)])
@pytest.mark.parametrize("T,n", [(1, 1), (20, 3), (131, 2)])
def test_sizes(lib, act, hidden, out, T, n):
    case(lib, mixed(T, n, 2, 0.1), hidden, out, 16, n, act)


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("T,n,pattern", [
    (1, 1, "none"), (1, 8, "last"), (15, 1, "one"), (16, 1, "one"), (17, 1, "one"), (64, 1, "one"), (65, 1, "one"), (300, 1, "one"),
    (64, 64, "each"), (64, 1000, "each"), (100, 1024, "last"), (513, 4, "chunk"), (512, 7, "none"), (1030, 3, "turns"), (600, 9, "out")])
def test_patterns(lib, act, T, n, pattern):
    i = np.arange(T)
    rows = {"none": np.full(T, -1), "one": np.zeros(T, int), "last": np.full(T, n - 1), "each": i % n, "turns": i % n,
            "chunk": np.where(i < T // 2, 1, np.where(i % 5, 3, -1)),
            # numbers outside the set are rows without an adapter
            "out": np.where(i % 3 == 0, [n, n + 1, -5, 2 ** 31 - 1, -2 ** 31][T % 5], i % n)}[pattern]
    case(lib, rows, 320, 96, 16, n, act, with_scale=T % 2 == 0)


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("pad,shift", [(8, 8), (64, 0), (1, 0), (0, 1), (4, 4), (3, 5)])
@pytest.mark.parametrize("T,n", [(40, 6), (150, 2)])
def test_strides_and_alignment(lib, act, pad, shift, T, n):
    case(lib, mixed(T, n, 3), 128, 96, 8, n, act, pad=pad, shift=shift)
    case(lib, mixed(T, n, 4), 128, 96, 32, n, act, pad=pad, shift=shift, unaligned=True)


@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (1, 3)])
@pytest.mark.parametrize("T,n", [(70, 10), (300, 3)])
@pytest.mark.parametrize("rank", [16, 64])
def test_in_place(lib, pad, shift, T, n, rank):
    got = case(lib, mixed(T, n, 5), 256, 200, rank, n, pad=pad, shift=shift, in_place=True)
    assert np.array_equal(got, case(lib, mixed(T, n, 5), 256, 200, rank, n, pad=pad, shift=shift))


@pytest.mark.parametrize("rank", [8, 16, 64])
@pytest.mark.parametrize("T,n", [(30, 4), (200, 2)])
def test_small_differences_of_large_shares(lib, rank, T, n):
    """y is the share's negative, rounded: what is left shows the precision that the share is computed with."""
    def y(x, a, b, rows):
        bits = I.f32_to_bf16_bits((-A.share(x, a, b, None, rows)).astype(np.float32))
        return bits, R.bf16_bits_to_f64(bits)
    case(lib, mixed(T, n, 6), 512, 128, rank, n, with_scale=False, y=y)


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("T,hidden,out,rank,n", [(700, 11008, 2048, 8, 12), (2056, 2048, 1200, 32, 6), (1, 2048, 2048, 16, 8),
                                                 (64, 2048, 5504, 16, 24)])
def test_workload_sizes(lib, act, T, hidden, out, rank, n):
    rows = mixed(T, n, 7) if T < 2000 else np.concatenate((np.full(2048, 2), np.arange(8) % n))
    case(lib, rows, hidden, out, rank, n, act)


@pytest.mark.parametrize("T,n", [(1, 1), (63, 5), (64, 5), (65, 1), (511, 64), (512, 3), (513, 1024), (4099, 17), (100000, 300)])
@pytest.mark.parametrize("pattern", ["random", "runs", "none"])
def test_order(lib, T, n, pattern):
    """The list itself: every row once, by adapter and then by number, in tiles of one adapter."""
    ppas, step, torch = lib
    g = I.rng(8, T, n)
    r = {"random": g.integers(-1, n + 1, T), "runs": np.sort(g.integers(0, n, T))[::-1].copy(), "none": np.full(T, -1)}[pattern]
    o = ppas.AdapterRows(T, n)
    o.buf.fill_(0xff)
    o.sort(torch.from_numpy(r.astype(np.int32)).cuda())
    torch.cuda.synchronize()
    words = o.buf.cpu().numpy().view(np.int32)
    groups = A.order(r, n)
    k = min(n + 1, T)
    slots = [(T - k) // h + k for h in (16, 64)]
    order = words[4 + 4 * sum(slots):]
    assert len(order) == T and np.array_equal(order, np.concatenate(groups))
    for i, h in enumerate((16, 64)):
        tiles = words[4 + 4 * (slots[0] if i else 0):][:4 * words[i]].reshape(-1, 4)
        want, at = [], 0
        for a, rows in enumerate(groups):
            for c in range(0, len(rows), h):
                part = rows[c:c + h]       # and the first row, where they follow each other
                want.append((a if a < n else -1, at + c, len(part), part[0] if part[-1] - part[0] == len(part) - 1 else -1))
            at += len(rows)
        assert words[i] <= slots[i] and tiles.tolist() == [list(w) for w in want]


def test_infinities_and_nans_stay_in_their_row(lib):
    ppas, step, torch = lib
    T, H, N, r, n = 40, 128, 64, 16, 3
    g = I.rng(9)
    rows = mixed(T, n, 10)
    a, b = (torch.from_numpy(g.normal(size=s)).cuda().bfloat16() for s in ((n, r, H), (n, N, r)))
    x, y = (torch.from_numpy(g.normal(size=s)).cuda().bfloat16() for s in ((T, H), (T, N)))
    s, order = ppas.adapters(a, b), ppas.AdapterRows(T, n)
    order.sort(torch.from_numpy(rows.astype(np.int32)).cuda())
    ws = torch.empty(ppas.adapter_workspace_bytes(T, H, r, n), dtype=torch.uint8, device="cuda")
    clean, got = torch.empty_like(y), torch.empty_like(y)
    ppas.adapter_add(s, x, y, clean, order, ws)
    sick = [int(np.flatnonzero(rows == 1)[0]), int(np.flatnonzero(rows == 2)[1]), int(np.flatnonzero(rows < 0)[0])]
    x[sick[0], 5], x[sick[1], 7], x[sick[2], 9] = float("nan"), float("inf"), float("nan")
    y[sick[2], 3] = float("inf")
    ppas.adapter_add(s, x, y, got, order, ws)
    torch.cuda.synchronize()
    well = torch.ones(T, dtype=torch.bool, device="cuda")
    well[sick] = False
    assert torch.equal(got[well], clean[well])
    assert bool(got[sick[0]].isnan().all()) and not bool(got[sick[1]].isfinite().any())
    assert torch.equal(got[sick[2]].view(torch.int16), y[sick[2]].view(torch.int16))


def test_other_stream_and_replay(lib):
    """A captured step: the rows' order is made again by each replay; two graphs share a workspace, one after the other."""
    ppas, step, torch = lib
    T, H, N, r, n = 50, 256, 192, 16, 6
    t = lambda *s: torch.randn(s, device="cuda").bfloat16()                    # noqa: E731
    a, b, x, y = t(n, r, H), t(n, N, r), t(T, H), t(T, N)
    s = ppas.adapters(a, b, torch.rand(n, device="cuda"))
    ids = torch.randint(-1, n, (T,), dtype=torch.int32, device="cuda")
    orders = [ppas.AdapterRows(T, n) for _ in range(2)]
    wss = [torch.empty(ppas.adapter_workspace_bytes(T, H, r, n), dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = [torch.empty_like(y), t(T, N // 2)]
    got = [torch.empty_like(y), t(T, N // 2)]

    def step_of(i, out, stream=None):
        orders[i].sort(ids, stream=stream)
        ppas.adapter_add(s, x, y, out[0], orders[i], wss[i], stream=stream)
        ppas.adapter_act(s, x, y, out[1], orders[i], wss[i], stream=stream)

    def same(label):
        torch.cuda.synchronize()
        for w, g in zip(want, got):
            assert torch.equal(w.view(torch.int16), g.view(torch.int16)), label
    step_of(0, want)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    step_of(1, got, stream)
    same("stream")
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph, stream=stream):
            step_of(1, got)
    for k in range(4):
        x.copy_(t(T, H))
        ids.copy_(torch.randint(-1, n, (T,), dtype=torch.int32, device="cuda"))
        step_of(0, want)
        for o in got:
            o.zero_()
        graphs[k % 2].replay()
        same(k)


def test_order_of_another_call_stays_inside(lib):
    """An order that says anything: nothing outside the call's rows is written (the kernels check what it says)."""
    ppas, step, torch = lib
    T, H, N, r, n = 33, 64, 48, 8, 4
    t = lambda *s: torch.randn(s, device="cuda").bfloat16()                    # noqa: E731
    s, x, y = ppas.adapters(t(n, r, H), t(n, N, r)), t(T, H), t(T, N)
    ws = torch.zeros(ppas.adapter_workspace_bytes(T, H, r, n), dtype=torch.uint8, device="cuda")
    buf = torch.full((T + 2, N), 7.0, dtype=torch.bfloat16, device="cuda")
    o = ppas.AdapterRows(T, n)
    o.sorted = True
    g = np.random.default_rng(1)
    for k in range(4):
        words = g.integers(-2 ** 31, 2 ** 31, o.buf.numel() // 4) if k < 2 else g.integers(-3, 70, o.buf.numel() // 4)
        o.buf.copy_(torch.from_numpy(words.astype(np.int32).view(np.uint8)))
        ppas.adapter_add(s, x, y, buf[1:-1], o, ws)
        torch.cuda.synchronize()
        assert bool((buf[0] == 7).all()) and bool((buf[-1] == 7).all())


def test_binding_refusals(lib):
    ppas, step, torch = lib
    T, H, N, r, n = 8, 64, 32, 8, 2
    t = lambda *s: torch.zeros(s, device="cuda", dtype=torch.bfloat16)         # noqa: E731
    s, x, y, out = ppas.adapters(t(n, r, H), t(n, N, r)), t(T, H), t(T, N), t(T, N)
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    o = ppas.AdapterRows(T, n)
    with pytest.raises(ValueError, match="sorted"):
        ppas.adapter_add(s, x, y, out, o, ws)
    o.sort(torch.zeros(T, dtype=torch.int32, device="cuda"))
    ppas.adapter_add(s, x, y, out, o, ws)
    for args in ((x.cpu(), y, out), (x, y.cpu(), out), (x, y, out.cpu()), (x[:, ::2], y, out), (x, y[:, :16], out), (x, y, out[:7])):
        with pytest.raises(ValueError):
            ppas.adapter_add(s, *args, o, ws)
    for kw in (dict(ws=ws[:16]), dict(out=y[:, :16], act=True)):
        with pytest.raises(ppas.PPASError):
            (ppas.adapter_act if kw.get("act") else ppas.adapter_add)(s, x, y, kw.get("out", out), o, kw.get("ws", ws))
    with pytest.raises(ValueError):
        ppas.adapters(t(n, r, H).transpose(1, 2), t(n, N, H))


@pytest.mark.parametrize("T,n", [(3, 2), (70, 1)])
def test_rows_past_32_bit_offsets(lib, T, n):
    """Rows of x, y and out behind 2^32 elements of others, in tiles of 16 and of 64."""
    ppas, step, torch = lib
    H, N, r = 64, 72, 16
    stride = 2 ** 32 // (T - 1) // 8 * 8 + 64
    g = I.rng(21, T)
    rows = np.arange(T) % n
    (xb, x), (yb, y), (ab, a), (bb, b) = (bf16(g, s) for s in ((T, H), (T, N), (n, r, H), (n, N, r)))
    xv, yv = (torch.empty(stride * (T - 1) + cols, dtype=torch.int16, device="cuda").as_strided((T, cols), (stride, 1))
              for cols in (H, N))
    to = lambda bits: torch.from_numpy(bits.view(np.int16)).cuda()              # noqa: E731
    xv.copy_(to(xb))
    yv.copy_(to(yb))
    bf = torch.bfloat16
    s, order = ppas.adapters(to(ab).view(bf), to(bb).view(bf)), ppas.AdapterRows(T, n)
    order.sort(torch.from_numpy(rows.astype(np.int32)).cuda())
    ws = torch.empty(ppas.adapter_workspace_bytes(T, H, r, n), dtype=torch.uint8, device="cuda")
    out = torch.empty(T, N, dtype=bf, device="cuda")
    ppas.adapter_add(s, xv.view(bf), yv.view(bf), out, order, ws)
    z = y + A.share(x, a, b, None, rows)
    tol = 2.0 ** -8 * np.abs(z) + bounds(x, a, b, None, rows, z) + 2.0 ** -133
    assert (np.abs(R.bf16_bits_to_f64(step.bits_of(out)) - z) <= tol).all()
    ppas.adapter_add(s, xv.view(bf), yv.view(bf), yv.view(bf), order, ws)
    torch.cuda.synchronize()
    assert torch.equal(yv, out.view(torch.int16))
    assert torch.equal(xv, to(xb))
