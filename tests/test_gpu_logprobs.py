"""GPU parity of ppas_logprobs against the 64-bit oracle: ids and ranks equal, the rest within the bound below.

In units of u = 2^-24, for a row whose unmasked l = scale x spread over D and a lane that holds n vectors: t = x c - r is one
rounding of |t| (in natural units at most D u), c = scale log2 e is off by 2 u, which t shares; the exponential is off by 2 u.
A term of S is off by (3 D + 2) u. Its sum goes over 3 levels of its vector, n vectors, and 8 levels of lanes and waves, with
two or three changes of reference (each an exponential and a product: 3 u, and its exponent's rounding, D u) on the way and 6
more where workgroups meet: S is off by (n + 30 + 6 D) u, relative, and so is ln S, absolutely, with its own rounding of at
most 12 u. l_t - l_ref is two roundings of at most D u, and one more of the result:
    |logprob - exact| <= (n + 45 + 9 D) u + u |exact|.
The entropy is ln S - U / S, U's terms p |t| being off by what S's are and their own rounding, and p |t| sums to at most
H + 2 (references are at most 2 below a lane's largest): |entropy - exact| <= (n + 45 + 9 D) u (3 + H). D counts to 104: below
that terms are 0 in either.
"""
import math

import numpy as np
import pytest

import oracle.logprobs as L
import oracle.rope as OR
from paper_2608_15171_amd import inputs as I

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas, step
    return ppas, step, torch


def run(lib, x, tokens, top, scale=1.0, workspace="full", stream=None, **outs):
    """The results on the GPU for a device tensor of logits, as NumPy arrays."""
    ppas, step, torch = lib
    R, V = x.shape
    new = lambda *s, dt: torch.full(s, -7, dtype=dt, device="cuda")      # noqa: E731
    o = {"logprob": new(R, dt=torch.float32), "rank": new(R, dt=torch.int32), "entropy": new(R, dt=torch.float32)}
    if top:
        o |= {"top_ids": new(R, top, dt=torch.int32), "top_logprobs": new(R, top, dt=torch.float32)}
    ws = None
    size = ppas.logprobs_workspace_bytes(R, V, top)
    if workspace == "full" and size:
        ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    elif workspace == "some" and size:
        ws = torch.full((max(16, size // 3),), 0xff, dtype=torch.uint8, device="cuda")
    ppas.logprobs(x, tokens=torch.from_numpy(np.asarray(tokens, np.int32)).cuda(), scale=scale, workspace=ws, stream=stream, **o)
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in o.items()}


def check(got, x, tokens, top, scale, label, lanes=256, width=8):
    """x: float64 [R, V]."""
    u, worst = 2.0 ** -24, 0.0
    for r in range(x.shape[0]):
        want = L.row(x[r], scale, int(tokens[r]), top)
        assert got["rank"][r] == want["rank"], (label, r, got["rank"][r], want["rank"])
        if top:
            assert got["top_ids"][r].tolist() == want["top_ids"], (label, r, got["top_ids"][r].tolist(), want["top_ids"])
        live = x[r][np.isfinite(x[r])]
        D = min(104.0, scale * float(live.max() - live.min())) if len(live) else 0.0
        n = x.shape[1] / (lanes * width) + 1
        H = want["entropy"]
        for name, a, b, tol in (("logprob", got["logprob"][r], want["logprob"], None), ("entropy", got["entropy"][r], H, 3 + H),
                                *((f"top{j}", got["top_logprobs"][r][j], want["top_logprobs"][j], None) for j in range(top))):
            if math.isnan(b) or math.isinf(b):
                assert (math.isnan(a) and math.isnan(b)) or a == b, (label, r, name, a, b)
                continue
            # a masked or far token's own distance is past the spread that counts in the sums
            far = u * abs(b) * 4
            lim = (n + 45 + 9 * D) * u * (1.0 if tol is None else tol) + far
            worst = max(worst, abs(a - b) / lim)
            assert abs(a - b) <= lim, (label, r, name, a, b, lim)
    print(f"{label}: worst/tol={worst:.3f}", flush=True)


def logits(lib, values, dtype, pad=0, shift=0):
    """A device tensor of such rows, `pad` elements apart and `shift` into their buffer, and what it holds in 64 bits."""
    ppas, step, torch = lib
    R, V = values.shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((shift + R * (V + pad) + 16,), float("nan"), dtype=dt, device="cuda")
    x = buf.as_strided((R, V), (V + pad, 1), shift)
    x.copy_(torch.from_numpy(np.ascontiguousarray(values, dtype=np.float32)))
    return x, x.double().cpu().numpy()


def case(lib, values, dtype="bf16", tokens=None, top=5, scale=1.0, pad=0, shift=0, seed=0, workspace="full", label=""):
    g = I.rng(seed, *values.shape)
    tokens = g.integers(0, values.shape[1], values.shape[0]) if tokens is None else tokens
    x, exact = logits(lib, values, dtype, pad, shift)
    print(f"logprobs {label} {values.shape} {dtype} top={top} scale={scale} pad={pad} shift={shift} ws={workspace}", flush=True)
    got = run(lib, x, tokens, top, scale, workspace)
    check(got, exact, tokens, top, scale, label or "rows", width=8 if dtype == "bf16" else 4)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (2, 63), (3, 500), (2, 2047), (2, 2048), (2, 2049),
                                        (1, 4097), (7, 10007), (1, 65536), (3, 131072), (40, 30001), (2000, 300)])
@pytest.mark.parametrize("top", [0, 1, 20])
def test_sizes(lib, dtype, rows, vocab, top):
    case(lib, 3.0 * I.rng(1, rows, vocab).normal(size=(rows, vocab)), dtype, top=top, seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (0, 4), (1, 0), (3, 5), (8, 8), (7, 7)])
@pytest.mark.parametrize("vocab", [3, 13, 20000, 20011])
def test_strides_and_alignment(lib, dtype, pad, shift, vocab):
    """Rows that start anywhere: what lies between them (NaNs) is not read as theirs."""
    case(lib, 2.5 * I.rng(3, vocab).normal(size=(6, vocab)), dtype, top=7, pad=pad, shift=shift)


@pytest.mark.parametrize("workspace", ["full", "some", "none"])
@pytest.mark.parametrize("top", [0, 5, 64])
def test_splits(lib, workspace, top):
    case(lib, 3.0 * I.rng(4).normal(size=(3, 50021)), "bf16", top=top, workspace=workspace, pad=3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("workspace", ["full", "none"])
@pytest.mark.parametrize("top", [1, 5, 63, 64])
@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "two", "steps", "zeros", "last", "waves"])
def test_orders_and_ties(lib, dtype, workspace, top, order):
    """Orders that fill the lists at every step, and equal logits, which go to the lowest tokens."""
    V = 40000
    i = np.arange(V)
    v = {"ascending": i / 1000.0 - 20, "descending": 20 - i / 1000.0, "equal": np.full(V, 1.5), "two": (i % 3 == 1) * 2.0,
         "steps": (i // 700) % 9 * 1.0, "zeros": np.where(i % 2, 0.0, -0.0), "last": np.where(i >= V - 30, 3.0, -1.0),
         # one wave's tokens are the large ones, and rise
         "waves": np.where((i // 512) % 4 == 2, i / 2000.0, -5.0)}[order]
    tokens = [0, V - 1, 12345]
    case(lib, np.stack([v] * 3), dtype, tokens=tokens, top=top, workspace=workspace, label=order)
    case(lib, np.stack([v] * 3), dtype, tokens=tokens, top=top, workspace=workspace, label=order, pad=1, shift=3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("top", [3, 64])
@pytest.mark.parametrize("order", ["normal", "ascending", "equal", "one split"])
def test_most_splits(lib, dtype, top, order):
    """A row in 64 splits: its best in all of them, or all in one, which leaves the merge many candidates."""
    V = 600003
    i = np.arange(V)
    v = {"normal": 3.0 * I.rng(12).normal(size=V), "ascending": i / 10000.0, "equal": np.zeros(V),
         "one split": np.where((i > 300000) & (i < 300900), 2.0 + i % 7, i % 3)}[order]
    case(lib, v[None], dtype, tokens=[300500], top=top, label=order)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [200, 33000])
@pytest.mark.parametrize("workspace", ["full", "none"])
def test_masks(lib, dtype, vocab, workspace):
    """Few tokens left, in one place or spread, none, one, and masks of the type's lowest value; tokens that are masked."""
    g = I.rng(5, vocab)
    x = 2.0 * g.normal(size=(12, vocab))
    lowest = -3.3895313892515355e38
    keep = g.random((12, vocab)) < np.array([1, 0.5, 0.02, 0.02, 0.001, 0, 0, 1, 1, 0.02, 0, 0.3])[:, None]
    keep[0, :], keep[4, vocab - 3:], keep[5, 77] = True, True, True
    keep[7, :vocab // 2], keep[8, vocab // 2:] = False, False
    x[~keep] = -np.inf
    x[9][~keep[9]] = lowest
    x[10] = lowest                                         # all equal, none masked
    x[11][~keep[11]] = lowest
    x[11, 5] = -np.inf
    tokens = g.integers(0, vocab, 12)
    tokens[2], tokens[5], tokens[11] = int(np.flatnonzero(keep[2])[0]), 77, 5
    case(lib, x, dtype, tokens=tokens, top=8, workspace=workspace)
    case(lib, x, dtype, tokens=tokens, top=8, workspace=workspace, scale=0.25, pad=1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("vocab", [50, 9001])
def test_infinities_and_nans(lib, dtype, vocab):
    x = I.rng(6, vocab).normal(size=(6, vocab))
    x[0, 3], x[1, vocab - 1], x[2, :], x[3, 7], x[4, 0] = np.nan, np.inf, np.nan, np.inf, np.nan
    x[3, 8] = -np.inf
    got = case(lib, x, dtype, tokens=[0] * 6, top=3)
    assert np.isnan(got["logprob"][:5]).all() and not np.isnan(got["logprob"][5])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-3, 0.7, 30.0, 2.0 ** 100])
def test_scales(lib, dtype, scale):
    case(lib, 4.0 * I.rng(7).normal(size=(3, 5000)), dtype, top=4, scale=float(np.float32(scale)))


@pytest.mark.parametrize("at", [1e3, -5e4, 1e7, -3e38, 3e38])
def test_far_from_zero(lib, at):
    """fp32 logits in a cluster far from zero (as near one another as the type allows), and bf16 ones."""
    g = I.rng(8)
    step_of = float(np.spacing(np.float32(abs(at))))
    case(lib, at + step_of * g.integers(-4, 5, (3, 3000)), "fp32", top=6, scale=min(1.0, 30.0 / step_of))
    case(lib, at * (1.0 + g.integers(0, 3, (3, 3000)) / 128.0) if abs(at) < 1e38 else np.full((3, 3000), at), "bf16", top=6,
         scale=max(1e-30, min(1.0, 300.0 / abs(at))))


def test_confident_rows(lib):
    """One token far ahead: its log probability is a small difference from 0."""
    x = I.rng(9).normal(size=(4, 32768))
    x[0, 100], x[1, 32767], x[2, 0] = 40.0, 25.0, 200.0
    got = case(lib, x, "fp32", tokens=[100, 32767, 0, 5], top=2)
    assert got["rank"][:3].tolist() == [0, 0, 0] and (got["logprob"][:3] <= 0).all() and (got["entropy"] >= 0).all()


def test_tokens_out_of_range(lib):
    got = case(lib, I.rng(10).normal(size=(5, 100)), "bf16", tokens=[-1, 100, 2 ** 31 - 1, -2 ** 31, 99], top=1)
    assert got["rank"][:4].tolist() == [-1] * 4 and np.isnan(got["logprob"][:4]).all() and got["rank"][4] >= 0


def test_ranks_of_every_token(lib):
    """One row many times over, each time with another token, ties among them."""
    V = 777
    v = np.round(4.0 * I.rng(11).normal(size=V)) / 2.0
    got = case(lib, np.tile(v, (V, 1)), "bf16", tokens=np.arange(V), top=0)
    assert sorted(got["rank"].tolist()) == list(range(V))


def test_some_results_only(lib):
    ppas, step, torch = lib
    x = torch.randn(3, 5000, device="cuda").bfloat16()
    t = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    ws = torch.empty(max(16, ppas.logprobs_workspace_bytes(3, 5000, 4)), dtype=torch.uint8, device="cuda")
    want = run(lib, x, [1, 2, 3], 4)
    f = lambda *s: torch.zeros(s, device="cuda")                          # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")       # noqa: E731
    for name, out in (("logprob", f(3)), ("rank", i(3)), ("entropy", f(3)), ("top_ids", i(3, 4)), ("top_logprobs", f(3, 4))):
        ppas.logprobs(x, **{name: out}, **({"tokens": t} if name in ("logprob", "rank") else {}), workspace=ws)
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), want[name]), name
    with pytest.raises(ppas.PPASError):
        ppas.logprobs(x, logprob=f(3))
    ppas.logprobs(x[:0], entropy=f(0))
    with pytest.raises(ppas.PPASError):
        ppas.logprobs(x[:1].expand(3, -1), entropy=f(3))                  # rows on top of one another


def test_other_stream_and_replay(lib):
    ppas, step, torch = lib
    R, V, k = 5, 40009, 6
    size = ppas.logprobs_workspace_bytes(R, V, k)
    assert size > 0
    x = torch.randn(R, V, device="cuda").bfloat16()
    t = torch.randint(0, V, (R,), device="cuda", dtype=torch.int32)

    def outs():
        f = lambda *s: torch.zeros(s, device="cuda")                      # noqa: E731
        i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")   # noqa: E731
        return dict(logprob=f(R), rank=i(R), entropy=f(R), top_ids=i(R, k), top_logprobs=f(R, k))
    want, got = outs(), outs()
    ws, other = (torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2))

    def same(label):
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(want[name], got[name]), (label, name)
    ppas.logprobs(x, tokens=t, workspace=ws, **want)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    ppas.logprobs(x, tokens=t, workspace=other, stream=s, **got)
    same("stream")
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    s.wait_stream(torch.cuda.current_stream())
    for graph in graphs:                                                  # two graphs share a workspace, one after the other
        with torch.cuda.graph(graph, stream=s):
            ppas.logprobs(x, tokens=t, workspace=other, **got)
    for n in range(4):
        x.copy_(torch.randn(R, V, device="cuda") * (n + 1))
        t.copy_(torch.randint(0, V, (R,), device="cuda", dtype=torch.int32))
        ppas.logprobs(x, tokens=t, workspace=ws, **want)
        for o in got.values():
            o.zero_()
        graphs[n % 2].replay()
        same(n)


def test_rows_past_32_bit_offsets(lib):
    """Rows behind 2^32 bytes of others."""
    ppas, step, torch = lib
    V, far = 131072, 17000
    buf = torch.empty((far + 2) * V, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, V), (far * V, 1), 0)
    x.copy_(torch.randn(2, V, device="cuda"))
    got = run(lib, x, [3, 4], 9)
    check(got, x.double().cpu().numpy(), [3, 4], 9, 1.0, "far")


@pytest.mark.parametrize("V", [777, 40000])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_differences_past_fp32(lib, dtype, V):
    """Logits whose differences pass fp32's range, at scales that bring them back into it."""
    x = np.zeros((4, V))
    x[:2, 5], x[:2, 100], x[1, 400] = -2.0 ** 127.5, 2.0 ** 127.9, -np.inf
    x[2:, 7], x[2, 300], x[3] = 2.0 ** 127, -2.0 ** 127.9, -2.0 ** 127.9
    x[3, 9] = 2.0 ** 127.9
    case(lib, x, dtype, tokens=[5, 400, 300, 11], top=64, scale=2.0 ** -100)
    case(lib, x, dtype, tokens=[5, 5, 300, 11], top=3, scale=2.0 ** -60)


@pytest.mark.parametrize("dtype,V", [("bf16", 16384), ("fp32", 8192), ("bf16", 131072), ("fp32", 131072), ("bf16", 20003)])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_crowded_lanes(lib, dtype, V, top):
    """All of a few lanes' logits above all others: more candidates than a workgroup has room for."""
    W = 8 if dtype == "bf16" else 4
    g = I.rng(13, V)
    high = np.arange(V) // W % 256 < 80
    x = np.where(high, 5.0 + g.random((3, V)), -g.random((3, V)))
    x[1] = np.where(high, 5.0, -1.0)
    case(lib, x, dtype, top=top)
    case(lib, np.where(np.arange(V) % 7 == 3, x, -np.inf), dtype, top=top, shift=5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,V", [(1, 8191), (2, 8193), (3, 16385), (1, 262144), (200, 40000), (700, 8000), (90, 65537), (1100, 5000)])
def test_parts(lib, dtype, rows, V):
    """Rows about as long as a workgroup holds, and in as many parts as rows and lengths make."""
    x = 2.0 * I.rng(14, rows, V).normal(size=(rows, V))
    some = I.rng(15).permutation(rows)[:7]
    case(lib, x[some], dtype, top=33)
    if rows > 7:                      # all of them at once: the same, by the 7 that are looked at
        ppas, step, torch = lib
        t, exact = logits(lib, x, dtype)
        tokens = I.rng(16).integers(0, V, rows)
        got = run(lib, t, tokens, 20)
        check({k: v[some] for k, v in got.items()}, exact[some], tokens[some], 20, 1.0, f"{rows} rows",
              width=8 if dtype == "bf16" else 4)


@pytest.mark.parametrize("V", [75816, 131072, 300000])
@pytest.mark.parametrize("top", [2, 30, 64])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_join(lib, dtype, top, V):
    """Parts whose lists hold the first ones in every way: at random, all in one of them, equal ones, few of them not masked."""
    g = I.rng(17, V)
    x = np.stack([2.0 * g.normal(size=V), np.arange(V) / V, -np.arange(V) / V, np.full(V, -3.0),
                  np.where(g.random(V) < 0.5, 2.0 * g.normal(size=V), -np.inf),
                  np.where(np.arange(V) % (V // 11) == 5, g.normal(size=V), -np.inf),
                  np.round(2.0 * g.normal(size=V))])
    case(lib, x, dtype, top=top, scale=0.5)
