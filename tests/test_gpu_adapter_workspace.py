"""One workspace for steps of every size: hidden is split as far as it holds. Inputs are small whole numbers and powers of
two, so that every sum is exact, in any number of splits, and results are rounded once."""
import numpy as np
import pytest

from paper_2608_15171_amd import inputs as I

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas
    return ppas, torch


def inputs(torch, T, hidden, out, rank, n, wide):
    """A tenth of the features are not 0: v is at most a few thousand, 128 of those with B below 2^20, in quarters below 2^22."""
    g = I.rng(41, T, hidden, rank)
    dev = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda().bfloat16()       # noqa: E731
    x = dev(g.integers(-1, 2, (T, hidden)) * (g.random((T, hidden)) < 0.1))
    a, b = dev(g.integers(-3, 4, (n, rank, hidden))), dev(g.integers(-1, 2, (n, wide, rank)))
    y = dev(g.integers(-100, 101, (T, wide)))
    scale = torch.from_numpy(np.float32(2.0) ** g.integers(-2, 1, n).astype(np.float32)).cuda()
    rows = torch.from_numpy(g.integers(-1, n, T).astype(np.int32)).cuda()
    z = y.double()
    for k in range(n):
        at = (rows == k).nonzero()[:, 0]
        z[at] += torch.matmul(torch.matmul(x[at].double(), a[k].double().t()) * scale[k].double(), b[k].double().t())
    return x, a, b, y, scale, rows, z


def call(ppas, torch, x, a, b, y, scale, rows, ws, act=False):
    T, n = len(x), len(a)
    order = ppas.AdapterRows(T, n)
    order.sort(rows)
    out = torch.empty(T, y.shape[1] // (2 if act else 1), dtype=torch.bfloat16, device="cuda")
    (ppas.adapter_act if act else ppas.adapter_add)(ppas.adapters(a, b, scale), x, y, out, order, ws)
    return out


@pytest.mark.parametrize("hidden,rank,n", [(2048, 16, 4), (11008, 8, 24), (5504, 64, 1)])
def test_made_for_the_largest_step(lib, hidden, rank, n):
    ppas, torch = lib
    most = 16384
    ws = torch.empty(ppas.adapter_workspace_bytes(most, hidden, rank, n), dtype=torch.uint8, device="cuda")
    sizes = (16384, 16132, 12000, 8200, 4097, 2048, 700, 65, 64, 17, 1)
    assert max(ppas.adapter_workspace_bytes(T, hidden, rank, n) for T in sizes) > ws.numel()
    for T in sizes:
        print(f"one workspace: T={T} hidden={hidden} rank={rank} n={n}", flush=True)
        *args, z = inputs(torch, T, hidden, 40, rank, n, 40)
        ws.fill_(0xff)
        got = call(ppas, torch, *args, ws)
        assert torch.equal(got, z.float().bfloat16()), T


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("T,rank", [(1, 16), (40, 17), (300, 8), (700, 128)])
def test_fewer_splits(lib, act, T, rank):
    """Every number of splits down to one, and nothing written past the buffer; below one the call is refused."""
    ppas, torch = lib
    hidden, n, N = 4096 + 520, 3, 48
    one = 4 * T * min(k for k in (16, 32, 64, 128) if k >= rank)
    full = ppas.adapter_workspace_bytes(T, hidden, rank, n)
    assert full % one == 0 and full // one > 2
    *args, z = inputs(torch, T, hidden, N, rank, n, 2 * N if act else N)
    want = call(ppas, torch, *args, torch.empty(full, dtype=torch.uint8, device="cuda"), act)
    if not act:
        assert torch.equal(want, z.float().bfloat16())
    for size in (*range(one, full + 1, one), one + 16, 2 * one - 16):
        print(f"fewer splits: T={T} rank={rank} act={act} {size} of {full} bytes", flush=True)
        buf = torch.full((size + 64,), 0xff, dtype=torch.uint8, device="cuda")
        assert torch.equal(call(ppas, torch, *args, buf[:size], act), want), size
        assert bool((buf[size:] == 0xff).all())
    with pytest.raises(ppas.PPASError) as e:
        call(ppas, torch, *args, torch.empty(one - 16, dtype=torch.uint8, device="cuda"), act)
    assert e.value.status == ppas.PPAS_ENOSPACE
