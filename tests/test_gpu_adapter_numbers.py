"""Every number that is no adapter's, in one step: such rows are without one. Whole numbers, so that results are exact."""
import numpy as np
import pytest

import oracle.adapters as A
from paper_2608_15171_amd import inputs as I

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,n", [(600, 9), (600, 64), (65, 1), (1500, 1024), (23, 3)])
@pytest.mark.parametrize("act", [False, True])
def test_numbers_outside_the_set(T, n, act):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas
    H, N, r = 64, 48, 16
    g = I.rng(61, T, n)
    i = np.arange(T)
    outside = np.array([n, n + 1, -5, 2 ** 31 - 1, -2 ** 31, -1, 1024, 1025, -n])
    outside = outside[(outside < 0) | (outside >= n)]
    rows = np.where(i % 3 == 0, outside[i // 3 % len(outside)], i % n).astype(np.int32)
    if T >= 3 * len(outside):
        assert set(outside.tolist()) <= set(rows.tolist())
    dev = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda().bfloat16()       # noqa: E731
    x, y = g.integers(-2, 3, (T, H)), g.integers(-100, 101, (T, 2 * N if act else N))
    a, b = g.integers(-2, 3, (n, r, H)), g.integers(-2, 3, (n, y.shape[1], r))
    if act:
        y[:, :N], b[:, :N] = 0, 0                       # silu(64) is 64 in fp32: 64 times the second half is left
        y[:, :N] = 64
    order = ppas.AdapterRows(T, n)
    order.sort(torch.from_numpy(rows).cuda())
    ws = torch.empty(max(16, ppas.adapter_workspace_bytes(T, H, r, n)), dtype=torch.uint8, device="cuda")
    out = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    (ppas.adapter_act if act else ppas.adapter_add)(ppas.adapters(dev(a), dev(b)), dev(x), dev(y), out, order, ws)
    torch.cuda.synchronize()
    z = y + A.share(x.astype(float), a.astype(float), b.astype(float), None, rows)
    z = 64 * z[:, N:] if act else z
    assert torch.equal(out, torch.from_numpy(z).float().bfloat16().cuda())
    none = (rows < 0) | (rows >= n)
    groups = A.order(rows, n)
    assert np.array_equal(groups[-1], np.flatnonzero(none)) and none.sum() == (T + 2) // 3
    words = order.buf.cpu().numpy().view(np.int32)
    assert np.array_equal(words[-T:], np.concatenate(groups))
