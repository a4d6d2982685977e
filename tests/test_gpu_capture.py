"""Capture into a HIP graph: every call that reads a step's lists from the pool of pinned buffers refuses it and leaves the
capture as it was; the call that allocates nothing can be captured and replayed."""
import numpy as np
import pytest

from paper_2608_15171_amd import inputs as I

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas, step
    return ppas, step, torch


def make(lib, n, cached, seed=1):
    ppas, step, torch = lib
    spec = I.StepSpec(f"capture{n}", [I.Seq(1, cached, i) for i in range(n)])
    data = I.make_step_data(spec, seed)
    bt, pages = I.make_block_table(spec, seed)
    ds = step.DeviceStep(data, bt, pages)
    ds.fill_history()
    ds.append()
    return ds


@pytest.mark.parametrize("n", [2, 80])
def test_calls_that_read_lists_refuse_capture(lib, n):
    ppas, step, torch = lib
    ds = make(lib, n, 64)
    shared_bt = ds.bt_host.copy()
    shared_bt[:, :4] = shared_bt[0, :4]
    prefixes = [(0, n, 64)]
    plain = ppas.StepPlan(ds.shape, ds.desc, ds.bt_host)
    shared = ppas.StepPlan(ds.shape, ds.desc, shared_bt, prefixes=prefixes, opts=ppas.plan_opts(64, 0, 0))
    bt = torch.from_numpy(shared_bt).cuda()
    work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    q, r = ds.q.clone(), ppas.rope()
    pools = ds.k_pages, ds.v_pages
    step_of = ds.desc, ds.bt
    new = ds.k_new, ds.v_new
    calls = {
        "append": lambda: ppas.kv_append(ds.shape, *pools, *new, *step_of, ds.bt_host),
        "rotating append": lambda: ppas.rope_kv_append(ds.shape, 1e6, q, *pools, *new, *step_of, ds.bt_host),
        "rotary append": lambda: ppas.rope_qkv_append(ds.shape, r, q, *pools, ds.q, *new, *step_of, ds.bt_host),
        "attention": lambda: ppas.attn_step(ds.shape, ds.out, ds.q, *pools, *step_of, work, ds.bt_host),
        "attention, no prefix": lambda: ppas.attn_step_shared(ds.shape, ds.out, ds.q, *pools, ds.desc, [], ds.bt, work, ds.bt_host),
        "attention, prefix": lambda: ppas.attn_step_shared(ds.shape, ds.out, ds.q, *pools, ds.desc, prefixes, bt, work, shared_bt),
        "append, planned": lambda: plain.kv_append(*pools, *new, ds.bt),
        "rotating append, planned": lambda: plain.rope_kv_append(1e6, q, *pools, *new, ds.bt),
        "rotary append, planned": lambda: plain.rope_qkv_append(r, q, *pools, ds.q, *new, ds.bt),
        "attention, planned": lambda: plain.attn_step(ds.out, ds.q, *pools, ds.bt, work),
        "attention, planned with a prefix": lambda: shared.attn_step(ds.out, ds.q, *pools, bt, work)}
    pos, rows = torch.arange(n, device="cuda", dtype=torch.int32), torch.empty_like(ds.q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        for name, f in calls.items():
            with pytest.raises(ppas.PPASError) as e:
                f()
            assert e.value.status == ppas.PPAS_EUNSUPPORTED, name
        ppas.rope_rows(r, ds.q, pos, rows)
    want = torch.empty_like(rows)
    ppas.rope_rows(r, ds.q, pos, want)
    for _ in range(3):
        rows.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(rows.view(torch.int16), want.view(torch.int16))
        for f in calls.values():
            f()
        torch.cuda.synchronize()
    plain.close()
    shared.close()


def test_the_call_that_allocates_nothing_is_replayed(lib):
    """Between the replays another step's list takes the device array, and host memory as large as the list is written."""
    ppas, step, torch = lib
    a, b = make(lib, 7, 3000, seed=3), make(lib, 30, 500, seed=4)

    def call(ds):
        ppas.attn_step_noalloc(ds.shape, ds.out, ds.q, ds.k_pages, ds.v_pages, ds.desc, ds.bt, ds.bt_host)
    call(a)
    torch.cuda.synchronize()
    want = a.out.clone()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(a)
    for k in range(4):
        call(b)
        torch.cuda.synchronize()
        junk = [np.full(n, 7, np.uint8) for n in (1 << 10, 1 << 12, 1 << 14, 1 << 16) for _ in range(20)]
        a.out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out.view(torch.int16), want.view(torch.int16)), k
        del junk
