"""GPU parity of decode rows that one wave takes (their own keys behind a shared prefix, or all they have), against the same
64-bit oracle and bounds as the shared prefixes' tests. Every case first checks that its plan holds such rows."""
import numpy as np
import pytest

import oracle.attention as OA
from paper_2608_15171_amd import inputs as I
from test_gpu_shared_prefix import W_REL, attend, compare, make_step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas, step
    return ppas, step, torch


# keys of a row's own: parts of a 32-key block, whole ones, odd and even numbers of blocks, up to sixteen; the last is one too
# many for a wave
OWN = [1, 31, 32, 33, 63, 64, 65, 96, 100, 127, 128, 129, 300, 511, 512, 513]


def single_waves(lib, ds, prefixes, opts):
    it = lib[0].plan_items(ds.shape, ds.desc, opts=opts, prefixes=prefixes)
    return it[it[:, 0] == 2]


@pytest.mark.parametrize("tile", [16, 32])
@pytest.mark.parametrize("hkv,n,prefix,cus", [(1, 100, 1024, 16), (2, 64, 1024, 16), (2, 40, 2048, 4), (1, 64, 2048, 8)])
def test_own_lengths(lib, hkv, n, prefix, cus, tile):
    """Behind a prefix, where a wave's result is a partial, and apart from one, where it is written whole."""
    heads = dict(n_q_heads=8, n_kv_heads=1) if hkv == 1 else {}
    seqs = [I.Seq(1, prefix + OWN[i % 16] - 1, i) for i in range(n)]
    loose = [I.Seq(1, OWN[i] - 1, n + i) for i in range(16)]
    spec, prefixes = I.StepSpec("waves", loose[:8] + seqs + loose[8:], **heads), [(8, n, prefix)]
    data, ds = make_step(lib, spec, prefixes, 31)
    opts = lib[0].plan_opts(0, 0, tile, cus)
    rows = single_waves(lib, ds, prefixes, opts)
    for behind in (True, False):
        lengths = (rows[:, 7] - rows[:, 6])[(rows[:, 6] > 0) == behind]
        assert set(lengths.tolist()) == set(OWN[:-1]), behind
    ref = OA.step_attention_from_data(data, ds.shape.scale, with_abs=True)
    compare(attend(lib, ds, prefixes, opts), ref, f"hkv={hkv} n={n} prefix={prefix} tile={tile}")


@pytest.mark.parametrize("n", [29, 30, 31, 32, 33])
def test_last_workgroup_of_rows(lib, n):
    """Numbers of rows that leave some of the last workgroup's waves without one."""
    seqs = [I.Seq(1, 4096 + 10 * (i % 7), i) for i in range(n)]
    spec, prefixes = I.StepSpec("last", seqs), [(0, n, 4096)]
    data, ds = make_step(lib, spec, prefixes, 32)
    ref = OA.step_attention_from_data(data, ds.shape.scale, with_abs=True)
    for tile in (16, 32):
        opts = lib[0].plan_opts(0, 0, tile, 8)
        assert len(single_waves(lib, ds, prefixes, opts)) == 2 * n
        compare(attend(lib, ds, prefixes, opts), ref, f"n={n} tile={tile}")


def test_dominant_keys_on_either_side(lib):
    """Logits around +-60 in the prefix or among a wave's own keys."""
    ppas, step, torch = lib
    seqs = [I.Seq(1, 1024 + OWN[i % 15] - 1, i) for i in range(64)]
    spec, prefixes = I.StepSpec("dominant", seqs), [(0, 64, 1024)]
    data, ds = make_step(lib, spec, prefixes, 33)
    q = ds.q.clone()
    q[::2] *= 16
    q[1::4] = 0
    ds.q.copy_(q)
    moved = I.StepData(data.spec, data.desc, step.bits_of(ds.q), data.k_new, data.v_new, data.k_hist, data.v_hist)
    O, A = OA.step_attention_from_data(moved, ds.shape.scale, with_abs=True)
    for tile in (16, 32):
        opts = ppas.plan_opts(0, 0, tile, 16)
        assert len(single_waves(lib, ds, prefixes, opts)) == 128
        g = attend(lib, ds, prefixes, opts).float().cpu().numpy().astype(np.float64)
        # logits are 16 times larger: their fp32 error (128 products, sums of up to ~100) moves a weight by up to 16 x 2e-4
        bound = 2.0 ** -8 * np.abs(g) + (W_REL + 16 * 2e-4) * (A + np.abs(O)) + 1e-6
        assert (np.abs(g - O) <= bound).all(), tile


def test_a_whole_chip_of_them(lib):
    """256 continuations of a 24,576-token document, planned as a program would; the reference in 64 bits on the GPU."""
    ppas, step, torch = lib
    n, prefix, hkv = 256, 24576, 2
    g = torch.Generator(device="cuda").manual_seed(5)
    own = [OWN[i % 15] for i in range(n)]
    desc = np.array([[i, 1, prefix + own[i] - 1] for i in range(n)], np.int32)
    shared, per = prefix // 16, 33
    pages = shared + n * per
    order = I.rng(5, 5).permutation(pages).astype(np.int32)
    bt_host = np.empty((n, shared + per), np.int32)
    bt_host[:, :shared], bt_host[:, shared:] = order[:shared], order[shared:].reshape(n, per)
    shape = ppas.make_shape(8 * hkv, hkv, pages)
    kp = torch.randn(pages, hkv, 16, 16, 8, device="cuda", generator=g).bfloat16()
    vp = torch.randn(pages, hkv, 128, 16, device="cuda", generator=g).bfloat16()
    q = torch.randn(n, 8 * hkv, 128, device="cuda", generator=g).bfloat16()
    bt, out = torch.from_numpy(bt_host).cuda(), torch.zeros_like(q)
    prefixes = [(0, n, prefix)]
    assert (ppas.plan_items(shape, desc, prefixes=prefixes)[:, 0] == 2).sum() == n * hkv
    ws = torch.empty(ppas.attn_shared_workspace_bytes(shape, desc, prefixes), dtype=torch.uint8, device="cuda")
    ppas.attn_step_shared(shape, out, q, kp, vp, desc, prefixes, bt, ws, bt_host)
    for i in range(n):
        ids, keys = bt[i].long(), prefix + own[i]
        for h in range(hkv):
            k = kp[ids, h].permute(0, 2, 1, 3).reshape(-1, 128)[:keys].double()
            v = vp[ids, h].transpose(1, 2).reshape(-1, 128)[:keys].double()
            p = torch.softmax(torch.matmul(q[i, 8 * h:8 * h + 8].double(), k.t().contiguous()) * shape.scale, -1)
            o, a = torch.matmul(p, v), torch.matmul(p, v.abs())
            got = out[i, 8 * h:8 * h + 8].double()
            bound = 2.0 ** -8 * got.abs() + W_REL * (a + o.abs()) + 1e-6
            assert bool(((got - o).abs() <= bound).all()), (i, h)
