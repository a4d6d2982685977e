"""GPU parity of attention with shared prefixes (ppas_step_plan_create_shared, ppas_attn_step_shared) against the
64-bit oracle, which knows no sharing: every request has its whole history to itself there.

Bounds are those of the plain attention's parity tests: each weight is rounded to bf16 (2^-8, shared by numerator and
denominator), logits and sums are fp32 (6e-4 covers them and the joins), and the output is rounded by 2^-8 of itself:
    |gpu - O| <= 2^-8 |gpu| + (2^-8 + 6e-4) (A + |O|) + 1e-6,  A the weighted mean of |V|.
"""
import numpy as np
import pytest

import oracle.attention as OA
from paper_2608_15171_amd import inputs as I

pytestmark = pytest.mark.gpu

W_REL = 2.0 ** -8 + 6e-4
SENTINEL = 0xFFFF


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas, step
    return ppas, step, torch


def make_step(lib, spec, prefixes, seed):
    """A step whose groups' members hold the first member's first rows, in its pages; unowned slots are NaN."""
    ppas, step, torch = lib
    data = I.make_step_data(spec, seed)
    bt, npages = I.make_block_table(spec, seed, spare_pages=3)
    lead = {}
    for first, n, length in prefixes:
        for s in range(first, first + n):
            lead[s] = (first, length)
            data.k_hist[s][:length] = data.k_hist[first][:length]
            data.v_hist[s][:length] = data.v_hist[first][:length]
            bt[s, :length // 16] = bt[first, :length // 16]
    ds = step.DeviceStep(data, bt, npages, pool_fill=SENTINEL)
    # each request writes what is its own; the first member of a group writes the prefix too
    todo = [(s, 0 if lead.get(s, (s, 0))[0] == s else lead[s][1]) for s in range(len(spec.seqs))]
    todo = [(s, at) for s, at in todo if spec.seqs[s].cached_len > at]
    if todo:
        k = np.concatenate([data.k_hist[s][at:] for s, at in todo])
        v = np.concatenate([data.v_hist[s][at:] for s, at in todo])
        desc, row = np.zeros((len(todo), 3), np.int32), 0
        for i, (s, at) in enumerate(todo):
            desc[i] = (row, spec.seqs[s].cached_len - at, at)
            row += desc[i, 1]
        host = np.ascontiguousarray(bt[[s for s, _ in todo]])
        ppas.kv_append(ds.shape, ds.k_pages, ds.v_pages, step.to_device_bf16(k), step.to_device_bf16(v), desc,
                       torch.from_numpy(host).cuda(), host)
    ds.append()
    return data, ds


def attend(lib, ds, prefixes, opts=None, direct=False):
    """The output, with rows behind the step's last one that have to stay as they were."""
    ppas, step, torch = lib
    T = ds.data.spec.n_rows
    out = torch.full((T + 2, *ds.out.shape[1:]), -1, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    if direct:
        ws = torch.full((ppas.attn_shared_workspace_bytes(ds.shape, ds.desc, prefixes),), 255, dtype=torch.uint8, device="cuda")
        ppas.attn_step_shared(ds.shape, out, ds.q, ds.k_pages, ds.v_pages, ds.desc, prefixes, ds.bt, ws, ds.bt_host)
    else:
        with ppas.StepPlan(ds.shape, ds.desc, ds.bt_host, opts=opts, prefixes=prefixes) as plan:
            ws = torch.full((plan.workspace_bytes,), 255, dtype=torch.uint8, device="cuda")
            plan.attn_step(out, ds.q, ds.k_pages, ds.v_pages, ds.bt, ws)
    torch.cuda.synchronize()
    assert (step.bits_of(out[T:]) == SENTINEL).all()
    return out[:T]


def compare(out, ref, label):
    O, A = ref
    g = out.float().cpu().numpy().astype(np.float64)
    assert np.isfinite(g).all(), label
    err, bound = np.abs(g - O), 2.0 ** -8 * np.abs(g) + W_REL * (A + np.abs(O)) + 1e-6
    print(f"{label}: max_abs={err.max():.3e} err/bound={float((err / bound).max()):.3f}", flush=True)
    assert (err <= bound).all(), f"{label}: {int((err > bound).sum())} elements beyond the bound"


def random_step(seed):
    """Groups of decode rows and chunks behind a prefix, with requests that share nothing among them."""
    g = I.rng(seed, 77)
    seqs, prefixes = [], []

    def loose():
        for _ in range(int(g.integers(0, 3))):
            seqs.append(I.Seq(int(g.choice([1, 1, 5, 40])), int(g.integers(0, 200)), len(seqs)))
    for _ in range(int(g.integers(1, 4))):
        loose()
        n, length = int(g.integers(1, 9)), 16 * int(g.integers(0, 40))
        prefixes.append((len(seqs), n, length))
        for _ in range(n):
            rows = int(g.choice([1, 1, 1, 2, 7, 16, 17, 33, 64, 65, 100]))
            seqs.append(I.Seq(rows, length + int(g.choice([0, 1, 15, 16, 63, 64, 200, int(g.integers(0, 400))])), len(seqs)))
    loose()
    heads = dict(n_q_heads=8, n_kv_heads=1) if seed % 3 == 2 else {}
    return I.StepSpec(f"shared{seed}", seqs, **heads), prefixes


@pytest.mark.parametrize("seed", range(10))
def test_random_steps(lib, seed):
    spec, prefixes = random_step(seed)
    print(f"shared seed={seed} prefixes={prefixes} seqs={[(s.n_query, s.cached_len) for s in spec.seqs]}", flush=True)
    data, ds = make_step(lib, spec, prefixes, seed)
    ref = OA.step_attention_from_data(data, ds.shape.scale, with_abs=True)
    ppas = lib[0]
    for tile in (0, 16, 32):
        for splits in ((0, 0), (64, 32), (192, 96)):
            out = attend(lib, ds, prefixes, ppas.plan_opts(splits[0], splits[1], tile))
            compare(out, ref, f"seed={seed} tile={tile} splits={splits}")
    direct = attend(lib, ds, prefixes, direct=True)
    assert bool((direct == attend(lib, ds, prefixes)).all())


@pytest.mark.parametrize("length", [0, 16, 48, 64, 80, 128, 1024])
@pytest.mark.parametrize("rows", [1, 2, 16])
def test_prefix_lengths(lib, length, rows):
    """Whole and part 64-key blocks; requests with nothing of their own but their new rows."""
    seqs = [I.Seq(rows, length + own, i) for i, own in enumerate((0, 0, 1, 16, 70))]
    spec, prefixes = I.StepSpec("lengths", seqs), [(0, 5, length)]
    data, ds = make_step(lib, spec, prefixes, 3)
    ref = OA.step_attention_from_data(data, ds.shape.scale, with_abs=True)
    for tile in (16, 32):     # a split size shares whatever a step saves
        compare(attend(lib, ds, prefixes, lib[0].plan_opts(128, 0, tile)), ref, f"length={length} rows={rows} tile={tile}")


@pytest.mark.parametrize("n", [1, 2, 3, 17, 33, 130])
def test_group_sizes(lib, n):
    seqs = [I.Seq(1, 320 + 3 * i, i) for i in range(n)]
    spec, prefixes = I.StepSpec("sizes", seqs), [(0, n, 320)]
    data, ds = make_step(lib, spec, prefixes, 4)
    ref = OA.step_attention_from_data(data, ds.shape.scale, with_abs=True)
    for tile in (16, 32):
        compare(attend(lib, ds, prefixes, lib[0].plan_opts(128, 0, tile)), ref, f"n={n} tile={tile}")


@pytest.mark.parametrize("prefix,n,own", [(8192, 40, 700), (20000, 24, 64), (30000, 3, 2000)])
def test_long_prefixes(lib, prefix, n, own):
    g = I.rng(6, prefix)
    seqs = [I.Seq(1, prefix + int(g.integers(0, own)), i) for i in range(n)] + [I.Seq(30, prefix + 5, n), I.Seq(1, 900, n + 1)]
    spec, prefixes = I.StepSpec("long", seqs), [(0, n + 1, prefix)]
    data, ds = make_step(lib, spec, prefixes, 5)
    ref = OA.step_attention_from_data(data, ds.shape.scale, with_abs=True)
    for tile in (0, 16, 32):
        compare(attend(lib, ds, prefixes, lib[0].plan_opts(0, 0, tile)), ref, f"prefix={prefix} tile={tile}")


def test_dominant_keys_on_either_side_of_the_join(lib):
    """Logits around +-60 in the prefix or among the own keys: the join's rescaling on both sides."""
    ppas, step, torch = lib
    seqs = [I.Seq(1, 640 + 40 * (i % 3), i) for i in range(12)]
    spec, prefixes = I.StepSpec("dominant", seqs), [(0, 12, 640)]
    data = I.make_step_data(spec, 8)
    data, ds = make_step(lib, spec, prefixes, 8)
    q = ds.q.clone()
    q[::2] *= 16
    q[1::4] = 0
    ds.q.copy_(q)
    moved = I.StepData(data.spec, data.desc, step.bits_of(ds.q), data.k_new, data.v_new, data.k_hist, data.v_hist)
    O, A = OA.step_attention_from_data(moved, ds.shape.scale, with_abs=True)
    g = attend(lib, ds, prefixes, ppas.plan_opts(256, 0, 0)).float().cpu().numpy().astype(np.float64)
    # logits are 16 times larger: their fp32 error (128 products, sums of up to ~100) moves a weight by up to 16 x 2e-4
    bound = 2.0 ** -8 * np.abs(g) + (2.0 ** -8 + 6e-4 + 16 * 2e-4) * (A + np.abs(O)) + 1e-6
    assert (np.abs(g - O) <= bound).all()


def test_plan_serves_layers_streams_and_other_pools(lib):
    """One plan, two layers' pools on two streams with their own workspaces, twice each."""
    ppas, step, torch = lib
    spec, prefixes = I.StepSpec("layers", [I.Seq(1, 512 + 9 * i, i) for i in range(20)]), [(0, 20, 512)]
    made = [make_step(lib, spec, prefixes, s) for s in (11, 12)]
    refs = [OA.step_attention_from_data(d, ds.shape.scale, with_abs=True) for d, ds in made]
    a, b = made[0][1], made[1][1]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    with ppas.StepPlan(a.shape, a.desc, None, a.bt_host.shape[1], ppas.plan_opts(256, 0, 0), prefixes) as plan:
        ws = [torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda") for _ in range(2)]
        outs = [torch.zeros_like(a.out) for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(2):
            for k, (_, ds) in enumerate(made):
                plan.attn_step(outs[k], ds.q, ds.k_pages, ds.v_pages, ds.bt, ws[k], stream=streams[k])
        torch.cuda.synchronize()
    for k in range(2):
        compare(outs[k], refs[k], f"layer {k}")


def test_same_results_whenever_run(lib):
    spec, prefixes = random_step(21)
    _, ds = make_step(lib, spec, prefixes, 21)
    for opts in (None, lib[0].plan_opts(64, 0, 0)):
        a = attend(lib, ds, prefixes, opts)
        assert bool((a == attend(lib, ds, prefixes, opts)).all())


def test_without_prefixes_is_the_plain_step(lib):
    ppas, step, torch = lib
    spec, _ = random_step(5)
    data, ds = make_step(lib, spec, [], 5)
    plain = torch.empty_like(ds.out)
    ppas.attn_step(ds.shape, plain, ds.q, ds.k_pages, ds.v_pages, ds.desc, ds.bt, ds.workspace, ds.bt_host)
    for p in ([], None, [(0, len(spec.seqs), 0)]):
        assert bool((attend(lib, ds, p) == plain).all())
        assert bool((attend(lib, ds, p, direct=True) == plain).all())


def test_pages_past_32_bit_offsets(lib, monkeypatch):
    """Pools of 4.9 GB each, in whose last pages the step's keys and values lie."""
    make = I.make_block_table

    def shifted(spec, seed, spare_pages=0):
        bt, pages = make(spec, seed, spare_pages=spare_pages)
        return np.where(bt >= 0, bt + (600000 - pages), bt).astype(np.int32), 600000

    monkeypatch.setattr(I, "make_block_table", shifted)
    seqs = [I.Seq(1, 2048 + 50 * i, i) for i in range(20)] + [I.Seq(20, 2048, 20)]
    spec, prefixes = I.StepSpec("far", seqs), [(0, 21, 2048)]
    data, ds = make_step(lib, spec, prefixes, 9)
    ref = OA.step_attention_from_data(data, ds.shape.scale, with_abs=True)
    for tile in (16, 32):
        compare(attend(lib, ds, prefixes, lib[0].plan_opts(512, 0, tile)), ref, f"far tile={tile}")


@pytest.mark.parametrize("own", [16385, 32767])
def test_own_ranges_in_the_longest_pieces(lib, own):
    seqs = [I.Seq(1, 1024 + own - 1, i) for i in range(2)] + [I.Seq(1, 1030, 2)]
    spec, prefixes = I.StepSpec("pieces", seqs), [(0, 3, 1024)]
    data, ds = make_step(lib, spec, prefixes, 10)
    ref = OA.step_attention_from_data(data, ds.shape.scale, with_abs=True)
    for tile in (16, 32):
        compare(attend(lib, ds, prefixes, lib[0].plan_opts(1024, 1 << 20, tile)), ref, f"own={own} tile={tile}")
