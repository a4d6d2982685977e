"""A served, fine-tuned model's operators together: two decoder layers over three iterations of requests that bring adapters of
their own, with normalised queries and keys, and the log probabilities that the requests are answered with.

An iteration sorts its rows by adapter once and makes one plan, for both layers. Each layer projects Q, K and V and adds the
adapters' shares to the queries and the values where they lie in the fused rows, normalises, turns and appends, attends, projects
the output with adapters in place, and runs the MLP with adapters before the activation and behind the down projection (one layer
in bf16, the other on 8-bit weights); the vocabulary projection's logits become log probabilities. Every stage is checked on the
inputs that it was given (the previous stage's own outputs), by the bounds of its operator's own tests.
"""
import numpy as np
import pytest

import oracle.adapters as A
import oracle.attention as OA
import oracle.kv_cache as OK
import oracle.rope as R
import test_gpu_adapters as TA
import test_gpu_logprobs as TL
import test_gpu_norm_rope as TN
from paper_2608_15171_amd import inputs as I

pytestmark = pytest.mark.gpu

HIDDEN, INTER, VOCAB, HQ, HKV, D = 256, 384, 5003, 16, 2, 128
N_ADAPTERS, RANK = 5, 16
RAMP = dict(scaling="ramp", factor=4.0, original_len=512, low=1.0, high=32.0)
W_REL = 2.0 ** -8 + 6e-4


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2608_15171_amd import ppas, step
    return ppas, step, torch


class Layer:
    def __init__(self, lib, seed, pages, eight_bit):
        ppas, step, torch = lib
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, scale=0.05: (torch.randn(*s, device="cuda", generator=g) * scale).bfloat16()      # noqa: E731
        self.eight_bit = eight_bit
        self.w, self.sets = {}, {}
        for name, n, k in (("qkv", (HQ + 2 * HKV) * D, HIDDEN), ("o", HIDDEN, HQ * D), ("gate_up", 2 * INTER, HIDDEN),
                           ("down", HIDDEN, INTER)):
            w = rand(n, k)
            if eight_bit:
                q, s = torch.empty(n, k, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
                ppas.quant_i8(w, q, s)
                w = (q, s)
            self.w[name] = w
        for name, n, k in (("q", HQ * D, HIDDEN), ("v", HKV * D, HIDDEN), ("o", HIDDEN, HQ * D), ("gate_up", 2 * INTER, HIDDEN),
                           ("down", HIDDEN, INTER)):
            self.sets[name] = ppas.adapters(rand(N_ADAPTERS, RANK, k), rand(N_ADAPTERS, n, RANK, scale=0.2),
                                            torch.rand(N_ADAPTERS, device="cuda", generator=g) + 0.5)
        self.norms = [ppas.head_norm(rand(D, scale=0.2), offset=1.0) for _ in range(2)]
        self.kp = torch.full((pages, HKV, D // 8, 16, 8), -1, dtype=torch.int16, device="cuda").view(torch.bfloat16)
        self.vp = torch.full((pages, HKV, D, 16), -1, dtype=torch.int16, device="cuda").view(torch.bfloat16)
        self.hist = {}                                  # request -> appended keys and values, as bf16 bits


def project(lib, x, w):
    """The shared projection, by the library's calls (which have tests of their own)."""
    ppas, step, torch = lib
    n = (w[0] if isinstance(w, tuple) else w).shape[0]
    y = torch.empty(x.shape[0], n, dtype=torch.bfloat16, device="cuda")
    if isinstance(w, tuple):
        q, s = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(x.shape[0], device="cuda")
        ppas.quant_i8(x, q, s)
        ppas.gateup_proj_i8(q, s, *w, y)
    else:
        ppas.gateup_proj(x, w, y)
    return y


def adapt(lib, s, x, y, order, ws, row_adapter, act=False, in_place=False):
    """The adapters' call on a projection's output, checked."""
    ppas, step, torch = lib
    f64 = lambda t: t.double().cpu().numpy()                                                                  # noqa: E731
    before = f64(y)
    out = y if in_place else torch.full((x.shape[0], y.shape[1] // (2 if act else 1)), float("nan"), dtype=torch.bfloat16, device="cuda")
    (ppas.adapter_act if act else ppas.adapter_add)(s, x, y, out, order, ws)
    a, b, scale = map(f64, s.tensors)
    z = before + A.share(f64(x), a, b, scale, row_adapter)
    d = TA.bounds(f64(x), a, b, scale, row_adapter, z)
    if act:
        want = A.silu_gate(z)
        (zg, zu), (dg, du) = np.split(z, 2, 1), np.split(d, 2, 1)
        tol = 2.0 ** -8 * np.abs(want) + 1.1 * dg * np.abs(zu) + (np.abs(A.silu_gate(np.concatenate((zg, np.ones_like(zg)), 1))) +
                                                                1.1 * dg) * du + 8 * TA.U * np.abs(want)
    else:
        want, tol = z, 2.0 ** -8 * np.abs(z) + d
    assert (np.abs(f64(out) - want) <= tol + 2.0 ** -133).all()
    return out


def run_layer(lib, L, x, plan, shape, desc, bt, bt_host, ids, order, ws, row_adapter):
    ppas, step, torch = lib
    T, wide = x.shape[0], (HQ + 2 * HKV) * D
    fused = project(lib, x, L.w["qkv"])
    keys = step.bits_of(fused[:, HQ * D:(HQ + HKV) * D])
    # shares of the queries and of the values, in place in the fused rows; the keys between them stay
    adapt(lib, L.sets["q"], x, fused[:, :HQ * D], order, ws, row_adapter, in_place=True)
    adapt(lib, L.sets["v"], x, fused[:, -HKV * D:], order, ws, row_adapter, in_place=True)
    assert np.array_equal(step.bits_of(fused[:, HQ * D:(HQ + HKV) * D]), keys) and fused.shape == (T, wide)
    rows = fused.view(T, HQ + 2 * HKV, D)
    q = torch.empty(T, HQ, D, dtype=torch.bfloat16, device="cuda")
    rope = ppas.rope(magnitude=1.1386, **RAMP)
    plan.norm_rope_qkv_append(*L.norms, rope, q, L.kp, L.vp, rows[:, :HQ], rows[:, HQ:-HKV], rows[:, -HKV:], bt)
    bits, pos = step.bits_of(rows), R.row_positions(desc)
    kp, vp = step.bits_of(L.kp), step.bits_of(L.vp)
    got_k = np.empty((T, HKV, D), np.uint16)
    for s, (at, n, c) in enumerate(desc.tolist()):
        got_k[at:at + n] = OK.gather(kp, vp, bt_host[s], c + n, 16)[0][c:]
    for name, got, src, norm in (("q", step.bits_of(q), bits[:, :HQ], L.norms[0]), ("k", got_k, bits[:, HQ:-HKV], L.norms[1])):
        ref, tol = TN.exact(R.bf16_bits_to_f64(src), norm.tensor.double().cpu().numpy(), pos, "half", D, 1e6,
                            float(np.float32(1e-6)), 1.0, False, magnitude=1.1386, **RAMP)
        TN.check(got, ref, tol, name)
    for s, (at, n, c) in enumerate(desc.tolist()):
        k, v = L.hist.get(ids[s], (np.zeros((0, HKV, D), np.uint16),) * 2)
        assert len(k) == c
        L.hist[ids[s]] = np.concatenate([k, got_k[at:at + n]]), np.concatenate([v, bits[at:at + n, -HKV:]])
    out = torch.empty_like(q)
    work = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    plan.attn_step(out, q, L.kp, L.vp, bt, work)
    O, Abs = OA.mixed_step_attention(step.bits_of(q), desc, [L.hist[i][0] for i in ids], [L.hist[i][1] for i in ids],
                                     shape.scale, HKV, with_abs=True)
    g = out.double().cpu().numpy()
    assert (np.abs(g - O) <= 2.0 ** -8 * np.abs(g) + W_REL * (Abs + np.abs(O)) + 1e-6).all()
    out = out.view(T, -1)
    h = x + adapt(lib, L.sets["o"], out, project(lib, out, L.w["o"]), order, ws, row_adapter, in_place=True)
    m = adapt(lib, L.sets["gate_up"], h, project(lib, h, L.w["gate_up"]), order, ws, row_adapter, act=True)
    return h + adapt(lib, L.sets["down"], m, project(lib, m, L.w["down"]), order, ws, row_adapter)


def test_iterations_of_two_adapted_layers(lib):
    ppas, step, torch = lib
    users, pages = 7, 120
    layers = [Layer(lib, 1, pages, False), Layer(lib, 2, pages, True)]
    shape = ppas.make_shape(HQ, HKV, pages)
    g = torch.Generator(device="cuda").manual_seed(3)
    head = (torch.randn(VOCAB, HIDDEN, device="cuda", generator=g) * 0.05).bfloat16()
    table = I.rng(1, 7).permutation(pages).astype(np.int32)[:7 * 14].reshape(7, 14)
    adapter = np.array([0, 3, -1, 3, 4, -1, 1])          # of each user; 2 is nobody's
    length = np.zeros(users, int)
    for it, new in enumerate(([130, 1, 40, 17, 3, 64, 90], [1] * 7, [1, 1, 1, 20, 1, 1, 1])):
        ids = list(range(users))
        desc = np.zeros((users, 3), np.int32)
        desc[:, 1], desc[:, 2] = new, length
        desc[1:, 0] = np.cumsum(new)[:-1]
        T = int(sum(new))
        length += new
        bt = torch.from_numpy(table).cuda()
        row_adapter = np.repeat(adapter, new).astype(np.int32)
        order = ppas.AdapterRows(T, N_ADAPTERS)
        order.sort(torch.from_numpy(row_adapter).cuda())
        ws = torch.empty(max(ppas.adapter_workspace_bytes(T, k, RANK, N_ADAPTERS) for k in (HIDDEN, HQ * D, INTER)),
                         dtype=torch.uint8, device="cuda")
        x = torch.randn(T, HIDDEN, device="cuda", generator=g).bfloat16()
        print(f"iteration {it}: rows={T} desc={desc.tolist()}", flush=True)
        with ppas.StepPlan(shape, desc, table) as plan:
            for L in layers:
                x = run_layer(lib, L, x, plan, shape, desc, bt, table, ids, order, ws, row_adapter)
                assert bool(torch.isfinite(x).all())
        # the last row of each request is answered
        last = x[torch.from_numpy(np.cumsum(new) - 1).cuda()]
        logits = project(lib, last, head)
        tokens = I.rng(it, 8).integers(0, VOCAB, users)
        TL.check(TL.run(lib, logits, tokens, 5, 0.8), logits.double().cpu().numpy(), tokens, 5, float(np.float32(0.8)), f"answers {it}")
    for L in layers:
        kp, vp = step.bits_of(L.kp), step.bits_of(L.vp)
        for u in range(users):
            k, v = OK.gather(kp, vp, table[u], int(length[u]), 16)
            assert np.array_equal(k, L.hist[u][0]) and np.array_equal(v, L.hist[u][1])


def calls(lib):
    """One valid call of every entry point, by name."""
    ppas, step, torch = lib
    spec = I.StepSpec("pair", [I.Seq(1, 64, 0), I.Seq(1, 64, 1)])
    data = I.make_step_data(spec, 1)
    bt, pages = I.make_block_table(spec, 1)
    ds = step.DeviceStep(data, bt, pages)
    plan = ds.plan()
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")                                 # noqa: E731
    rows, r, n = ds.q.clone(), ppas.rope(), ppas.head_norm(z(128))
    order, s = ppas.AdapterRows(2, 3), ppas.adapters(z(3, 8, 64), z(3, 32, 8), z(3, dt=torch.float32))
    ids, x, y, out, half = z(2, dt=torch.int32), z(2, 64), z(2, 32), z(2, 32), z(2, 16)
    ws, ent, pos = z(1 << 16, dt=torch.uint8), z(2, dt=torch.float32), z(2, dt=torch.int32)
    return plan, {
        "rows": lambda: ppas.norm_rope_rows(n, r, ds.q, pos, rows),
        "append": lambda: ppas.norm_rope_qkv_append(ds.shape, n, n, r, rows, ds.k_pages, ds.v_pages, ds.q, ds.k_new, ds.v_new,
                                                    ds.desc, ds.bt, ds.bt_host),
        "append planned": lambda: plan.norm_rope_qkv_append(n, n, r, rows, ds.k_pages, ds.v_pages, ds.q, ds.k_new, ds.v_new, ds.bt),
        "order": lambda: order.sort(ids),
        "adapters": lambda: ppas.adapter_add(s, x, y, out, order, ws),
        "adapters' activation": lambda: ppas.adapter_act(s, x, y, half, order, ws),
        "log probabilities": lambda: ppas.logprobs(y, entropy=ent, workspace=ws)}


def test_another_current_device_is_refused(lib, monkeypatch):
    ppas, step, torch = lib
    plan, each = calls(lib)
    for f in each.values():
        f()
    torch.cuda.synchronize()
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for name, f in each.items():
            with pytest.raises(ValueError, match="current device is 1"):
                f()
    plan.close()


def test_capture(lib):
    """Calls that stage lists refuse a capturing stream and leave the capture as it was; the others are captured."""
    ppas, step, torch = lib
    plan, each = calls(lib)
    for f in each.values():
        f()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        for name, f in each.items():
            if name.startswith("append"):
                with pytest.raises(ppas.PPASError) as e:
                    f()
                assert e.value.status == ppas.PPAS_EUNSUPPORTED, name
            else:
                f()
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        for f in each.values():
            f()
        torch.cuda.synchronize()
    plan.close()
