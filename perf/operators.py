"""Timed cases of the operators around one decoder layer's serving step: rotary positions in all their forms, the
page write that applies them on the way, attention for requests that share a prefix, and 8-bit products.

Shapes are those of the repository's workloads (16 query and 2 KV heads of 128 features, or the two-way shard's 8 and
1; pages of 16 tokens; hidden 2048 and 11008 intermediate features, or the shard's 5504). Every case has a kind:
  rotate  the query and key heads of a step's rows, where the QKV projection left them, turned by their positions
  append  a step's QKV rows: rotated queries to their buffer, rotated keys and plain values to the pages
  shared  one step's attention where groups of requests share their first cached tokens, with a plan that the
          program keeps for the layers of an iteration ("planned") or by the call that plans for itself ("direct")
  step    append, then shared
  i8      activations quantised by token, then a product with weights quantised by channel ("proj"), or the gate
          and up products with the gated activation ("act")
`run` computes them in plain torch, or where `own` is true by the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE, DIM, GROUP = 16, 128, 8
THETA = 1e6
# frequency scaling: the length that positions were learned over, the bands in rotations over it, the ramp's ends in
# rotations over it
ORIGINAL, BAND_LOW, BAND_HIGH, RAMP_FAST, RAMP_SLOW = 8192, 1.0, 4.0, 32.0, 1.0
GOLDEN = 0.6180339887498949


def _rope(layout="half", rotary=DIM, scaling="none", factor=1.0):
    return {"layout": layout, "rotary": rotary, "scaling": scaling, "factor": factor}


def _rows_case(kind, name, rows, position, kv_heads=2, **rope):
    return {"name": name, "kind": kind, "rows": rows, "position": position, "kv_heads": kv_heads, **_rope(**rope)}


def _attn_case(kind, name, prefix, decodes, own_lo, own_hi, **kw):
    c = {"name": name, "kind": kind, "call": "planned", "kv_heads": 2, "groups": 1, "prefix": prefix,
         "decodes": decodes, "own_lo": own_lo, "own_hi": own_hi, "chunks": 0, "chunk": 0, "loose": 0}
    if kind == "step":
        c.update(_rope())
    c.update(kw)
    return c


def _i8_case(name, tokens, hidden, out, form):
    return {"name": name, "kind": "i8", "tokens": tokens, "hidden": hidden, "out": out, "form": form}


def listed():
    return [
        # one decode iteration's rows at far positions: a launch
        _rows_case("rotate", "rotate-32", 32, 90000, layout="interleaved", rotary=64, scaling="bands", factor=8.0),
        # a 16k chunk's rows
        _rows_case("rotate", "rotate-16384", 16384, 8616, scaling="ramp", factor=4.0),
        # one decode row of each of 64 requests goes to its page
        _rows_case("append", "append-64", 64, 25000, scaling="linear", factor=2.0),
        # a 16k chunk goes to its pages, three quarters of each head rotated
        _rows_case("append", "append-16384", 16384, 8616, layout="interleaved", rotary=96),
        # a few requests with a short system prompt, by the call that plans for itself
        _attn_case("shared", "shared-8", 2048, 8, 30, 600, call="direct"),
        # a server's ordinary decode step: a long system prompt, own contexts of a conversation
        _attn_case("shared", "shared-64", 8192, 64, 100, 4000),
        # many continuations of one long document
        _attn_case("shared", "shared-256", 24576, 256, 16, 512),
        # two documents, their readers decoding and asking new questions, beside requests that share nothing
        _attn_case("step", "step-mixed", 16000, 20, 200, 2000, groups=2, chunks=1, chunk=700, loose=6, scaling="bands",
                   factor=4.0),
        # the MLP of a decode iteration: the weights are streamed for a few rows
        _i8_case("i8-act-24", 24, 2048, 11008, "act"),
        # the output projection of a ragged prompt tail
        _i8_case("i8-proj-700", 700, 2048, 2048, "proj"),
        # the down projection of a 2,048-token chunk with eight decode rows
        _i8_case("i8-proj-2056", 2056, 11008, 2048, "proj"),
        # the MLP's first half of a 16,384-token chunk
        _i8_case("i8-act-16384", 16384, 2048, 11008, "act"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges, never more work than the largest listed ones."""
    while True:
        kind = rng.choice(("rotate", "append", "shared", "shared", "step", "i8", "i8"))
        if kind == "i8":
            form = rng.choice(("act", "proj"))
            c = _i8_case("", _log(rng, 1, 16384), 128 * rng.choice((16, 86, 43, rng.randint(1, 86))),
                         rng.choice((11008, 5504, 2048, rng.randint(100, 11008))), form)
            ok = work(c)["flops"] <= 1.5e12
        else:
            scaling = rng.choice(("none", "linear", "base", "bands", "ramp"))
            layout = rng.choice(("half", "interleaved"))
            rope = _rope(layout, rng.choice((128, 96, 64, 32, 2 * rng.randint(1, 64))), scaling,
                         1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)))
            heads = rng.choice((2, 2, 1))
            if kind in ("rotate", "append"):
                c = _rows_case(kind, "", _log(rng, 1, 16384), rng.choice((0, rng.randint(1, 120000))), heads, **rope)
                ok = True
            else:
                hi = _log(rng, 16, 4000)
                c = _attn_case(kind, "", PAGE * _log(rng, 1, 2048), _log(rng, 1, 256), rng.randint(0, hi), hi,
                               groups=rng.choice((1, 1, 2, 4)), kv_heads=heads, loose=rng.choice((0, 0, 3, 17)))
                if rng.random() < 0.4:
                    c["chunks"], c["chunk"] = rng.choice((1, 2)), _log(rng, 2, 1024)
                if kind == "step":
                    c.update(rope)
                else:
                    c["call"] = rng.choice(("planned", "planned", "direct"))
                s = _seqs(c)
                most = c["prefix"] + c["own_hi"] + c["chunk"]
                ok = work(c)["flops"] <= 0.2e12 and len(s) * most <= 6.4e6 and \
                    c["groups"] * c["chunks"] * c["chunk"] * most <= 8e7
        if ok:
            del c["name"]
            return c


# ---------------------------------------------------------------------------
# What a case comes to
# ---------------------------------------------------------------------------

def _spread(lo, hi, i, n):
    return hi if n == 1 else lo + int((hi - lo) * ((i * GOLDEN) % 1.0))


def _seqs(case):
    """(group or -1, new tokens, cached tokens) of each request: each group's decode rows and chunks, then the loose
    decode rows."""
    out, lo, hi = [], case["own_lo"], case["own_hi"]
    for g in range(case["groups"]):
        n = case["decodes"]
        out += [(g, 1, case["prefix"] + _spread(lo, hi, i + 3 * g, n)) for i in range(n)]
        n = case["chunks"]
        out += [(g, case["chunk"], case["prefix"] + _spread(lo, hi, i + 1, n) // 2) for i in range(n)]
    n = case["loose"]
    return out + [(-1, 1, _spread(lo, hi, i, n)) for i in range(n)]


def work(case):
    kind = case["kind"]
    if kind == "i8":
        t, h, n = case["tokens"], case["hidden"], case["out"]
        wide = 2 * n if case["form"] == "act" else n
        return {"flops": 2.0 * t * h * wide, "bytes": 2.0 * t * h + h * wide + 4.0 * wide + 2.0 * t * n}
    g = case["kv_heads"]
    if kind in ("rotate", "append"):
        heads = (GROUP + (1 if kind == "rotate" else 2)) * g
        return {"flops": 3.0 * case["rows"] * (GROUP + 1) * g * case["rotary"],
                "bytes": 4.0 * DIM * heads * case["rows"]}
    seqs = _seqs(case)
    rows = sum(n for _, n, _ in seqs)
    pairs = sum(n * c + n * (n + 1) // 2 for _, n, c in seqs)
    keys = case["groups"] * case["prefix"] + sum(n + c - (case["prefix"] if k >= 0 else 0) for k, n, c in seqs)
    w = {"flops": 4.0 * DIM * GROUP * g * pairs, "bytes": 512.0 * g * (keys + GROUP * rows)}
    if kind == "step":
        w["bytes"] += 4.0 * DIM * (GROUP + 2) * g * rows
    return w


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _rand(g, *shape, scale=1.0):
    """Normal values rounded to bf16: hidden states, queries, keys and values after normalisation, or weights."""
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, scale, generator=g)


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "i8":
        wide = case["out"] * (2 if case["form"] == "act" else 1)
        s["x"] = _rand(g, case["tokens"], case["hidden"])
        # the weights as a program keeps them: quantised by channel once, when it loads them
        w = _rand(g, wide, case["hidden"], scale=0.02).float()
        top = w.abs().amax(1)
        s["w"] = (127.0 * w / top[:, None]).round().to(torch.int8)
        s["w_scale"] = top / 127.0
        return s
    hkv = case["kv_heads"]
    heads = (GROUP + 2) * hkv
    rng = np.random.Generator(np.random.PCG64(seed))
    if case["kind"] in ("rotate", "append"):
        rows, at = case["rows"], case["position"]
        if rows > 256:      # one chunk
            seqs = [(-1, rows, at)]
        else:               # one row of each request, a few positions apart
            seqs = [(-1, 1, _spread(at, at + 64, i, rows)) for i in range(rows)]
        prefix, groups = 0, 0
    else:
        seqs, prefix, groups = _seqs(case), case["prefix"], case["groups"]
        rows = sum(n for _, n, _ in seqs)
    qkv = _rand(g, rows, heads, DIM)
    s["q_new"], s["k_new"], s["v_new"] = qkv[:, :GROUP * hkv], qkv[:, GROUP * hkv:-hkv], qkv[:, -hkv:]
    pos = np.concatenate([c + np.arange(n) for _, n, c in seqs])
    if case["kind"] == "rotate":
        s["x"], s["positions"] = qkv[:, :-hkv], _dev(pos.astype(np.int32))
        return s
    # block tables: a group's prefix pages are the first entries of every member
    shared = prefix // PAGE
    need = [(n + c + PAGE - 1) // PAGE - (shared if k >= 0 else 0) for k, n, c in seqs]
    pages = groups * shared + sum(need)
    order = rng.permutation(pages).astype(np.int32)
    bt = np.full((len(seqs), max(m + (shared if k >= 0 else 0) for m, (k, _, _) in zip(need, seqs))), -1, np.int32)
    at = groups * shared
    for i, (m, (k, _, _)) in enumerate(zip(need, seqs)):
        first = 0
        if k >= 0:
            bt[i, :shared] = order[k * shared:(k + 1) * shared]
            first = shared
        bt[i, first:first + m] = order[at:at + m]
        at += m
    desc = np.zeros((len(seqs), 3), np.int32)
    desc[:, 1], desc[:, 2] = [n for _, n, _ in seqs], [c for _, _, c in seqs]
    desc[1:, 0] = np.cumsum(desc[:-1, 1])
    member = [k for k, _, _ in seqs]
    s["desc"], s["bt_host"], s["pages"], s["bt"] = desc, bt, pages, _dev(bt)
    s["prefixes"] = np.array([(member.index(k), member.count(k), prefix) for k in range(groups)],
                             np.int32).reshape(groups, 3)
    s["row_seq"], s["row_pos"] = _dev(np.repeat(np.arange(len(seqs)), desc[:, 1])), _dev(pos)
    s["k_pages"], s["v_pages"] = _rand(g, pages, hkv, DIM // 8, PAGE, 8), _rand(g, pages, hkv, DIM, PAGE)
    if case["kind"] == "append":
        return s
    if case["kind"] == "shared":
        s["q"] = s.pop("q_new").contiguous()
        del s["k_new"], s["v_new"]
    one = desc[:, 1] == 1
    s["parts"] = [(_dev(np.nonzero(m)[0]), n) for m, n in ((one, 1), (~one, case["chunk"])) if m.any()]
    s["starts"], s["cached"] = _dev(desc[:, 0].astype(np.int64)), _dev(desc[:, 2].astype(np.int64))
    return s


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------

def _frequencies(case, device):
    """Radians per position of each pair, in 64 bits, and the magnitude of the turned features."""
    r, f = case["rotary"], case["factor"]
    j = torch.arange(r // 2, dtype=torch.float64, device=device)
    base = THETA * f ** (r / (r - 2)) if case["scaling"] == "base" and r > 2 else THETA
    w = base ** (-2.0 * j / r)
    if case["scaling"] == "linear":
        return w / f, 1.0
    if case["scaling"] == "bands":
        turns = ORIGINAL * w / (2.0 * math.pi)
        keep = ((turns - BAND_LOW) / (BAND_HIGH - BAND_LOW)).clamp(0.0, 1.0)
        return w * (keep + (1.0 - keep) / f), 1.0
    if case["scaling"] == "ramp":
        lo, hi = (r * math.log(ORIGINAL / (2.0 * math.pi * b)) / (2.0 * math.log(THETA)) for b in (RAMP_FAST, RAMP_SLOW))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), r - 1)
        t = ((j - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return w * (1.0 - t + t / f), 0.1 * math.log(f) + 1.0
    return w, 1.0


def _turn(x, pos, case):
    """[rows, heads, 128] turned by the rows' positions: angles in 64 bits, the turn in 32, rounded once."""
    w, m = _frequencies(case, x.device)
    a = pos.double()[:, None] * w
    c, n = (a.cos() * m).float()[:, None], (a.sin() * m).float()[:, None]
    r = case["rotary"]
    u = x[..., :r].float()
    if case["layout"] == "half":
        p, q = u[..., :r // 2], u[..., r // 2:]
        t = torch.cat((p * c - q * n, q * c + p * n), -1)
    else:
        p, q = u[..., ::2], u[..., 1::2]
        t = torch.stack((p * c - q * n, q * c + p * n), -1).flatten(-2)
    return torch.cat((t.to(x.dtype), x[..., r:]), -1)


def _append(s):
    case, pos = s["case"], s["row_pos"]
    q, k = _turn(s["q_new"], pos, case), _turn(s["k_new"], pos, case)
    page, slot = s["bt"][s["row_seq"], pos // PAGE].long(), pos % PAGE
    s["k_pages"][page, :, :, slot] = k.unflatten(-1, (DIM // 8, 8))
    s["v_pages"][page, :, :, slot] = s["v_new"]
    return q


def _attend(s, q):
    """Every request's rows against its own table, the requests of one row count together: [requests, KV heads,
    rows x 8, keys] logits, their softmax, and its product with the values."""
    out = torch.empty_like(q)
    hkv = s["case"]["kv_heads"]
    for seq, n in s["parts"]:   # decode rows, then chunks
        rows = s["starts"][seq][:, None] + torch.arange(n, device=q.device)
        pos = s["cached"][seq][:, None] + torch.arange(n, device=q.device)
        top = s["case"]["prefix"] + s["case"]["own_hi"] + n
        ids = s["bt"][seq, :(top + PAGE - 1) // PAGE].clamp(min=0).long()
        k = s["k_pages"][ids].permute(0, 2, 3, 5, 1, 4).reshape(len(seq), hkv, DIM, -1).float()
        v = s["v_pages"][ids].permute(0, 2, 1, 4, 3).reshape(len(seq), hkv, -1, DIM).float()
        x = q[rows].unflatten(2, (hkv, GROUP)).permute(0, 2, 1, 3, 4).flatten(2, 3).float() / math.sqrt(DIM)
        p = torch.matmul(x, k).unflatten(2, (n, GROUP))
        hidden = torch.arange(k.shape[-1], device=q.device) > pos[:, None, :, None, None]
        p = p.masked_fill_(hidden, -math.inf).flatten(2, 3)
        p = torch.exp(p - p.amax(-1, keepdim=True))
        o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
        o = o.unflatten(2, (n, GROUP)).permute(0, 2, 1, 3, 4).flatten(2, 3)
        out[rows] = o.to(q.dtype)
    return out


def _quantise(x):
    x = x.float()
    top = x.abs().amax(1)
    return (127.0 * x / top[:, None]).round(), top / 127.0


def _product(s):
    x, sx = _quantise(s["x"])
    w = s["w"].float()
    y = torch.matmul(x, w.t()) * (sx[:, None] * s["w_scale"])
    if s["case"]["form"] == "act":
        g, u = y.chunk(2, 1)
        y = g / (1.0 + torch.exp(-g)) * u
    return {"y": y.to(torch.bfloat16)}


# ---------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------

def _lib():
    from paper_2608_15171_amd import ppas
    return ppas


def _lib_rope(s):
    c = s["case"]
    if "rope" not in s:
        s["rope"] = _lib().rope(layout=c["layout"], rotary_dim=c["rotary"], theta=THETA, scaling=c["scaling"],
                                factor=c["factor"], original_len=ORIGINAL,
                                low={"bands": BAND_LOW, "ramp": RAMP_SLOW}.get(c["scaling"], 0.0),
                                high={"bands": BAND_HIGH, "ramp": RAMP_FAST}.get(c["scaling"], 0.0),
                                magnitude=0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "ramp" else 1.0)
    return s["rope"]


def _kept(s, name, *shape, dtype=torch.bfloat16):
    """An output or workspace that the program keeps."""
    if name not in s:
        s[name] = torch.empty(shape, dtype=dtype, device="cuda")
    return s[name]


def _lib_plan(s):
    """The iteration's plan, made when its first layer runs and kept for the others."""
    if "plan" not in s:
        p = _lib()
        s["shape"] = p.make_shape(GROUP * s["case"]["kv_heads"], s["case"]["kv_heads"], s["pages"])
        s["plan"] = p.StepPlan(s["shape"], s["desc"], s["bt_host"], prefixes=s["prefixes"])
    return s["plan"]


def _lib_append(s):
    q = _kept(s, "q_out", *s["q_new"].shape)
    _lib_plan(s).rope_qkv_append(_lib_rope(s), q, s["k_pages"], s["v_pages"], s["q_new"], s["k_new"], s["v_new"],
                                 s["bt"])
    return q


def _lib_attend(s, q):
    out = _kept(s, "out", *q.shape)
    pools = s["k_pages"], s["v_pages"]
    if s["case"].get("call") == "direct":
        p, hkv = _lib(), s["case"]["kv_heads"]
        shape = p.make_shape(GROUP * hkv, hkv, s["pages"])
        if "ws" not in s:
            _kept(s, "ws", p.attn_shared_workspace_bytes(shape, s["desc"], s["prefixes"]), dtype=torch.uint8)
        p.attn_step_shared(shape, out, q, *pools, s["desc"], s["prefixes"], s["bt"], s["ws"], s["bt_host"])
    else:
        plan = _lib_plan(s)
        plan.attn_step(out, q, *pools, s["bt"], _kept(s, "ws", plan.workspace_bytes, dtype=torch.uint8))
    return out


def _lib_product(s):
    p, c = _lib(), s["case"]
    t, h = s["x"].shape
    act = c["form"] == "act"
    xq, sx = _kept(s, "xq", t, h, dtype=torch.int8), _kept(s, "sx", t, dtype=torch.float32)
    y = _kept(s, "y", t, c["out"])
    if "ws" not in s:
        size = p.gateup_act_i8_workspace_bytes if act else p.gateup_i8_workspace_bytes
        _kept(s, "ws", max(256, size(t, h, c["out"])), dtype=torch.uint8)
    p.quant_i8(s["x"], xq, sx)
    (p.gateup_act_i8 if act else p.gateup_proj_i8)(xq, sx, s["w"], s["w_scale"], y, s["ws"])
    return {"y": y}


def run(s):
    kind = s["case"]["kind"]
    if kind == "rotate":
        if own:
            y = _kept(s, "y", *s["x"].shape)
            _lib().rope_rows(_lib_rope(s), s["x"], s["positions"], y)
            return {"y": y}
        return {"y": _turn(s["x"], s["positions"], s["case"])}
    if kind == "i8":
        return _lib_product(s) if own else _product(s)
    r = {}
    q = s.get("q")
    if kind != "shared":
        q = _lib_append(s) if own else _append(s)
        r = {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if kind != "append":
        r["out"] = _lib_attend(s, q) if own else _attend(s, q)
    return r


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------

def _exact_turn(x, pos, case):
    """Pair by pair, as complex numbers."""
    r, f, kind = case["rotary"], case["factor"], case["scaling"]
    z = x[..., :r].double()
    z = torch.complex(z[..., :r // 2], z[..., r // 2:]) if case["layout"] == "half" else torch.view_as_complex(
        z.unflatten(-1, (r // 2, 2)).contiguous())
    base, size = THETA, 1.0
    if kind == "base" and r > 2:
        base = THETA * math.exp(math.log(f) * r / (r - 2))
    freq = []
    for j in range(r // 2):
        w = math.exp(-2.0 * j / r * math.log(base))
        if kind == "linear":
            w = w / f
        elif kind == "bands":
            length = 2.0 * math.pi / w
            if length > ORIGINAL / BAND_LOW:
                w = w / f
            elif length >= ORIGINAL / BAND_HIGH:
                mix = (ORIGINAL / length - BAND_LOW) / (BAND_HIGH - BAND_LOW)
                w = (1.0 - mix) * w / f + mix * w
        elif kind == "ramp":
            ends = [r / 2.0 * math.log(ORIGINAL / (b * 2.0 * math.pi), THETA) for b in (RAMP_FAST, RAMP_SLOW)]
            a, b = max(math.floor(ends[0]), 0), min(math.ceil(ends[1]), r - 1)
            mix = 0.0 if j <= a else 1.0 if j >= b else (j - a) / (b - a)
            w = mix * w / f + (1.0 - mix) * w
            size = 1.0 + math.log(f) / 10.0
        freq.append(w)
    a = pos.double()[:, None, None] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    z = z * torch.polar(torch.full_like(a, size), a)
    t = torch.cat((z.real, z.imag), -1) if case["layout"] == "half" else torch.view_as_real(z).flatten(-2)
    return torch.cat((t, x[..., r:].double()), -1)


def _exact_rows(s, q):
    """Request by request and head by head, over the keys that each row sees."""
    out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    for i, (at, n, c) in enumerate(s["desc"].tolist()):
        ids = s["bt"][i, :(n + c + PAGE - 1) // PAGE].long()
        for g in range(s["case"]["kv_heads"]):
            k = s["k_pages"][ids, g].permute(0, 2, 1, 3).reshape(-1, DIM)[:n + c].double()
            v = s["v_pages"][ids, g].transpose(1, 2).reshape(-1, DIM)[:n + c].double()
            for r in range(0, n, 256):
                m = min(256, n - r)
                x = q[at + r:at + r + m, GROUP * g:GROUP * (g + 1)].double()
                logit = torch.matmul(x, k.t()) / math.sqrt(DIM)
                seen = torch.arange(n + c, device=q.device)[None] <= torch.arange(c + r, c + r + m, device=q.device)[:, None]
                p = torch.softmax(torch.where(seen[:, None], logit, -math.inf), -1)
                out[at + r:at + r + m, GROUP * g:GROUP * (g + 1)] = torch.matmul(p, v)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotate":
        return {"y": _exact_turn(s["x"], s["positions"], case)}
    if kind == "i8":
        x = s["x"].double()
        top = x.abs().max(dim=1, keepdim=True).values
        xq, sx = torch.round(x * 127.0 / top), top / 127.0
        w, sw, out = s["w"].double(), s["w_scale"].double(), []
        for r in range(0, x.shape[0], 2048):
            y = torch.matmul(xq[r:r + 2048], w.t()) * sx[r:r + 2048] * sw
            if case["form"] == "act":
                n = case["out"]
                y = torch.nn.functional.silu(y[:, :n]) * y[:, n:]
            out.append(y)
        return {"y": torch.cat(out)}
    r, q = {}, s.get("q")
    if kind != "shared":
        q, k = _exact_turn(s["q_new"], s["row_pos"], case), _exact_turn(s["k_new"], s["row_pos"], case)
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        for i, (at, n, c) in enumerate(s["desc"].tolist()):
            p = torch.arange(c, c + n, device=q.device)
            ids, slot = s["bt"][i].long()[p // PAGE], p % PAGE
            kp[ids, :, :, slot] = k[at:at + n].reshape(n, -1, DIM // 8, 8)
            vp[ids, :, :, slot] = s["v_new"][at:at + n].double()
        r = {"q": q, "k_pages": kp, "v_pages": vp}
        # what the cache and the query buffer hold is bf16
        s["k_pages"], s["v_pages"], q = kp.bfloat16(), vp.bfloat16(), q.bfloat16()
    if kind != "append":
        r["out"] = _exact_rows(s, q)
    return r
