"""Timed cases of the operators that a served, fine-tuned model adds to a decoder layer's step: norms of query and key
heads in the pass that turns them and writes the pages, low-rank adapters of many requests beside a shared projection,
and the log probabilities that a request is answered with.

Shapes are those of the repository's workloads (16 query and 2 KV heads of 128 features, or the two-way shard's 8 and
1; pages of 16 tokens; hidden 2048 and 11008 intermediate features, or the shard's 5504). Every case has a kind:
  rows    heads of a step's rows, normalised and turned by their positions
  append  a step's QKV rows: queries to their buffer, keys and values to the pages, queries and keys normalised and
          turned on the way
  add     the adapters' share added to a projection's output, rows of one adapter wherever they lie; the program keeps
          the rows' order for the projections of an iteration ("kept"), or makes it for this one ("each")
  act     the same before a gated activation of the two halves
  logp    logit rows: the given tokens' log probabilities and ranks, the rows' entropy, the top alternatives
`run` computes them in plain torch, or where `own` is true by the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE, DIM, GROUP = 16, 128, 8
THETA, EPS = 1e6, 1e-6
# frequency scaling: the length that positions were learned over, the ramp's ends in rotations over it
ORIGINAL, RAMP_FAST, RAMP_SLOW = 8192, 32.0, 1.0
GOLDEN = 0.6180339887498949


def _head(layout="half", rotary=DIM, scaling="none", factor=1.0, center=False, offset=0.0):
    return {"layout": layout, "rotary": rotary, "scaling": scaling, "factor": factor, "center": center, "offset": offset}


def _rows_case(name, rows, position, heads=18, dim=DIM, **kw):
    return {"name": name, "kind": "rows", "rows": rows, "position": position, "heads": heads, "dim": dim, **_head(**kw)}


def _append_case(name, chunk, decodes, cached, kv_heads=2, **kw):
    return {"name": name, "kind": "append", "chunk": chunk, "decodes": decodes, "cached": cached, "kv_heads": kv_heads,
            **_head(**kw)}


def _adapter_case(name, kind, hidden, out, rank, adapters, chunks, chunk, decodes, loose=0, call="kept"):
    """`chunks` requests of `chunk` rows, `decodes` of one row, `loose` decode rows without an adapter."""
    return {"name": name, "kind": kind, "hidden": hidden, "out": out, "rank": rank, "adapters": adapters,
            "chunks": chunks, "chunk": chunk, "decodes": decodes, "loose": loose, "call": call}


def _logp_case(name, rows, vocab, top, dtype="bf16", keep=1.0, scale=1.0, pad=0):
    """`keep`: the share of tokens that a grammar leaves; `pad`: elements between rows."""
    return {"name": name, "kind": "logp", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "keep": keep,
            "scale": scale, "pad": pad}


def listed():
    return [
        # one decode iteration's query and key heads at far positions, each head with weights of its own: a launch
        _rows_case("norm-rows-32", 32, 90000, layout="interleaved", rotary=64, center=True),
        # one decode row of each of 64 requests goes to its page
        _append_case("norm-append-64", 0, 64, 25000, scaling="linear", factor=2.0),
        # a 16k chunk goes to its pages, the norms' weights held as differences from one
        _append_case("norm-append-16384", 16384, 0, 8616, scaling="ramp", factor=4.0, offset=1.0),
        # a single request decodes with its adapter on the attention's output projection
        _adapter_case("adapter-add-1", "add", 2048, 2048, 16, 8, 0, 0, 1, call="each"),
        # a decode iteration of many customers' adapters, some requests on the plain model: the gate and up projections
        _adapter_case("adapter-add-64", "add", 2048, 22016, 16, 24, 0, 0, 56, loose=8),
        # ragged prompt tails beside decode rows on the down projection
        _adapter_case("adapter-add-700", "add", 11008, 2048, 8, 12, 5, 137, 15),
        # the MLP's first half of a 2,048-token chunk with eight decode rows
        _adapter_case("adapter-act-2056", "act", 2048, 11008, 32, 6, 1, 2048, 8),
        # the gate and up projections of a 16,384-token chunk
        _adapter_case("adapter-add-16384", "add", 2048, 22016, 64, 4, 1, 16384, 0),
        # one sampled token and its alternatives
        _logp_case("logp-1", 1, 131072, 20),
        # an iteration's decode rows under a grammar, an odd vocabulary, rows behind one another with a gap
        _logp_case("logp-48-masked", 48, 100003, 5, keep=0.02, scale=1.25, pad=5),
        # an iteration's decode rows in fp32
        _logp_case("logp-64-fp32", 64, 131072, 20, dtype="fp32"),
        # a 2,048-token chunk's prompt log probabilities
        _logp_case("logp-2048", 2048, 131072, 5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges, never more work than the largest listed ones."""
    while True:
        kind = rng.choice(("rows", "append", "add", "add", "act", "logp", "logp"))
        if kind in ("rows", "append"):
            dim = DIM if kind == "append" else rng.choice((128, 128, 64, 256, 2 * rng.randint(4, 128)))
            scaling = rng.choice(("none", "linear", "ramp"))
            kw = _head(rng.choice(("half", "interleaved")), rng.choice((dim, dim, dim // 4 * 2, 2 * rng.randint(1, dim // 2))),
                       scaling, 1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0)), rng.random() < 0.3,
                       rng.choice((0.0, 1.0)))
            at = rng.choice((0, rng.randint(1, 120000)))
            if kind == "rows":
                c = _rows_case("", _log(rng, 1, 16384), at, rng.choice((18, 9, 16, 2, rng.randint(1, 40))), dim, **kw)
                ok = c["rows"] * c["heads"] * dim <= 4e7
            else:
                c = _append_case("", rng.choice((0, _log(rng, 2, 16384))), rng.choice((0, _log(rng, 1, 256))), at,
                                 rng.choice((2, 2, 1)), **kw)
                ok = 0 < c["chunk"] + c["decodes"] <= 16384
        elif kind == "logp":
            c = _logp_case("", _log(rng, 1, 2048), _log(rng, 1000, 262144), rng.choice((0, 1, 5, 20, rng.randint(1, 32))),
                           rng.choice(("bf16", "bf16", "fp32")), rng.choice((1.0, 1.0, 0.5, 0.01)),
                           rng.choice((1.0, 0.5, 1.25, rng.uniform(0.3, 3.0))), rng.choice((0, 0, rng.randint(1, 64))))
            ok = work(c)["bytes"] <= 5.4e8
        else:
            chunks = rng.choice((0, 1, 1, 2, 5))
            c = _adapter_case("", kind, 64 * rng.choice((32, 172, 86, rng.randint(1, 172))),
                              rng.choice((2048, 2560, 5504, 11008, rng.randint(100, 11008))) * (2 if kind == "add" and
                                                                                               rng.random() < 0.3 else 1),
                              rng.choice((8, 16, 32, 64, 128, rng.randint(1, 128))), _log(rng, 1, 64), chunks,
                              _log(rng, 2, 16384) if chunks else 0, rng.choice((0, _log(rng, 1, 256))),
                              rng.choice((0, 0, 3, 17)), rng.choice(("kept", "kept", "each")))
            t = _tokens(c)
            ok = 0 < t <= 16384 and t * c["rank"] * c["adapters"] <= 1.4e8 and work(c)["bytes"] <= 1.5e9
        if ok:
            del c["name"]
            return c


# ---------------------------------------------------------------------------
# What a case comes to
# ---------------------------------------------------------------------------

def _requests(case):
    """(rows, adapter or -1) of each request of an adapters' case: decode rows with and without one, in turn, between
    the chunks."""
    n, out = case["adapters"], []
    for i in range(case["chunks"]):
        out.append((case["chunk"], int(i * GOLDEN % 1.0 * n)))
    for i in range(max(case["decodes"], case["loose"])):
        if i < case["decodes"]:
            out.append((1, int((i + 3) * GOLDEN % 1.0 * n)))
        if i < case["loose"]:
            out.append((1, -1))
    return out


def _tokens(case):
    return case["chunks"] * case["chunk"] + case["decodes"] + case["loose"]


def _seqs(case):
    """(new tokens, cached tokens) of each request of a step: the chunk, then decode rows a few positions apart."""
    out = [(case["chunk"], case["cached"])] if case["chunk"] else []
    return out + [(1, case["cached"] + int(i * GOLDEN % 1.0 * 64)) for i in range(case["decodes"])]


def work(case):
    kind = case["kind"]
    if kind == "rows":
        n = float(case["rows"]) * case["heads"]
        return {"flops": n * (6.0 * case["dim"] + 3.0 * case["rotary"]), "bytes": 4.0 * n * case["dim"]}
    if kind == "append":
        n, g = float(case["chunk"] + case["decodes"]), case["kv_heads"]
        return {"flops": n * (GROUP + 1) * g * (6.0 * DIM + 3.0 * case["rotary"]), "bytes": 4.0 * DIM * (GROUP + 2) * g * n}
    if kind == "logp":
        n = float(case["rows"]) * case["vocab"]
        return {"flops": 10.0 * n, "bytes": n * (2 if case["dtype"] == "bf16" else 4) + 8.0 * case["rows"] * (2 + case["top"])}
    t, r, h = float(_tokens(case)), case["rank"], case["hidden"]
    wide = case["out"] * (2 if kind == "act" else 1)
    used = len({a for _, a in _requests(case) if a >= 0})
    with_one = t - case["loose"]
    return {"flops": 2.0 * with_one * r * (h + wide), "bytes": 2.0 * with_one * h + 2.0 * used * r * (h + wide) +
            2.0 * t * (wide + case["out"])}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _rand(g, *shape, scale=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=g)


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _norm_weight(g, case, *shape):
    """Weights near one, or their differences from it where the model adds it."""
    return (_rand(g, *shape, scale=0.1).float() + (1.0 - case["offset"])).bfloat16()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.Generator(np.random.PCG64(seed))
    s = {"case": case}
    kind = case["kind"]
    if kind == "rows":
        n, at = case["rows"], case["position"]
        pos = at + np.arange(n) if n > 256 else at + (np.arange(n) * GOLDEN % 1.0 * 64).astype(np.int64)
        s["positions"] = _dev(pos.astype(np.int32))
        s["x"] = _rand(g, n, case["heads"], case["dim"], scale=2.0)
        s["w"] = _norm_weight(g, case, case["heads"], case["dim"])
    elif kind == "append":
        hkv, seqs = case["kv_heads"], _seqs(case)
        rows = sum(n for n, _ in seqs)
        qkv = _rand(g, rows, (GROUP + 2) * hkv, DIM, scale=2.0)
        s["q_new"], s["k_new"], s["v_new"] = qkv[:, :GROUP * hkv], qkv[:, GROUP * hkv:-hkv], qkv[:, -hkv:]
        s["q_w"], s["k_w"] = _norm_weight(g, case, DIM), _norm_weight(g, case, DIM)
        need = [(n + c + PAGE - 1) // PAGE for n, c in seqs]
        order = rng.permutation(sum(need)).astype(np.int32)
        bt = np.full((len(seqs), max(need)), -1, np.int32)
        for i, m in enumerate(need):
            bt[i, :m], order = order[:m], order[m:]
        desc = np.zeros((len(seqs), 3), np.int32)
        desc[:, 1], desc[:, 2] = [n for n, _ in seqs], [c for _, c in seqs]
        desc[1:, 0] = np.cumsum(desc[:-1, 1])
        s["desc"], s["bt_host"], s["bt"], s["pages"] = desc, bt, _dev(bt), sum(need)
        s["row_seq"] = _dev(np.repeat(np.arange(len(seqs)), desc[:, 1]))
        s["row_pos"] = _dev(np.concatenate([c + np.arange(n) for n, c in seqs]))
        s["k_pages"] = _rand(g, s["pages"], hkv, DIM // 8, PAGE, 8)
        s["v_pages"] = _rand(g, s["pages"], hkv, DIM, PAGE)
    elif kind == "logp":
        rows, vocab = case["rows"], case["vocab"]
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        x = torch.empty((rows, vocab + case["pad"]), dtype=dtype, device="cuda").normal_(0.0, 2.5, generator=g)[:, :vocab]
        tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
        # most given tokens are likely ones
        at = torch.arange(rows, device="cuda")
        x[at, tokens] += 12.0 * torch.rand(rows, device="cuda", generator=g).to(dtype)
        if case["keep"] < 1.0:
            keep = torch.rand((rows, vocab), device="cuda", generator=g) < case["keep"]
            keep[at, tokens] = True
            x.masked_fill_(~keep, -math.inf)
        s["logits"], s["tokens"] = x, tokens.to(torch.int32)
    else:
        t, h, r, n = _tokens(case), case["hidden"], case["rank"], case["adapters"]
        wide = case["out"] * (2 if kind == "act" else 1)
        reqs = [_requests(case)[i] for i in rng.permutation(len(_requests(case)))]
        s["row_adapter"] = _dev(np.repeat([a for _, a in reqs], [m for m, _ in reqs]).astype(np.int32))
        s["x"], s["y"] = _rand(g, t, h), _rand(g, t, wide)
        s["a"], s["b"] = _rand(g, n, r, h, scale=h ** -0.5), _rand(g, n, wide, r, scale=0.5 * r ** -0.5)
        s["scale"] = 0.5 + 1.5 * torch.rand(n, device="cuda", generator=g)
    return s


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------

def _frequencies(case, device):
    """Radians per position of each pair, in 64 bits, and the magnitude of the turned features."""
    r, f = case["rotary"], case["factor"]
    j = torch.arange(r // 2, dtype=torch.float64, device=device)
    w = THETA ** (-2.0 * j / r)
    if case["scaling"] == "linear":
        return w / f, 1.0
    if case["scaling"] == "ramp":
        lo, hi = (r * math.log(ORIGINAL / (2.0 * math.pi * b)) / (2.0 * math.log(THETA)) for b in (RAMP_FAST, RAMP_SLOW))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), r - 1)
        t = ((j - lo) / (hi - lo)).clamp(0.0, 1.0) if hi > lo else (j > lo).double()
        return w * (1.0 - t + t / f), 0.1 * math.log(f) + 1.0
    return w, 1.0


def _norm_turn(x, weight, pos, case):
    """[rows, heads, features] normalised by head and turned by the rows' positions: statistics, norm and turn in 32
    bits, angles in 64, rounded once."""
    u = x.float()
    if case["center"]:
        u = u - u.mean(-1, keepdim=True)
    u = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + EPS) * (weight.float() + case["offset"])
    w, m = _frequencies(case, x.device)
    a = pos.double()[:, None] * w
    c, n = (a.cos() * m).float()[:, None], (a.sin() * m).float()[:, None]
    r = case["rotary"]
    if case["layout"] == "half":
        p, q = u[..., :r // 2], u[..., r // 2:r]
        t = torch.cat((p * c - q * n, q * c + p * n), -1)
    else:
        p, q = u[..., :r:2], u[..., 1:r:2]
        t = torch.stack((p * c - q * n, q * c + p * n), -1).flatten(-2)
    return torch.cat((t, u[..., r:]), -1).to(x.dtype)


def _append(s):
    case, pos = s["case"], s["row_pos"]
    q, k = _norm_turn(s["q_new"], s["q_w"], pos, case), _norm_turn(s["k_new"], s["k_w"], pos, case)
    page, slot = s["bt"][s["row_seq"], pos // PAGE].long(), pos % PAGE
    s["k_pages"][page, :, :, slot] = k.unflatten(-1, (DIM // 8, 8))
    s["v_pages"][page, :, :, slot] = s["v_new"]
    return q


def _adapt(s):
    """All adapters side by side, [rows, adapters x rank], and a row's own of them."""
    n, r, h = s["a"].shape
    v = torch.matmul(s["x"].float(), s["a"].float().view(n * r, h).t()).view(-1, n, r)
    own_one = s["row_adapter"][:, None] == torch.arange(n, device=v.device)
    v = v * (own_one * s["scale"])[:, :, None]
    y = s["y"].float() + torch.matmul(v.view(-1, n * r), s["b"].float().transpose(1, 2).reshape(n * r, -1))
    if s["case"]["kind"] == "act":
        g, u = y.chunk(2, 1)
        y = g / (1.0 + torch.exp(-g)) * u
    return {"out": y.to(torch.bfloat16)}


def _logp(s):
    """In 64 bits (sums over a vocabulary), the order by a stable sort of the logits themselves."""
    x, t = s["logits"], s["tokens"].long()[:, None]
    k = s["case"]["top"]
    z = x.double() * s["case"]["scale"]
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    lse = torch.log(total)
    mean = (e * z.masked_fill(e == 0.0, 0.0)).sum(1, keepdim=True) / total
    at = x.gather(1, t)
    before = (x > at) | ((x == at) & (torch.arange(x.shape[1], device=x.device) < t))
    out = {"logprob": (z.gather(1, t) - lse)[:, 0].float(), "rank": before.sum(1).to(torch.int32),
           "entropy": (lse - mean)[:, 0].float()}
    if k:
        first, ids = torch.sort(x, dim=1, descending=True, stable=True)
        ids = ids[:, :k]
        top = z.gather(1, ids) - lse
        out["top_ids"] = ids.masked_fill(first[:, :k] == -math.inf, -1).to(torch.int32)
        out["top_logprobs"] = top.float()
    return out


# ---------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------

def _lib():
    from paper_2608_15171_amd import ppas
    return ppas


def _kept(s, name, *shape, dtype=torch.bfloat16):
    """An output or workspace that the program keeps."""
    if name not in s:
        s[name] = torch.empty(shape, dtype=dtype, device="cuda")
    return s[name]


def _lib_rope(s):
    c = s["case"]
    if "rope" not in s:
        ramp = c["scaling"] == "ramp"
        s["rope"] = _lib().rope(layout=c["layout"], rotary_dim=c["rotary"], theta=THETA, scaling=c["scaling"],
                                factor=c["factor"], original_len=ORIGINAL, low=RAMP_SLOW if ramp else 0.0,
                                high=RAMP_FAST if ramp else 0.0,
                                magnitude=0.1 * math.log(c["factor"]) + 1.0 if ramp else 1.0)
    return s["rope"]


def _lib_norm(s, weight):
    key = "norm_" + weight
    if key not in s:
        s[key] = _lib().head_norm(s[weight], eps=EPS, offset=s["case"]["offset"], center=s["case"]["center"])
    return s[key]


def _lib_rows(s):
    y = _kept(s, "y", *s["x"].shape)
    _lib().norm_rope_rows(_lib_norm(s, "w"), _lib_rope(s), s["x"], s["positions"], y)
    return {"y": y}


def _lib_append(s):
    q = _kept(s, "q_out", *s["q_new"].shape)
    if "plan" not in s:   # the iteration's plan, made when its first layer runs and kept for the others
        p, hkv = _lib(), s["case"]["kv_heads"]
        s["plan"] = p.StepPlan(p.make_shape(GROUP * hkv, hkv, s["pages"]), s["desc"], s["bt_host"])
    s["plan"].norm_rope_qkv_append(_lib_norm(s, "q_w"), _lib_norm(s, "k_w"), _lib_rope(s), q, s["k_pages"], s["v_pages"],
                                   s["q_new"], s["k_new"], s["v_new"], s["bt"])
    return q


def _lib_adapt(s):
    p, c = _lib(), s["case"]
    if "order" not in s:   # the iteration's rows by adapter, and the layer's weights
        s["order"] = p.AdapterRows(s["x"].shape[0], c["adapters"])
        s["set"] = p.adapters(s["a"], s["b"], s["scale"])
        _kept(s, "ws", max(256, p.adapter_workspace_bytes(s["x"].shape[0], c["hidden"], c["rank"], c["adapters"])),
              dtype=torch.uint8)
        if c["call"] == "kept":
            s["order"].sort(s["row_adapter"])
    if c["call"] == "each":
        s["order"].sort(s["row_adapter"])
    out = _kept(s, "out", s["x"].shape[0], c["out"])
    (p.adapter_act if c["kind"] == "act" else p.adapter_add)(s["set"], s["x"], s["y"], out, s["order"], s["ws"])
    return {"out": out}


def _lib_logp(s):
    p, c = _lib(), s["case"]
    n, k = c["rows"], c["top"]
    f, i = torch.float32, torch.int32
    out = {"logprob": _kept(s, "logprob", n, dtype=f), "rank": _kept(s, "rank", n, dtype=i),
           "entropy": _kept(s, "entropy", n, dtype=f)}
    if k:
        out["top_ids"], out["top_logprobs"] = _kept(s, "ids", n, k, dtype=i), _kept(s, "top", n, k, dtype=f)
    if "ws" not in s:
        _kept(s, "ws", max(256, p.logprobs_workspace_bytes(n, c["vocab"], k)), dtype=torch.uint8)
    p.logprobs(s["logits"], tokens=s["tokens"], scale=c["scale"], workspace=s["ws"], **out)
    return out


def run(s):
    kind = s["case"]["kind"]
    if kind == "rows":
        return _lib_rows(s) if own else {"y": _norm_turn(s["x"], s["w"], s["positions"], s["case"])}
    if kind == "append":
        q = _lib_append(s) if own else _append(s)
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if kind == "logp":
        return _lib_logp(s) if own else _logp(s)
    return _lib_adapt(s) if own else _adapt(s)


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------

def _exact_turn(x, weight, pos, case):
    """The norm by its mean and variance, then pair by pair, as complex numbers."""
    x, r, f, kind = x.double(), case["rotary"], case["factor"], case["scaling"]
    var, mu = torch.var_mean(x, -1, unbiased=False, keepdim=True)
    if not case["center"]:
        var, mu = var + mu * mu, torch.zeros_like(mu)
    x = (x - mu) / (var + EPS).sqrt() * (weight.double() + case["offset"])
    freq, size = [], 1.0
    for j in range(r // 2):
        w = math.exp(-2.0 * j / r * math.log(THETA))
        if kind == "linear":
            w = w / f
        elif kind == "ramp":
            ends = [r / 2.0 * math.log(ORIGINAL / (b * 2.0 * math.pi), THETA) for b in (RAMP_FAST, RAMP_SLOW)]
            a, b = max(math.floor(ends[0]), 0), min(math.ceil(ends[1]), r - 1)
            mix = 0.0 if j <= a else 1.0 if j >= b else (j - a) / (b - a)
            w = mix * w / f + (1.0 - mix) * w
            size = 1.0 + math.log(f) / 10.0
        freq.append(w)
    z = x[..., :r]
    z = torch.complex(z[..., :r // 2], z[..., r // 2:]) if case["layout"] == "half" else torch.view_as_complex(
        z.unflatten(-1, (r // 2, 2)).contiguous())
    a = pos.double()[:, None, None] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    z = z * torch.polar(torch.full_like(a, size), a)
    t = torch.cat((z.real, z.imag), -1) if case["layout"] == "half" else torch.view_as_real(z).flatten(-2)
    return torch.cat((t, x[..., r:]), -1)


def _exact_append(s, case):
    q = _exact_turn(s["q_new"], s["q_w"], s["row_pos"], case)
    k = _exact_turn(s["k_new"], s["k_w"], s["row_pos"], case)
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    for i, (at, n, c) in enumerate(s["desc"].tolist()):
        p = torch.arange(c, c + n, device=q.device)
        ids, slot = s["bt"][i].long()[p // PAGE], p % PAGE
        kp[ids, :, :, slot] = k[at:at + n].reshape(n, -1, DIM // 8, 8)
        vp[ids, :, :, slot] = s["v_new"][at:at + n].double()
    return {"q": q, "k_pages": kp, "v_pages": vp}


def _exact_adapt(s, case):
    """Adapter by adapter, over the rows that have it."""
    y = s["y"].double()
    for a in range(case["adapters"]):
        rows = (s["row_adapter"] == a).nonzero()[:, 0]
        v = torch.matmul(s["x"][rows].double(), s["a"][a].double().t()) * s["scale"][a].double()
        y[rows] += torch.matmul(v, s["b"][a].double().t())
    if case["kind"] == "act":
        n = case["out"]
        y = torch.nn.functional.silu(y[:, :n]) * y[:, n:]
    return {"out": y}


def _exact_logp(s, case):
    """Some rows at a time, by the library's own log-softmax and entropy in 64 bits."""
    got = {"logprob": [], "entropy": [], "top_logprobs": []}
    for r in range(0, case["rows"], 256):
        x = s["logits"][r:r + 256].double() * case["scale"]
        lp = torch.log_softmax(x, 1)
        got["logprob"].append(lp.gather(1, s["tokens"][r:r + 256, None].long())[:, 0])
        got["entropy"].append(torch.special.entr(lp.exp()).sum(1))
        if case["top"]:
            got["top_logprobs"].append(lp.topk(case["top"], 1).values)
    out = {k: torch.cat(v) for k, v in got.items() if v}
    out["rank"] = None
    if case["top"]:
        out["top_ids"] = None
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rows":
        return {"y": _exact_turn(s["x"], s["w"], s["positions"], case)}
    if kind == "append":
        return _exact_append(s, case)
    return _exact_logp(s, case) if kind == "logp" else _exact_adapt(s, case)
