"""Log probabilities on the CPU: every refusal."""
import ctypes

import pytest
import torch

ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")

E, U, R, OK = ppas.PPAS_EINVAL, ppas.PPAS_EUNSUPPORTED, ppas.PPAS_ERANGE, ppas.PPAS_OK
P = 1 << 20
ALL = ppas.LogprobOut(P, P, P, P, P)


def call(out=ALL, **kw):
    a = dict(logits=1 << 24, type=0, stride=1000, rows=4, vocab=1000, scale=1.0, tokens=P, top=5, ws=None, ws_bytes=0, ev=None)
    a.update(kw)
    return ppas._lib.ppas_logprobs(a["logits"], a["type"], a["stride"], a["rows"], a["vocab"], a["scale"], a["tokens"], a["top"],
                                   None if out is None else ctypes.byref(out), a["ws"], a["ws_bytes"], a["ev"], None)


def test_refusals():
    half = ppas.events(start=1)
    for kw in (dict(logits=None), dict(type=2), dict(type=-1), dict(stride=999), dict(stride=-1000), dict(rows=-1), dict(vocab=0),
               dict(vocab=-3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(scale=2.0 ** -101), dict(scale=2.0 ** 101), dict(tokens=None), dict(top=-1), dict(ws_bytes=64), dict(ws=P + 8),
               dict(ev=ctypes.byref(half)), dict(logits=(1 << 24) + 1), dict(logits=(1 << 24) + 2, type=1), dict(tokens=P + 2),
               dict(out=None), dict(type=1, out=ppas.LogprobOut(None, None, (1 << 24) + 4 * 3999)),
               dict(out=ppas.LogprobOut(P, P, P, P, (1 << 24) - 4)), *(dict(out=ppas.LogprobOut(*[P + 2 * (i == j) for j in range(5)])) for i in range(5))):
        assert call(**kw) == E, kw
    assert call(top=65) == U
    assert call(vocab=(1 << 30) + 1, stride=1 << 31) == R
    assert call(stride=1 << 59) == R


def test_nothing_to_do():
    assert call(rows=0, logits=None, out=None) == OK
    assert call(out=ppas.LogprobOut()) == OK                                   # nothing is asked for
    assert call(out=ppas.LogprobOut(None, None, None, P, P), top=0, tokens=None) == OK
    assert call(rows=0, scale=0.0) == E


def test_workspace():
    f = ppas.logprobs_workspace_bytes
    assert f(0, 1000) == 0 and f(-1, 1000) == 0 and f(4, 0) == 0 and f(4, 1000, 65) == 0 and f(4, (1 << 30) + 1) == 0
    assert f(1, 1000) == 0 and f(4096, 131072) == 0                            # too short, or rows enough, to be split
    # parts of 1,024 vectors, of fp32 logits here: half as many tokens
    assert f(1, 131072, 0) == 32 * 16 and f(1, 131072, 20) == 32 * (16 + 160) and f(1, 1 << 30, 1) == 64 * 24
    assert f(64, 131072, 5) % 64 == 0 and f(64, 131072, 5) > 0


def test_binding_types():
    t = torch.zeros
    x = t((4, 100), dtype=torch.bfloat16)
    bad = [dict(logits=t((4, 100), dtype=torch.float16)), dict(logits=t(100)), dict(logits=t((4, 200))[:, ::2]),
           dict(tokens=t(4, dtype=torch.int64)), dict(tokens=t(3, dtype=torch.int32)), dict(logprob=t(4, dtype=torch.float64)),
           dict(logprob=t(5)), dict(rank=t(4)), dict(entropy=t((4, 1))), dict(top_ids=t((4, 3), dtype=torch.int64)),
           dict(top_ids=t((3, 3), dtype=torch.int32)), dict(top_logprobs=t((4, 3, 1))),
           dict(top_ids=t((4, 3), dtype=torch.int32), top_logprobs=t((4, 4)))]
    old = ppas._dev
    ppas._dev = lambda v, name: 0
    try:
        for kw in bad:
            with pytest.raises(ValueError, match="must be"):
                ppas.logprobs(**{"logits": x, **kw})
    finally:
        ppas._dev = old
    with pytest.raises(ValueError, match="device tensor"):
        ppas.logprobs(x, entropy=t(4))
