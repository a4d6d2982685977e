"""Adapters on the CPU: every refusal, and sizes."""
import ctypes

import pytest
import torch

ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")

E, U, R, N, OK = ppas.PPAS_EINVAL, ppas.PPAS_EUNSUPPORTED, ppas.PPAS_ERANGE, ppas.PPAS_ENOSPACE, ppas.PPAS_OK
P = 1 << 20


def make(a=P, b=P, scale=P, n=4, rank=16, hidden=128, out=256):
    return ppas.Adapters(a, b, scale, n, rank, hidden, out)


def call(act=False, adapters=None, **kw):
    s = make() if adapters is None else adapters
    a = dict(x=1 << 24, xs=128, y=1 << 26, ys=256, out=1 << 28, os=256, tokens=8, rows=1 << 21, rows_bytes=1 << 20, ws=1 << 22,
             ws_bytes=1 << 30, ev=None)
    a.update(kw)
    f = ppas._lib.ppas_adapter_act if act else ppas._lib.ppas_adapter_add
    return f(None if s is False else ctypes.byref(s), a["x"], a["xs"], a["y"], a["ys"], a["out"], a["os"], a["tokens"], a["rows"],
             a["rows_bytes"], a["ws"], a["ws_bytes"], a["ev"], None)


@pytest.mark.parametrize("act", [False, True])
def test_refusals(act):
    half = ppas.events(start=1)
    for kw in (dict(adapters=False), dict(adapters=make(a=None)), dict(adapters=make(b=None)), dict(adapters=make(a=P + 1)),
               dict(adapters=make(b=P + 1)), dict(adapters=make(scale=P + 2)), dict(adapters=make(n=0)), dict(adapters=make(n=-1)),
               dict(adapters=make(rank=0)), dict(adapters=make(hidden=0)), dict(adapters=make(out=0)), dict(tokens=-1), dict(x=None),
               dict(y=None), dict(out=None), dict(rows=None), dict(ws=None), dict(xs=127), dict(ys=255), dict(ys=-256), dict(os=127),
               dict(x=(1 << 24) + 1), dict(y=(1 << 26) + 1), dict(out=(1 << 28) + 1), dict(rows=(1 << 21) + 8),
               dict(ws=(1 << 22) + 8), dict(ev=ctypes.byref(half)),
               # results over the inputs
               dict(out=(1 << 26) + 2), dict(out=1 << 26, os=300), dict(out=1 << 24), dict(out=(1 << 24) + 2 * (7 * 128 + 127)),
               dict(y=(1 << 28) + 2 * 7 * 256)):
        assert call(act, **kw) == E, kw
    assert call(act, adapters=make(n=1025)) == U and call(act, adapters=make(rank=129)) == U
    assert call(act, tokens=(1 << 24) + 1) == R and call(act, xs=1 << 60) == R and call(act, os=1 << 60) == R
    assert call(act, adapters=make(hidden=2 ** 31 - 1), xs=1 << 31) == R
    assert call(act, tokens=0, x=None, y=None, out=None, rows=None, ws=None) == OK
    assert call(act, tokens=0, adapters=make(rank=0)) == E
    assert call(act, rows_bytes=ppas._lib.ppas_adapter_rows_bytes(8, 4) - 1) == N


@pytest.mark.parametrize("act", [False, True])
def test_results_and_workspace_over_what_is_read(act):
    """The set at P (a of 16,384 bytes, b of 32,768, four scales), its order, and the workspace's one split of 512 bytes at least."""
    rows, ws, x, y, out = 1 << 21, 1 << 22, 1 << 24, 1 << 26, 1 << 28
    order = ppas._lib.ppas_adapter_rows_bytes(8, 4)
    far = 1 << 30
    for kw in (dict(out=P), dict(out=P + 32766), dict(adapters=make(b=far, scale=far), out=P + 16382),
               dict(adapters=make(a=far, b=far), out=P + 14), dict(out=P - 2), dict(out=rows), dict(out=rows + (order - 1) // 2 * 2),
               dict(out=ws), dict(out=ws + 510), dict(ws=P), dict(ws=P + 32752), dict(ws=rows), dict(ws=x), dict(ws=x + 2 * 1008),
               dict(ws=x - 496), dict(ws=y + 2 * 2032), dict(ws=out), dict(rows=ws)):
        assert call(act, **kw) == E, kw
    f = ppas._lib.ppas_adapter_rows
    assert f(rows, 8, 4, rows, 1 << 20, None, None) == E and f(rows + order - 4, 8, 4, rows, 1 << 20, None, None) == E
    assert f(rows - 28, 8, 4, rows, 1 << 20, None, None) == E


def test_only_the_activation_needs_halves():
    assert call(True, adapters=make(out=255)) == E
    # in place is for the sum
    assert call(True, out=1 << 26) == E


def test_rows_refusals():
    f, size = ppas._lib.ppas_adapter_rows, ppas._lib.ppas_adapter_rows_bytes
    assert f(None, 8, 4, P, 1 << 20, None, None) == E and f(P, 8, 4, None, 1 << 20, None, None) == E
    assert f(P + 2, 8, 4, P, 1 << 20, None, None) == E and f(P, 8, 4, P + 8, 1 << 20, None, None) == E
    assert f(P, -1, 4, P, 1 << 20, None, None) == E and f(P, 8, 0, P, 1 << 20, None, None) == E
    assert f(P, 8, 1025, P, 1 << 20, None, None) == U and f(P, (1 << 24) + 1, 4, P, 1 << 40, None, None) == R
    assert f(P, 8, 4, P, size(8, 4) - 1, None, None) == N
    assert f(None, 0, 4, None, 0, None, None) == OK
    assert size(0, 4) == 0 and size(-1, 4) == 0 and size(8, 0) == 0 and size(8, 1025) == 0


@pytest.mark.parametrize("tokens,n", [(1, 1), (1, 1000), (17, 3), (64, 24), (1000, 2), (16384, 64)])
def test_rows_hold_every_tile(tokens, n):
    """The worst case: each group's last tile holds one row."""
    groups = min(tokens, n + 1)
    for height in (16, 64):
        worst = max((sum(-(-c // height) for c in [tokens - (k - 1)] + [1] * (k - 1)) for k in range(1, groups + 1)))
        assert ppas._lib.ppas_adapter_rows_bytes(tokens, n) >= 16 + 16 * worst + 4 * tokens


def test_workspace():
    f = ppas.adapter_workspace_bytes
    assert f(0, 128, 16, 4) == 0 and f(8, 0, 16, 4) == 0 and f(8, 128, 129, 4) == 0 and f(8, 128, 16, 0) == 0
    assert f(1, 2048, 16, 8) == 4 * 64 and f(16384, 2048, 64, 4) % (16384 * 256) == 0


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("rank,padded", [(1, 16), (16, 16), (17, 32), (33, 64), (65, 128), (128, 128)])
def test_workspace_holds_a_split(act, rank, padded):
    """The least that a call takes: the rows' products with A once."""
    assert call(act, adapters=make(rank=rank), ws_bytes=8 * padded * 4 - 1) == N
    assert call(act, adapters=make(rank=rank), ws_bytes=0) == N


def test_binding_refusals(monkeypatch):
    t, BF = torch.zeros, torch.bfloat16
    monkeypatch.setattr(ppas, "_dev", lambda v, name: None if v is None else 64)
    monkeypatch.setattr(ppas, "_here", lambda s, *v: 0)
    a, b = t((3, 8, 64), dtype=BF), t((3, 32, 8), dtype=BF)
    for bad in ((a.float(), b), (a, b.half()), (a[0], b), (a, b[:2]), (a[:, :4], b), (a, b, t(2)), (a, b, t(3, dtype=torch.float64)),
                (a, b, t((3, 1)))):
        with pytest.raises(ValueError, match="must be"):
            ppas.adapters(*bad)
    s = ppas.adapters(a, b)
    rows = ppas.AdapterRows(4, 3, device="cpu")
    x, y, ws = t((4, 64), dtype=BF), t((4, 32), dtype=BF), t(4096, dtype=torch.uint8)
    with pytest.raises(ValueError, match="sorted"):
        ppas.adapter_add(s, x, y, y, rows, ws)
    for bad in (t(4, dtype=torch.int64), t(3, dtype=torch.int32), t((4, 1), dtype=torch.int32)):
        with pytest.raises(ValueError, match="row_adapter"):
            rows.sort(bad)
    rows.sorted = True
    with pytest.raises(ValueError, match="device tensor"):
        ppas.adapter_add(s, x, y, y, rows, ws)
    for kw, message in ((dict(x=x[:3]), "rows are of"), (dict(x=x.float()), "x must be"), (dict(y=y[:3]), "y must be"),
                        (dict(out=t((4, 16), dtype=BF)), "out must be"), (dict(x=t((4, 128), dtype=BF)[:, ::2]), "packed"),
                        (dict(rows=ppas.AdapterRows(4, 2, device="cpu")), "rows are of")):
        args = {**dict(x=x, y=y, out=y.clone(), rows=rows, workspace=ws), **kw}
        monkeypatch.setattr(torch.Tensor, "is_cuda", True)
        with pytest.raises(ValueError, match=message):
            ppas.adapter_add(s, **args)
        monkeypatch.undo()
        monkeypatch.setattr(ppas, "_dev", lambda v, name: None if v is None else 64)
        monkeypatch.setattr(ppas, "_here", lambda st, *v: 0)
    odd = ppas.adapters(a, t((3, 31, 8), dtype=BF))
    with pytest.raises(ValueError, match="half"):
        ppas.adapter_act(odd, x, t((4, 31), dtype=BF), t((4, 15), dtype=BF), rows, ws)
    for bad in ((-1, 3), (4, 0), (4, 1025)):
        with pytest.raises(ValueError, match="no rows"):
            ppas.AdapterRows(*bad, device="cpu")
    assert ppas.AdapterRows(0, 3, device="cpu").buf.numel() == 16


