"""The normalised turns on the CPU: every refusal."""
import ctypes

import numpy as np
import pytest
import torch

ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")

E, U, R = ppas.PPAS_EINVAL, ppas.PPAS_EUNSUPPORTED, ppas.PPAS_ERANGE
BF = torch.bfloat16
W = 1 << 24
BAD = [ppas.HeadNorm(W, 0, eps, 0.0, 0) for eps in (0.0, -1e-6, float("nan"), float("inf"), 2.0 ** -101)] + \
      [ppas.HeadNorm(W, 0, 1e-6, float("inf"), 0), ppas.HeadNorm(W, 0, 1e-6, float("nan"), 0),
       ppas.HeadNorm(W + 1, 0, 1e-6, 0.0, 0), ppas.HeadNorm(W, 127, 1e-6, 0.0, 0), ppas.HeadNorm(W, -128, 1e-6, 0.0, 0), None]


def ref(s):
    return None if s is None else ctypes.byref(s)


def rows_call(norm, **kw):
    r = ppas.rope()
    a = [ref(norm), ctypes.byref(r), 1 << 20, 256, 1 << 30, 256, 64, 4, 2, 128, None, None]
    for i, v in kw.items():
        a[int(i[1:])] = v
    return ppas._lib.ppas_norm_rope_rows(*a)


def test_rows_refusals():
    ok = ppas.HeadNorm(W, 128, 1e-6, 1.0, 0)
    for bad in BAD:
        assert rows_call(bad) == E
    assert rows_call(ppas.HeadNorm(W, 1 << 61, 1e-6, 0.0, 0)) == R
    half = ppas.events(start=1)
    for kw in (dict(a1=None), dict(a2=None), dict(a4=None), dict(a6=None), dict(a7=-1), dict(a8=0), dict(a9=127),
               dict(a9=64), dict(a3=255), dict(a5=255), dict(a2=(1 << 20) + 1), dict(a6=66), dict(a4=(1 << 20) + 2),
               dict(a10=ctypes.byref(half))):
        assert rows_call(ok, **kw) == E, kw
    assert rows_call(ok, a9=258, a3=600, a5=600) == U
    assert rows_call(ok, a7=0, a2=None, a4=None, a6=None) == ppas.PPAS_OK
    assert rows_call(BAD[0], a7=0) == E
    # without weights nothing is read of their place or stride
    assert rows_call(ppas.HeadNorm(None, -5, 1e-6, 0.0, 1), a7=0) == ppas.PPAS_OK


def append_call(q_norm, k_norm, **kw):
    sh = ppas.make_shape(16, 2, 100)
    desc = np.array([[0, 1, 30], [1, 20, 5]], dtype=np.int32)
    bt = np.array([[0, 1, -1], [2, 3, -1]], dtype=np.int32)
    rows = ppas.Qkv(1 << 20, (1 << 20) + 4096, (1 << 20) + 4608, 2560, 2560, 2560)
    a = dict(shape=sh, rope=ppas.rope(), rows=rows, q_out=1 << 30, kp=1 << 31, vp=1 << 32, desc=desc, bt=1 << 16)
    a.update(kw)
    return ppas._lib.ppas_norm_rope_qkv_append(ref(a["shape"]), ref(q_norm), ref(k_norm), ref(a["rope"]), ref(a["rows"]),
                                               a["q_out"], a["kp"], a["vp"], a["desc"].ctypes.data, len(a["desc"]), a["bt"],
                                               3, bt.ctypes.data, None)


def test_append_refusals():
    ok = ppas.HeadNorm(W, 0, 1e-6, 0.0, 0)
    for bad in BAD:
        assert append_call(bad, ok) == E and append_call(ok, bad) == E
    q = 1 << 20
    for kw in (dict(rope=None), dict(rope=ppas.rope(rotary_dim=7)), dict(rows=None), dict(q_out=None), dict(kp=None), dict(vp=None),
               dict(bt=None), dict(kp=(1 << 31) + 8), dict(q_out=q), dict(rows=ppas.Qkv(q, q, q, 2047, 2560, 2560)),
               dict(desc=np.array([[0, 0, 3]], np.int32))):
        assert append_call(ok, ok, **kw) == E, kw
    assert append_call(ok, ok, shape=ppas.make_shape(16, 2, 3)) == R
    assert append_call(ok, ok, desc=np.zeros((0, 3), np.int32)) == ppas.PPAS_OK
    f = ppas._lib.ppas_norm_rope_qkv_append_planned
    assert f(None, ref(ok), ref(ok), ref(ppas.rope()), None, None, None, None, None, None, None) == E


def test_outputs_over_the_weights():
    """Rows: y of 4 rows of 256 features at 1 << 30. A step: q_out of 21 rows of 2,048, pools of 100 pages of 4,096."""
    y = 1 << 30
    for stride, at in ((0, y), (0, y - 254), (0, y + 2 * 1023), (128, y - 510), (1000, y - 2254)):
        assert rows_call(ppas.HeadNorm(at, stride, 1e-6, 0.0, 0)) == E, (stride, at)
    ok = ppas.HeadNorm(W, 0, 1e-6, 0.0, 0)
    q, kp, vp = 1 << 30, 1 << 31, 1 << 32
    pool = 100 * 4096 * 2
    for at in (q, q - 254, q + 2 * (21 * 2048 - 1), kp, kp + pool - 2, kp - 2, vp, vp + pool - 2):
        bad = ppas.HeadNorm(at, 0, 1e-6, 0.0, 0)
        assert append_call(bad, ok) == E and append_call(ok, bad) == E, at
    assert append_call(ppas.HeadNorm(q - 16 * 256, 128, 1e-6, 0.0, 0), ok, q_out=q - 2) == E
    assert append_call(ok, ppas.HeadNorm(kp - 2 * 1024 - 254, 1024, 1e-6, 0.0, 0)) == E


def test_binding_takes_bf16_weights(monkeypatch):
    for w in (torch.zeros(128), torch.zeros(128, dtype=torch.float16), torch.zeros((2, 2, 128), dtype=BF),
              torch.zeros((128, 2), dtype=BF).t(), torch.zeros(256, dtype=BF)[::2], torch.zeros((), dtype=BF)):
        with pytest.raises(ValueError, match="weight must be"):
            ppas.head_norm(w)
    with pytest.raises(ValueError, match="device tensor"):
        ppas.head_norm(torch.zeros(128, dtype=BF))
    monkeypatch.setattr(ppas, "_heads", lambda v, name: (0, 256))
    monkeypatch.setattr(ppas, "_dev", lambda v, name: 0)
    x, pos = torch.zeros((4, 2, 128), dtype=BF), torch.zeros(4, dtype=torch.int32)
    for shape in ((64,), (3, 128), (1, 128), (2, 64)):
        n = ppas.head_norm()
        n.tensor = torch.zeros(shape, dtype=BF)
        with pytest.raises(ValueError, match="weight must be"):
            ppas.norm_rope_rows(n, ppas.rope(), x, pos, x)
