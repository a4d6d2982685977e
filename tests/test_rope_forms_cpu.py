"""The rotary forms on the CPU: the library's frequency table against the oracle's, and every refusal."""
import ctypes

import numpy as np
import pytest

import oracle.rope_forms as F

ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")

SCALED = [("none", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
          ("bands", dict(factor=8.0, original_len=8192, low=1.0, high=4.0)),
          ("ramp", dict(factor=4.0, original_len=8192, low=1.0, high=32.0)),
          ("ramp", dict(factor=16.0, original_len=100, low=20.0, high=21.0)),      # the ends cross: pairs below one turn
          ("linear", dict(factor=0.5))]


@pytest.mark.parametrize("scaling,kw", SCALED)
@pytest.mark.parametrize("rotary", [2, 4, 20, 64, 96, 128, 256])
@pytest.mark.parametrize("theta", [1e4, 1e6, 5e5])
def test_frequencies(scaling, kw, rotary, theta):
    got = ppas.rope_frequencies(ppas.rope("half", rotary, theta, scaling, **kw), 256)
    want = [F.frequency(j, rotary, theta, scaling, **kw) for j in range(rotary // 2)]
    # powers and logarithms of 64 bits, each within a few units of 2^-53 times an exponent below 20
    np.testing.assert_allclose(got, want, rtol=1e-13, atol=0)


BAD = [dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=130), dict(theta=0.0), dict(theta=-1.0),
       dict(theta=float("nan")), dict(theta=float("inf")), dict(magnitude=-1.0), dict(magnitude=float("inf")),
       dict(magnitude=1e300), dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=float("nan")),
       dict(scaling="base", factor=-2.0), dict(scaling="base", factor=1e300, rotary_dim=4),
       dict(scaling="bands", factor=2.0, original_len=0, low=1.0, high=4.0),
       dict(scaling="bands", factor=2.0, original_len=10, low=4.0, high=4.0),
       dict(scaling="bands", factor=2.0, original_len=10, low=0.0, high=4.0),
       dict(scaling="ramp", factor=2.0, original_len=10, low=1.0, high=float("inf")),
       dict(scaling="ramp", factor=2.0, original_len=10, low=1.0, high=4.0, theta=1.0)]


@pytest.mark.parametrize("bad", BAD)
def test_forms_out_of_range(bad):
    r = ppas.rope(**bad)
    with pytest.raises(ppas.PPASError) as e:
        ppas.rope_frequencies(r)
    assert e.value.status == ppas.PPAS_EINVAL
    f = ppas._lib.ppas_rope_rows
    assert f(ctypes.byref(r), 64, 128, 4096, 128, 64, 1, 1, 128, 0, None, None) == ppas.PPAS_EINVAL


def test_unknown_names():
    for kw in (dict(layout="both"), dict(scaling="some")):
        with pytest.raises(ValueError):
            ppas.rope(**kw)
    r = ppas.rope()
    for field, v in (("layout", 2), ("layout", -1), ("scaling", 5), ("scaling", -1)):
        s = ppas.Rope.from_buffer_copy(r)
        setattr(s, field, v)
        with pytest.raises(ppas.PPASError):
            ppas.rope_frequencies(s)


def test_rows_refusals():
    f, r, half = ppas._lib.ppas_rope_rows, ppas.rope(), ppas.events(start=1)
    ok = [ctypes.byref(r), 1 << 20, 256, 1 << 30, 256, 64, 4, 2, 128, 0, None, None]

    def call(**kw):
        a = list(ok)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return f(*a)
    E, U, R = ppas.PPAS_EINVAL, ppas.PPAS_EUNSUPPORTED, ppas.PPAS_ERANGE
    assert call(a0=None) == E and call(a1=None) == E and call(a3=None) == E and call(a5=None) == E
    assert call(a6=-1) == E and call(a7=0) == E and call(a7=65537) == E and call(a8=127) == E and call(a8=0) == E
    assert call(a8=258, a2=600, a4=600) == U and call(a8=64) == E                # rotary_dim above the head
    assert call(a2=255) == E and call(a4=255) == E and call(a2=-256) == E         # strides below a row
    assert call(a1=(1 << 20) + 1) == E and call(a5=66) == E                       # alignment of an element
    assert call(a2=1 << 60) == R
    assert call(a10=ctypes.byref(half)) == E
    assert call(a3=(1 << 20) + 2) == E and call(a3=1 << 20, a4=512) == E          # overlapping, not in place
    assert call(a3=(1 << 20) + 2 * (3 * 256 + 256) - 2) == E                      # the last element
    assert call(a6=0, a1=None, a3=None, a5=None) == ppas.PPAS_OK                  # no rows


def _append(**kw):
    sh = ppas.make_shape(16, 2, 100)
    desc = np.array([[0, 1, 30], [1, 20, 5]], dtype=np.int32)
    bt = np.array([[0, 1, -1], [2, 3, -1]], dtype=np.int32)
    rows = ppas.Qkv(1 << 20, (1 << 20) + 4096, (1 << 20) + 4608, 2560, 2560, 2560)
    a = dict(shape=sh, rope=ppas.rope(), rows=rows, q_out=1 << 30, kp=1 << 31, vp=1 << 32, desc=desc, bt=1 << 16,
             stride=3, bt_host=bt)
    a.update(kw)
    p = lambda s: None if s is None else ctypes.byref(s)     # noqa: E731
    return ppas._lib.ppas_rope_qkv_append(p(a["shape"]), p(a["rope"]), p(a["rows"]), a["q_out"], a["kp"], a["vp"],
                                          a["desc"].ctypes.data, len(a["desc"]), a["bt"], a["stride"],
                                          None if a["bt_host"] is None else a["bt_host"].ctypes.data, None)


def test_append_refusals():
    E = ppas.PPAS_EINVAL
    q = 1 << 20
    for bad in (dict(rope=None), dict(rope=ppas.rope(rotary_dim=7)), dict(rows=None), dict(q_out=None), dict(kp=None),
                dict(vp=None), dict(bt=None), dict(kp=(1 << 31) + 8), dict(vp=(1 << 32) + 2), dict(q_out=(1 << 30) + 1),
                dict(rows=ppas.Qkv(None, q, q, 2560, 2560, 2560)), dict(rows=ppas.Qkv(q, q, None, 2560, 2560, 2560)),
                dict(rows=ppas.Qkv(q, q, q, 2047, 2560, 2560)), dict(rows=ppas.Qkv(q, q, q, 2560, 255, 2560)),
                dict(rows=ppas.Qkv(q, q, q, 2560, 2560, 0)), dict(rows=ppas.Qkv(q + 1, q, q, 2560, 2560, 2560)),
                dict(q_out=q), dict(q_out=q + 2 * 20 * 2560), dict(q_out=q - 2),
                # in place, but over the keys beside the queries
                dict(q_out=q, rows=ppas.Qkv(q, q + 4096, q + 4096, 2048, 2048, 2048)),
                dict(desc=np.array([[0, 0, 3]], np.int32)), dict(stride=1)):
        assert _append(**bad) == E, bad
    assert _append(rows=ppas.Qkv(q, q, q, 1 << 60, 2560, 2560)) == ppas.PPAS_ERANGE
    assert _append(shape=ppas.make_shape(16, 2, 3)) == ppas.PPAS_ERANGE
    assert _append(desc=np.zeros((0, 3), np.int32)) == ppas.PPAS_OK
    assert _append(desc=np.zeros((0, 3), np.int32), rope=ppas.rope(rotary_dim=7)) == E
    f = ppas._lib.ppas_rope_qkv_append_planned
    r = ppas.rope()
    assert f(None, ctypes.byref(r), None, None, None, None, None, None, None) == E
