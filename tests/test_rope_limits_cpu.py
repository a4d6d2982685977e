"""Frequencies that fp64 cannot hold angles of are refused (they gave cos = 1 at every position, and NaN at far ones)."""
import ctypes
import math

import pytest

ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")

TURN = 2.0 * math.pi


@pytest.mark.parametrize("kw", [dict(theta=1e-300), dict(theta=1e-5), dict(scaling="linear", factor=1e-300),
                                dict(scaling="linear", factor=1 / (4100.0 * TURN)),
                                dict(scaling="bands", factor=1e-9, original_len=100, low=1.0, high=4.0, theta=100.0)])
def test_too_many_turns_are_refused(kw):
    rope = ppas.rope(**kw)
    with pytest.raises(ppas.PPASError) as e:
        ppas.rope_frequencies(rope)
    assert e.value.status == ppas.PPAS_EINVAL
    # and by every call, before any pointer is looked at
    f = ppas._lib.ppas_rope_rows
    assert f(ctypes.byref(rope), 16, 128, 16, 128, 16, 1, 1, 128, 0, None, None) == ppas.PPAS_EINVAL


@pytest.mark.parametrize("kw", [dict(theta=1e-3), dict(theta=0.5), dict(scaling="linear", factor=1 / (4090.0 * TURN)),
                                dict(theta=1e12)])
def test_the_others_are_not(kw):
    w = ppas.rope_frequencies(ppas.rope(**kw))
    assert (w > 0).all() and (w <= 4096 * TURN).all()
