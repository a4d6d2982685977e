"""The 8-bit calls' refusals and workspace sizes on the CPU, and the quantiser's rounding rule over every pair of values."""
import ctypes

import numpy as np
import pytest

ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")


def test_quantiser_refusals():
    f, half = ppas._lib.ppas_quant_i8, ppas.events(stop=1)
    E = ppas.PPAS_EINVAL
    assert f(64, 64, 4096, 64, 0, 64, None, None) == ppas.PPAS_OK
    assert f(64, 64, 4096, 64, -1, 64, None, None) == E and f(64, 64, 4096, 64, 2, 0, None, None) == E
    assert f(None, 64, 4096, 64, 2, 64, None, None) == E and f(64, 64, None, 64, 2, 64, None, None) == E
    assert f(64, 64, 4096, None, 2, 64, None, None) == E and f(64, 63, 4096, 64, 2, 64, None, None) == E
    assert f(65, 64, 4096, 64, 2, 64, None, None) == E and f(64, 64, 4096, 66, 2, 64, None, None) == E
    assert f(64, 1 << 60, 4096, 64, 4, 64, None, None) == ppas.PPAS_ERANGE
    assert f(64, 64, 4096, 64, 2, 64, ctypes.byref(half), None) == E


@pytest.mark.parametrize("name", ["ppas_gateup_proj_i8", "ppas_gateup_act_i8"])
def test_product_refusals(name):
    f, half = getattr(ppas._lib, name), ppas.events(start=1)
    ok = [64, 64, 64, 64, 64, 4, 96, 8, None, 0, None, None]
    E, R = ppas.PPAS_EINVAL, ppas.PPAS_ERANGE

    def call(**kw):
        a = list(ok)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return f(*a)
    assert call(a5=0) == ppas.PPAS_OK
    for i in range(5):
        assert call(**{f"a{i}": None}) == E, i
    assert call(a5=-1) == E and call(a6=0) == E and call(a7=0) == E and call(a7=-8) == E
    assert call(a1=66) == E and call(a3=65) == E and call(a4=65) == E and call(a8=72, a9=1024) == E
    assert call(a9=1024) == E and call(a10=ctypes.byref(half)) == E
    assert call(a6=131072) == R and call(a5=2 ** 31 - 1) == R and call(a7=2 ** 31 - 1) == R
    assert call(a5=2 ** 31 - 600, a7=2 ** 29) == R          # more tiles than a grid holds


def test_workspace_sizes():
    W, A = ppas.gateup_i8_workspace_bytes, ppas.gateup_act_i8_workspace_bytes
    # 43 stages of 128 features: at most ten splits of four; 8 tiles of 256 columns on 256 compute units
    assert W(16, 11008, 2048) == 21 * 16 * 2048 * 4
    assert W(16, 2048, 2048) == 4 * 16 * 2048 * 4
    assert W(2048, 2048, 22016) == 0 and W(16, 2000, 2048) == 0 and W(0, 2048, 2048) == 0 and W(4, 0, 8) == 0
    assert A(16, 2048, 1024) == W(16, 2048, 2048) and A(16, 2048, 2 ** 30) == 0 and A(16, 2048, -1) == 0


def test_rounding_rule_over_every_ratio():
    """The kernel's product with a rounded reciprocal, cut to 18 bits, gives the nearest even integer of 127 x / max for
    every pair of bf16 mantissas and binades apart (from 2^10 below the maximum on every integer is 0)."""
    top = np.arange(128, 256)
    r = np.float32(127) / top.astype(np.float32)
    for d in range(12):
        m = np.arange(128, 256)
        t = ((m / 2.0 ** d).astype(np.float32)[None, :] * r[:, None]).astype(np.float32).view(np.uint32)
        q = np.rint(((t + np.uint32(0x20)) & ~np.uint32(0x3f)).view(np.float32)).astype(np.int64)
        num, den = (127 * m)[None, :], (top << d)[:, None]
        fl, rem = num // den, num % den
        want = fl + ((2 * rem > den) | ((2 * rem == den) & (fl % 2 == 1)))
        smaller = (m[None, :] <= top[:, None]) | (d > 0)
        assert np.array_equal(q[smaller], want[smaller]), d
