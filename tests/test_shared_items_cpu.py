"""ppas_plan_shared_items on the CPU: what a shared plan's introspection reports, and its refusals."""
import ctypes

import numpy as np
import pytest

ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")


def test_rows_of_single_waves_come_last_with_kind_two():
    n, prefix = 64, 2048
    desc = np.array([[i, 1, prefix + 8 * i] for i in range(n)], np.int32)
    shape = ppas.make_shape(16, 2, 10000)
    it = ppas.plan_items(shape, desc, opts=ppas.plan_opts(0, 0, 16, 8), prefixes=[(0, n, prefix)])
    kinds = it[:, 0].tolist()
    assert kinds == sorted(kinds, key=lambda k: k == 2) and kinds.count(2) == 2 * n
    rows = it[it[:, 0] == 2]
    assert sorted(map(tuple, rows[:, 1:3].tolist())) == [(s, g) for s in range(n) for g in range(2)]
    assert (rows[:, 6] == prefix).all() and (rows[:, 7] == prefix + 8 * rows[:, 1] + 1).all() and (rows[:, 5] == 1).all()
    tiles = it[it[:, 0] == 0]
    assert (tiles[:, 7] <= prefix).all() and (tiles[:, 4] == prefix).all() and (tiles[:, 1] == 0).all()


def test_without_prefixes_it_is_plan_items():
    desc = np.array([[0, 40, 100], [40, 1, 3000], [41, 1, 7]], np.int32)
    shape = ppas.make_shape(16, 2, 1000)
    a = ppas.plan_items(shape, desc)
    out = np.zeros_like(a)
    n = ppas._lib.ppas_plan_items(ctypes.byref(shape), desc.ctypes.data, 3, None, out.ctypes.data, len(out))
    assert n == len(a) and np.array_equal(a, out)
    assert np.array_equal(ppas.plan_items(shape, desc, prefixes=[(1, 2, 0)]), a)


def test_capacity_and_refusals():
    desc = np.array([[0, 1, 64], [1, 1, 64]], np.int32)
    shape, p = ppas.make_shape(16, 2, 1000), np.array([[0, 2, 64]], np.int32)
    f = ppas._lib.ppas_plan_shared_items
    out = np.full((8, 8), -7, np.int32)
    n = f(ctypes.byref(shape), desc.ctypes.data, 2, p.ctypes.data, 1, None, out.ctypes.data, 1)
    assert n > 1 and (out[1:] == -7).all() and (out[0] != -7).all()
    assert f(ctypes.byref(shape), desc.ctypes.data, 2, p.ctypes.data, 1, None, out.ctypes.data, -1) == n
    assert f(ctypes.byref(shape), desc.ctypes.data, 2, None, 1, None, None, 0) == ppas.PPAS_EINVAL
    p[0, 2] = 80
    assert f(ctypes.byref(shape), desc.ctypes.data, 2, p.ctypes.data, 1, None, None, 0) == ppas.PPAS_EINVAL
