"""Shared prefixes on the CPU: the planner under the host sanitizers (tests/host/shared_plan_check.cpp) and every refusal."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_planner_under_asan_ubsan(tmp_path):
    exe = tmp_path / "shared_plan_check"
    csrc = os.path.join(ROOT, "paper_2608_15171_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "plan.cpp"),
           os.path.join(ROOT, "tests", "host", "shared_plan_check.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout + r.stderr)[-4000:]


ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")

DESC = np.array([[0, 1, 40], [1, 3, 36], [4, 1, 64], [5, 1, 10]], dtype=np.int32)
BT = np.array([[0, 1, 2, -1, -1], [0, 1, 3, -1, -1], [0, 1, 4, 5, 6], [7, -1, -1, -1, -1]], dtype=np.int32)


def create(prefixes, desc=DESC, bt=BT, n=None):
    p = np.asarray(prefixes, dtype=np.int32).reshape(-1, 3)
    h = ctypes.c_void_p(1)
    st = ppas._lib.ppas_step_plan_create_shared(ctypes.byref(ppas.make_shape(16, 2, 100)), desc.ctypes.data, len(desc),
                                                p.ctypes.data if len(p) else None, len(p) if n is None else n,
                                                None if bt is None else bt.ctypes.data, BT.shape[1], None, ctypes.byref(h))
    assert h.value is None
    return st


@pytest.mark.parametrize("bad", [
    [(-1, 2, 32)], [(0, 0, 32)], [(0, -1, 32)], [(0, 5, 0)], [(4, 1, 0)], [(3, 2, 0)],   # requests outside the step
    [(0, 2, -16)], [(0, 2, 8)], [(0, 2, 33)],                                            # no whole pages
    [(0, 2, 48)], [(0, 4, 16)],                                                          # longer than a member's cache
    [(0, 2, 32), (1, 2, 32)], [(2, 1, 16), (0, 2, 32)],                                  # overlapping, out of order
    [(0, 2 ** 31 - 1, 16)], [(2 ** 31 - 1, 1, 16)]])
def test_refused_prefixes(bad):
    assert create(bad) == ppas.PPAS_EINVAL
    assert create(bad, bt=None) == ppas.PPAS_EINVAL
    p = np.asarray(bad, np.int32)
    assert ppas.attn_shared_workspace_bytes(ppas.make_shape(16, 2, 100), DESC, p) == 0


def test_tables_that_differ_are_refused():
    bt = BT.copy()
    bt[1, 1] = 8
    assert create([(0, 3, 32)], bt=bt) == ppas.PPAS_EINVAL
    assert create([(0, 3, 32)], bt=BT) == ppas.PPAS_EUNSUPPORTED        # valid: no gfx950 device here
    assert create([(0, 3, 16)], bt=bt) == ppas.PPAS_EUNSUPPORTED
    assert create([(0, 3, 32)], bt=None) == ppas.PPAS_EUNSUPPORTED


def test_null_and_empty():
    assert create([], n=1) == ppas.PPAS_EINVAL and create([], n=-1) == ppas.PPAS_EINVAL
    assert create([(0, 1, 0)], desc=np.zeros((0, 3), np.int32)) == ppas.PPAS_EINVAL
    f = ppas._lib.ppas_step_plan_create_shared
    assert f(ctypes.byref(ppas.make_shape(16, 2, 100)), DESC.ctypes.data, 4, None, 0, None, 5, None, None) == ppas.PPAS_EINVAL
    g = ppas._lib.ppas_attn_step_shared
    p = np.array([(0, 3, 32)], np.int32)
    sh = ctypes.byref(ppas.make_shape(16, 2, 100))
    args = [sh, 1, 1, 1, 1, DESC.ctypes.data, 4, p.ctypes.data, 1, 1, 5, BT.ctypes.data, 1, 1 << 30, None]
    assert g(*args) == ppas.PPAS_EUNSUPPORTED
    for i in (1, 2, 3, 4, 9, 12):
        assert g(*[None if k == i else a for k, a in enumerate(args)]) == ppas.PPAS_EINVAL, i
    with pytest.raises(ValueError):
        ppas.attn_shared_workspace_bytes(ppas.make_shape(16, 2, 100), DESC, np.zeros((2, 2), np.int32))


def test_workspace_covers_the_plan_and_no_prefix_is_the_plain_step():
    sh = ppas.make_shape(16, 2, 10000)
    desc = np.array([[i, 1, 4096 + i] for i in range(40)], np.int32)
    assert ppas.attn_shared_workspace_bytes(sh, desc, []) == ppas.attn_workspace_bytes(sh, desc)
    assert ppas.attn_shared_workspace_bytes(sh, desc, [(0, 40, 0)]) == ppas.attn_workspace_bytes(sh, desc)
    assert ppas.attn_shared_workspace_bytes(sh, desc, [(0, 40, 4096)]) > 40 * 16 * 2 * 520


@pytest.mark.parametrize("bad", [np.array([[0, 2, 2 ** 32 + 32]]), np.array([[0, 2, 32.5]]), np.zeros((2, 2), np.int32),
                                 [(0, 2)], [0, 2, 32]])
def test_prefixes_that_are_no_int32_rows(bad):
    with pytest.raises(ValueError):
        ppas.attn_shared_workspace_bytes(ppas.make_shape(16, 2, 100), DESC, bad)
