"""The choice that steps with shared prefixes are planned by, on the CPU (tests/host/shared_choice_check.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_choice_of_shared_plans(tmp_path):
    exe = tmp_path / "shared_choice_check"
    csrc = os.path.join(ROOT, "paper_2608_15171_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "plan.cpp"),
           os.path.join(ROOT, "tests", "host", "shared_choice_check.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", (r.stdout + r.stderr)[-4000:]
