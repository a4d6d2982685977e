"""Build libppas.so for gfx950 with hipcc (in-tree, next to this file).

Usage: python -m paper_2608_15171_amd.build
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libppas.so")

SOURCES = ["api.cpp", "plan.cpp", "attn_step.hip", "kv_append.hip", "rope_append.hip", "rope.cpp", "rope_rows.hip",
           "norm_rope.hip", "logprobs.hip", "adapters.hip", "noalloc.hip", "gateup.hip", "gateup_any.hip",
           "gateup_i8.hip", "int8.hip", "stream_read.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    "-Wall",
    # code object v5 loads under both the system ROCm runtime and the one PyTorch bundles
    "-mcode-object-version=5",
    # no packed-fp32 instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def build(verbose: bool = False, defines=(), out: str | None = None) -> str:
    """Compile every source into libppas.so (always rebuilds). Returns the library path.
    `defines` are extra -D options (tuning constants); `out` writes the library elsewhere."""
    lib = out or LIB
    tmp = lib + ".tmp"
    cmd = [hipcc(), *HIPCC_FLAGS, *[f"-D{d}" for d in defines], "-I", INCLUDE, "-I", CSRC,
           *[os.path.join(CSRC, s) for s in SOURCES], "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed ({r.returncode}):\n{err}")
    if verbose and err.strip():
        print(err)
    os.replace(tmp, lib)
    return lib


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
