"""What the compiler gives each kernel of the library (CPU only): no kernel may keep anything in scratch memory.

A kernel argument or array that the compiler puts there costs more than its loads: in the kernels whose transfers
into LDS stay in flight, each of those loads waits for every transfer before it."""
import os
import re
import subprocess

import pytest

from paper_2608_15171_amd import build as B


@pytest.mark.parametrize("source", [s for s in B.SOURCES if s.endswith(".hip")])
def test_no_kernel_uses_scratch_memory(tmp_path, source):
    out = tmp_path / (source + ".s")
    cmd = [B.hipcc(), *[f for f in B.HIPCC_FLAGS if f != "-shared"], "--cuda-device-only", "-S", "-I", B.INCLUDE,
           "-I", B.CSRC, os.path.join(B.CSRC, source), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    text = out.read_text()
    size = re.findall(r"\.name:\s+(\S+)\n\s+\.private_segment_fixed_size:\s+(\d+)", text)
    assert len(size) == text.count(".amdhsa_kernel ")
    assert [s for s in size if s[1] != "0"] == []
    assert not re.search(r"^\s+scratch_", text, re.M)
