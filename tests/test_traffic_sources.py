"""A kernel's traffic record is dropped when its sources change: every header with device code that they include has to be
among them (CPU only)."""
import os
import re

import pytest

from paper_2608_15171_amd import profile_summary as P


def includes(path, seen):
    for name in re.findall(r'^#include "([^"]+)"', open(path).read(), re.M):
        header = os.path.join(os.path.dirname(path), name)
        if os.path.exists(header) and header not in seen:
            seen.add(header)
            includes(header, seen)
    return seen


@pytest.mark.parametrize("kernel", sorted(P.SOURCES))
def test_every_device_header_counts(kernel):
    listed = {os.path.join(P.ROOT, s) for s in P.SOURCES[kernel]}
    for source in [s for s in listed if s.endswith(".hip")]:
        device = {h for h in includes(source, set()) if "__device__" in open(h).read()}
        assert device <= listed, sorted(device - listed)
        assert any(kernel in open(s).read() for s in listed | {source})
