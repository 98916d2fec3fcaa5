"""CPU: the paged cache's sources compile without a warning under the build's flags (host and device)."""
import os
import subprocess

import pytest

from paper_2609_05707_amd import build as B


@pytest.mark.skipif(not os.path.exists(B.hipcc()), reason="hipcc not available")
@pytest.mark.parametrize("source", [s for s in B.SOURCES if s.startswith("paged_")])
def test_no_warnings(source):
    r = subprocess.run([B.hipcc(), *B.flags_for(source), "-fsyntax-only", os.path.join(B.CSRC, source)], capture_output=True,
                       text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    # (the sources' own; the driver's warn of flags that one of the passes does not use)
    found = [line for line in r.stderr.splitlines() if "warning:" in line and "csrc/" in line]
    assert not found, (len(found), found[:2])
