"""CPU: the paged cache's kernels ask no more of an address than the C interface promises: 16 bytes.

A vector type carries an alignment of its own, and eight floats' is 32 bytes: an access through
it at 16 mod 32 is undefined, whatever the hardware does with it.  Read from the kernels' LLVM IR."""
import os
import re
import subprocess

import pytest

from paper_2609_05707_amd import build as B


@pytest.mark.skipif(not os.path.exists(B.hipcc()), reason="hipcc not available")
@pytest.mark.parametrize("source", ["paged_append.hip", "paged_attend.hip"])
def test_global_accesses_ask_for_16_bytes_at_most(source, tmp_path):
    out = tmp_path / "device.ll"
    flags = [f for f in B.flags_for(source) if f != "-fPIC"]
    r = subprocess.run([B.hipcc(), *flags, "--cuda-device-only", "-S", "-emit-llvm", os.path.join(B.CSRC, source), "-o",
                        str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    seen, over = 0, []
    for line in out.read_text().splitlines():
        m = re.search(r"\b(?:load|store) .*ptr(?: addrspace\((\d+)\))? %.*?, align (\d+)", line)
        if m and m.group(1) in (None, "1"):                   # generic or global memory
            seen += 1
            if int(m.group(2)) > 16:
                over.append(line.strip())
    assert seen > 100
    assert not over, (len(over), over[:3])
