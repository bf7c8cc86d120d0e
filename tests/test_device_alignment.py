"""Arrays are aligned to 16 bytes: no access of the device code may count on more.  Looked up in what the compiler makes of it."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_17286_amd import build as bld

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which("hipcc")), reason="hipcc not found")
@pytest.mark.parametrize("source", ["gta_mx_cache.hip", "gta_norm_rope.hip", "gta_mx_decode.hip"])
def test_no_access_counts_on_more_than_16_bytes(source, tmp_path):
    out = str(tmp_path / "device.ll")
    p = subprocess.run([HIPCC, *bld.FLAGS, "-x", "hip", "--cuda-device-only", "-S", "-emit-llvm", os.path.join(bld.CSRC, source), "-o", out],
                       capture_output=True, text=True, timeout=600)
    assert p.returncode == 0, p.stderr[-3000:]
    text = open(out).read()
    assert re.search(r"= load .*align 16", text)
    wide = [line.strip() for line in text.splitlines() if re.search(r"\b(load|store) .*align (32|64|128)\b", line)]
    assert not wide, wide[:3]
