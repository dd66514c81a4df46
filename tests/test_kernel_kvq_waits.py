"""The checks of the other attention kernels' inline-assembly LDS reads
(test_kernel_lds_waits.py, test_kernel_lds_flow.py, test_kernel_chunk_waits.py) on
the gfx950 code of the attention over 8-bit codes (CPU only)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_03333_amd import build
from test_kernel_chunk_waits import counted_waits_behind_scalar_loads
from test_kernel_lds_flow import pending_read_uses
from test_kernel_lds_waits import HIPCC, lds_wait_hazards


@pytest.mark.skipif(shutil.which(HIPCC) is None and not os.path.exists(HIPCC), reason="hipcc not installed")
def test_kvq_kernels_wait_before_using_lds_reads(tmp_path):
    out = tmp_path / "kvq.s"
    cmd = [HIPCC, *build.DEVICE_FLAGS, f"-I{build.INCLUDE}", f"-I{build.CSRC}", "--cuda-device-only", "-S",
           "-o", str(out), os.path.join(build.CSRC, "chunk_kvq.hip")]
    subprocess.run(cmd, check=True, capture_output=True, timeout=600)
    asm = out.read_text()
    assert lds_wait_hazards(asm, r"chunk_attn") == []
    kernels, name = {}, None
    for line in asm.splitlines():
        t = line.strip()
        m = re.match(r"^(_Z\S*CodeEngine\S*):", t)
        if m:
            name = m.group(1)
            kernels[name] = []
        elif t.startswith(".Lfunc_end"):
            name = None
        elif name:
            kernels[name].append(t)
    assert len(kernels) == 12  # bf16 with and without shared stages, fp32; two head sizes, two block sizes
    for name, lines in kernels.items():
        assert sum("ds_read" in t for t in lines), name
        assert pending_read_uses(lines) == [], name
        assert counted_waits_behind_scalar_loads(lines) == [], name
