"""The chunk attention's inline-assembly LDS reads: the checks of the other
attention kernels' reads (test_kernel_lds_waits.py, test_kernel_lds_flow.py) on
its gfx950 code, and one more: scalar loads share the LDS counter and return in
any order, so none may be in flight at a wait that keeps some operations in
flight (CPU only)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_03333_amd import build
from test_kernel_lds_flow import _blocks, pending_read_uses
from test_kernel_lds_waits import HIPCC, lds_wait_hazards

SCALAR_LOADS = ("s_load", "s_buffer_load")


def counted_waits_behind_scalar_loads(lines):
    """Waits for all but some LDS operations that a scalar load may be in flight at, along any path."""
    bodies, succ = _blocks(lines)

    def flow(body, flying, report=None):
        for t in body:
            if t.startswith(SCALAR_LOADS):
                flying = True
            m = re.search(r"lgkmcnt\((\d+)\)", t) if t.startswith("s_waitcnt") else None
            if m:
                if int(m.group(1)) == 0:
                    flying = False
                elif flying and report is not None:
                    report.append(t)
        return flying

    entry, work = {0: False}, [0]
    while work:
        i = work.pop()
        out = flow(bodies[i], entry[i])
        for s in succ[i]:
            if s not in entry or (out and not entry[s]):
                entry[s] = out or entry.get(s, False)
                work.append(s)
    report = []
    for i in sorted(entry):
        flow(bodies[i], entry[i], report)
    return report


def test_the_scalar_load_check_follows_branches():
    bad = """s_load_dword s0, s[2:3], 0x0
s_cbranch_vccnz .LBB0_2
; %bb.1:
s_waitcnt lgkmcnt(0)
.LBB0_2:
s_waitcnt vmcnt(3) lgkmcnt(5)
s_endpgm""".splitlines()
    assert counted_waits_behind_scalar_loads(bad) == ["s_waitcnt vmcnt(3) lgkmcnt(5)"]
    assert counted_waits_behind_scalar_loads([t for t in bad if "cbranch" not in t]) == []


@pytest.mark.skipif(shutil.which(HIPCC) is None and not os.path.exists(HIPCC), reason="hipcc not installed")
def test_chunk_kernels_wait_before_using_lds_reads(tmp_path):
    out = tmp_path / "chunk.s"
    cmd = [HIPCC, *build.DEVICE_FLAGS, f"-I{build.INCLUDE}", f"-I{build.CSRC}", "--cuda-device-only", "-S",
           "-o", str(out), os.path.join(build.CSRC, "chunk.hip")]
    subprocess.run(cmd, check=True, capture_output=True, timeout=600)
    asm = out.read_text()
    assert lds_wait_hazards(asm, r"chunk_attn") == []
    kernels, name = {}, None
    for line in asm.splitlines():
        t = line.strip()
        m = re.match(r"^(_Z\S*chunk_attn\S*):", t)
        if m:
            name = m.group(1)
            kernels[name] = []
        elif t.startswith(".Lfunc_end"):
            name = None
        elif name:
            kernels[name].append(t)
    assert len(kernels) == 8  # two types, two head sizes, two block sizes
    reads = {n: sum("ds_read" in t for t in lines) for n, lines in kernels.items()}
    assert all(reads.values())
    for name, lines in kernels.items():
        assert pending_read_uses(lines) == [], name
        assert counted_waits_behind_scalar_loads(lines) == [], name
