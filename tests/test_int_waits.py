"""Waits of the int8 tile kernel that no run can show missing: read from the
gfx950 assembly of its source (CPU: compiled, not run)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_36070_amd import build

HAVE_HIPCC = shutil.which(build.HIPCC) is not None or os.path.exists(build.HIPCC)
pytestmark = pytest.mark.skipif(not HAVE_HIPCC, reason="needs hipcc")


def kernels(source, name):
    """Instruction lines of each instance of a kernel."""
    cmd = [build.HIPCC, *build.FLAGS, "--offload-device-only", "-S", os.path.join(build.CSRC, source), "-o", "-"]
    asm = subprocess.run(cmd, capture_output=True, text=True, check=True).stdout
    found = re.findall(rf"^(\S*{name}\S*):.*?\n(.*?)^\.Lfunc_end", asm, re.S | re.M)
    return {k: [ln.split(";")[0].strip() for ln in body.splitlines()] for k, body in found}


def test_scales_reach_lds_before_the_barrier_that_publishes_them():
    """A wave writes its thread's scale of a tile to LDS, for other waves to read
    in the epilogue.  Waves without rows read nothing from LDS in between, so
    that only a wait before the barrier makes the write complete."""
    found = kernels("gemm_i8.hip", "gemm_i8_kernel")
    assert len(found) == 2
    for name, lines in found.items():
        write = next(i for i, ln in enumerate(lines) if ln.startswith("ds_write"))
        barrier = next(i for i in range(write, len(lines)) if lines[i].startswith("s_barrier"))
        between = lines[write:barrier]
        assert any(ln.startswith("s_waitcnt") and "lgkmcnt(0)" in ln for ln in between), (name, between)
