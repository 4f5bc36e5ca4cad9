"""Registers of the selection by scores, from the compiler's own count for gfx950
(CPU: compiled, not run).  Past 128 a SIMD holds two waves instead of four, which
costs large batches 6 to 10 %; scratch is memory traffic."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_36070_amd import build

HAVE_HIPCC = shutil.which(build.HIPCC) is not None or os.path.exists(build.HIPCC)
pytestmark = pytest.mark.skipif(not HAVE_HIPCC, reason="needs hipcc")


def test_selection_keeps_four_waves_per_simd():
    cmd = [build.HIPCC, *build.FLAGS, "--offload-device-only", "-S", os.path.join(build.CSRC, "score.hip"), "-o", "-"]
    asm = subprocess.run(cmd, capture_output=True, text=True, check=True).stdout
    # the counts follow each function's end
    found = re.findall(r"^\s*\.size\s+(\S*score_select_kernel\S*),|^; NumVgprs: (\d+)|^; ScratchSize: (\d+)", asm, re.M)
    kernels, name = {}, None
    for label, vgprs, scratch in found:
        if label:
            name = label
        elif name and vgprs:
            kernels[name] = int(vgprs)
        elif name and scratch:
            assert int(scratch) == 0, name
            name = None
    assert len(kernels) == 40
    # 8 experts per lane and lists of up to 8: what batches of any size run
    common = {k: v for k, v in kernels.items() if re.search(r"ILi8ELi\d+ELi[1248]E", k)}
    assert len(common) == 28 and max(common.values()) <= 128, common
