"""A wait of the few-token kernel that no run can show missing: read from the gfx950 assembly of its
source (CPU: compiled, not run)."""
import os
import shutil

import pytest

from paper_2609_36070_amd import build
from tests.test_int_waits import kernels

HAVE_HIPCC = shutil.which(build.HIPCC) is not None or os.path.exists(build.HIPCC)
pytestmark = pytest.mark.skipif(not HAVE_HIPCC, reason="needs hipcc")


def test_sums_have_arrived_before_their_counter_rises():
    """A tile's sums are stored, 8 loads of the next item follow, and a wait that leaves 8 operations
    open comes before the barrier behind which another workgroup is told.  Operations end in order:
    the stores are done only if 8 loads or more stand between them and the wait, on every path."""
    found = kernels("few.hip", "few_kernel")
    assert len(found) == 2
    for lines in found.values():
        check_wait(lines)


def check_wait(lines):
    waits = [i for i, ln in enumerate(lines) if ln == "s_waitcnt vmcnt(8)"]
    # the one of the source is followed by the barrier; others are the compiler's own
    mine = [i for i in waits if any(ln.startswith("s_barrier") for ln in lines[i:i + 6])]
    assert len(mine) == 1
    i, loads = mine[0], 0
    while loads < 8:
        i -= 1
        ln = lines[i]
        # one straight run of loads: no label, branch, store or change of the lanes within it
        assert not ln.endswith(":") and not ln.startswith(("s_cbranch", "s_branch", "global_store", "scratch_store",
                                                           "s_and_saveexec", "s_or_saveexec")), ln
        loads += ln.startswith("global_load_dwordx4")


def test_other_workgroups_read_what_was_stored_to_memory():
    """Sums and H, which workgroups of other XCDs read, leave in device-scope stores (sc1: through the
    L2): 4 of sums, 4 of H at either of two places."""
    for lines in kernels("few.hip", "few_kernel").values():
        assert sum(ln.startswith("global_store_dwordx2") and ln.endswith("sc1") for ln in lines) >= 12
