"""The word of LDS that tells a workgroup's waves their next item, read from the gfx950 assembly of the
few-token kernel's source (CPU: compiled, not run): a missing barrier shows in no run."""
import re

from tests.test_few_waits import pytestmark  # noqa: F401
from tests.test_int_waits import kernels


def accesses(lines):
    """(line, "read" or "write") of the word that the search for first items writes, in the order of the text."""
    swap = next(i for i, ln in enumerate(lines) if ln.startswith("global_atomic_cmpswap"))
    offset = next(m[1] for ln in lines[swap:] if (m := re.match(r"ds_write_b32 .*(offset:\d+)$", ln)))
    return [(i, "read" if ln.startswith("ds_read_b32") else "write") for i, ln in enumerate(lines)
            if ln.startswith(("ds_read_b32", "ds_write_b32")) and ln.endswith(" " + offset)]


def test_every_wave_has_read_its_item_before_the_word_is_written_again():
    found = kernels("few.hip", "few_kernel")
    assert len(found) == 2
    for lines in found.values():
        words = accesses(lines)
        reads = [i for i, kind in words if kind == "read"]
        writes = [i for i, kind in words if kind == "write"]
        # written by the routing, the search and the end of an item, read before the loop, after the search
        # and at the end of an item
        assert len(reads) == len(writes) == 3 and writes[0] < reads[0] < writes[1] < reads[1] < writes[2] < reads[2]
        # the read before the loop: complete, and behind a barrier, before a wave can go another way
        barrier = next(i for i in range(reads[0], len(lines)) if lines[i].startswith("s_barrier"))
        between = lines[reads[0]:barrier]
        assert barrier < writes[1]
        assert not any(ln.endswith(":") or ln.startswith(("s_branch", "s_cbranch")) for ln in between), between
        assert any(ln.startswith("s_waitcnt") and "lgkmcnt(0)" in ln for ln in between), between
        # the other two: a barrier before the loop comes to a write again
        assert any(lines[i].startswith("s_barrier") for i in range(reads[1], writes[2]))
        assert any(lines[i].startswith("s_barrier") for i in range(reads[2], len(lines)))
