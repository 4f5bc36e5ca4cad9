"""Workspace sizes of layers with many experts, whose routers keep partial logits
for some batches only (host functions): a workspace made for a batch holds every
smaller one, up to sizes where no batch has slices any more, and no more than the
slices that some batch takes."""
import ctypes
import functools
import os
import subprocess
import tempfile

import pytest

from paper_2609_36070_amd import binding as B
from tests import dispatch

SIZES = {
    "one pass": lambda s: B.moe_workspace_bytes(s, False), "with backward": lambda s: B.moe_workspace_bytes(s, True),
    "ring": lambda s: B.moe_ring_workspace_bytes(s, 700, False), "MXFP8": lambda s: B.moe_mx_workspace_bytes(s, 0),
    "MXFP8 training": lambda s: B.moe_mx_workspace_bytes(s, 2), "int8": B.moe_int_workspace_bytes,
}
TOKENS = sorted({*range(300), *(128 * i + e for i in range(2, 1100) for e in (0, 1))})


@pytest.mark.parametrize("d,E,k,f", [(512, 256, 1, 256), (7168, 256, 8, 256), (256, 128, 1, 256), (2048, 128, 8, 256),
                                     (4096, 96, 1, 256), (512, 200, 2, 256), (1792, 65, 1, 256), (256, 64, 1, 256)])
def test_sizes_never_fall_with_the_tokens(d, E, k, f):
    for name, size in SIZES.items():
        last = 1
        for t in TOKENS:
            got = size(B.make_shape(t, d, E, k, f))
            if got == 0 and name == "MXFP8 training":
                break                    # past its limit of 32-bit offsets
            assert got >= last, f"{name}: {last} bytes below {t} tokens, {got} there"
            last = got


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        src, out = os.path.join(tmp, "rules.cpp"), os.path.join(tmp, "rules.so")
        with open(src, "w") as fh:
            fh.write('#include "rules.h"\nextern "C" {\n'
                     'long t_scored(long T, long d, long E) { return route_tile_slices(T, d, E); }\n'
                     'long t_plain(long T, long d, long E) { return route_split_slices(T, d, E); }\n'
                     'long t_direct(long T, long d, long E) { return route_slice_rows(T, d, E); }\n'
                     'long t_rows(long T, long d, long E) { return route_part_rows(T, d, E); } }\n')
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", dispatch.CSRC, "-o", out, src],
                       check=True)
        return ctypes.CDLL(out)


@pytest.mark.skipif(not dispatch.HAVE_CXX, reason="needs a host compiler")
@pytest.mark.parametrize("d,E", [(512, 256), (7168, 256), (256, 128), (2048, 128), (4096, 96), (1280, 200), (1792, 65),
                                 (16384, 129), (7168, 64)])
def test_partial_logits_of_the_slices_that_are_taken(d, E):
    def rule(name, T):
        fn = getattr(_lib(), "t_" + name)
        fn.restype = ctypes.c_long
        return fn(*(ctypes.c_long(v) for v in (T, d, E)))

    most = 0
    for T in range(1, 60_000, 127):
        for s in (rule("scored", T), rule("plain", T)):
            if s > 1:
                assert rule("rows", T) >= s * T
        # every whole tile up to here, and the last one
        for t in (*range(max(T - 127, 1), T), T):
            if t % 128 == 0 or t == T:
                most = max(most, *(n * t for n in (rule("scored", t), rule("plain", t)) if n > 1), 0)
        assert rule("rows", T) <= max(most + 8 * 128, rule("direct", T))
