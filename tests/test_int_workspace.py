"""Workspace of the int8 forward across its paths: small batches hold their
experts' outputs in fp32, larger ones in bf16, and the size still never falls."""
import ctypes
import os
import subprocess
import tempfile

import pytest

from paper_2609_36070_amd import binding as B
from tests import dispatch
from tests.score_int_rules import rule

LAYERS = [(2048, 128, 8, 768, 0), (7168, 8, 8, 2048, 2048), (4096, 32, 8, 1536, 0), (256, 4, 1, 256, 256),
          (256, 200, 16, 256, 0), (512, 1, 1, 256, 1024), (1024, 16, 15, 256, 256)]


@pytest.mark.parametrize("d,E,k,f,fs", LAYERS)
def test_sizes_never_fall_and_hold_the_outputs(d, E, k, f, fs):
    last = 0
    for t in [*range(0, 700), *range(700, 30_000, 97)]:
        got = B.moe_int_workspace_bytes(B.make_shape(t, d, E, k, f, fs))
        assert got >= max(last, 1)
        last = got
        if dispatch.HAVE_CXX and rule("tiles", t, d, E, k, f, fs):
            # codes and scales of X and H, H, and the outputs in fp32
            need = t * d + t * k * (4 * f + f + 4 * d) + (t * (4 * fs + fs + 4 * d) if fs else 0)
            assert got >= need


@pytest.mark.skipif(not dispatch.HAVE_CXX, reason="needs a host compiler")
def test_the_bound_of_small_batches_holds():
    with tempfile.TemporaryDirectory() as tmp:
        src, out = os.path.join(tmp, "r.cpp"), os.path.join(tmp, "r.so")
        with open(src, "w") as fh:
            fh.write('#include "rules.h"\n'
                     'extern "C" long most(long E, long k) { return skinny_i8_max_tokens(E, k); }\n')
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", dispatch.CSRC, "-o", out, src],
                       check=True)
        most = ctypes.CDLL(out).most
        most.restype = ctypes.c_long
        for E in (1, 2, 3, 8, 12, 31, 128, 256):
            for k in {1, 2, 3, 7, 8, 16, E}:
                if k > min(E, 16):
                    continue
                m = most(ctypes.c_long(E), ctypes.c_long(k))
                for f in (256, 1024, 8192):
                    for fs in (0, 256, 4096):
                        assert not any(rule("tiles", t, 512, E, k, f, fs) for t in range(m + 1, m + 400, 7))
