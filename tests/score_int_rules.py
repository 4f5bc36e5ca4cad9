"""The size rules of routing by scores and of the int8 experts (csrc/rules.h),
compiled for the host, so that a test can state which path its shapes take."""
import ctypes
import functools
import os
import subprocess
import tempfile

from tests.dispatch import CSRC

SRC = """
#include "rules.h"
extern "C" {
long t_token(long T, long d, long E, long k, long f, long fs) { return token_i8(T, d, k, f, fs); }
long t_tiles(long T, long d, long E, long k, long f, long fs) { return skinny_i8_tiles(T, k, E, f, fs); }
long t_up_dense(long T, long d, long E, long k, long f, long fs) {
    return k == E && T <= 16 * skinny_i8_tiles(T, k, E, f, fs); }
long t_up_waves(long T, long d, long E, long k, long f, long fs) {
    const long bm = 16 * skinny_i8_tiles(T, k, E, f, fs);
    return skinny_i8_waves(T, k, E, f, fs, bm, true, k == E && T <= bm); }
long t_down_waves(long T, long d, long E, long k, long f, long fs) {
    return skinny_i8_waves(T, k, E, d, fs > 0 ? d : 0, 16 * skinny_i8_tiles(T, k, E, f, fs), false, false); }
long t_slices(long T, long d, long E) { return route_slices(T, d, E); }
long t_slice_rows(long T, long d, long E) { return route_slice_rows(T, d, E); }
long t_slice_steps(long d, long E) { return route_slice_steps(d, E); }
}
"""


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        src, out = os.path.join(tmp, "rules.cpp"), os.path.join(tmp, "rules.so")
        with open(src, "w") as fh:
            fh.write(SRC)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, "-o", out, src], check=True)
        lib = ctypes.CDLL(out)
    for n in ("token", "tiles", "up_dense", "up_waves", "down_waves", "slices", "slice_rows", "slice_steps"):
        getattr(lib, "t_" + n).restype = ctypes.c_long
    return lib


def rule(name, *args):
    """One rule on its sizes: (T, d, E, k, f, fs) for the experts, (T, d, E) for the router."""
    return getattr(_lib(), "t_" + name)(*(ctypes.c_long(a) for a in args))


def layer(name, w):
    return rule(name, w.T, w.d, w.E, w.k, w.f, w.f_s)
