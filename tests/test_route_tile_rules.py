"""Slices of the tile router's d axis: the rule's count is near the fastest one
where every count was measured (us of the router by scores on one MI355X, by
slices; CPU: the rule alone)."""
import ctypes
import functools
import os
import subprocess
import tempfile

import pytest

from tests import dispatch

pytestmark = pytest.mark.skipif(not dispatch.HAVE_CXX, reason="needs a host compiler")


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as tmp:
        src, out = os.path.join(tmp, "rules.cpp"), os.path.join(tmp, "rules.so")
        with open(src, "w") as fh:
            fh.write('#include "rules.h"\n'
                     'extern "C" long t_slices(long T, long d, long E) { return route_tile_slices(T, d, E); }\n')
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", dispatch.CSRC, "-o", out, src],
                       check=True)
        return ctypes.CDLL(out)


def slices(T, d, E):
    fn = _lib().t_slices
    fn.restype = ctypes.c_long
    return fn(*(ctypes.c_long(v) for v in (T, d, E)))


@pytest.mark.parametrize("T,d,E,us", [
    (9000, 512, 256, {1: 31.5, 2: 29.7, 4: 37, 8: 42.6}),
    (12000, 512, 256, {1: 33.9, 2: 31.8, 4: 40.2, 8: 48.7}),
    (65536, 512, 256, {1: 92.4, 2: 114, 4: 157, 8: 276}),
    (4200, 256, 128, {1: 16.8, 2: 15.7, 4: 17.5}),
    (24000, 256, 128, {1: 23.8, 2: 29.8, 4: 35.2}),
    (8192, 1024, 256, {1: 36.7, 2: 28.3, 4: 30.7, 8: 39.8}),
    (16384, 2048, 128, {1: 31.9, 2: 28.3, 4: 36.2, 8: 47.3}),
    (16384, 2048, 256, {1: 53.6, 2: 44.8, 4: 54.4, 8: 72.9}),
    (20000, 2048, 128, {1: 33.8, 2: 39.1, 4: 43.2, 8: 53.1}),
    (4200, 7168, 256, {1: 109, 2: 64.4, 4: 44.8, 7: 37.7, 8: 51.3}),
    (9000, 7168, 200, {1: 112, 2: 69.5, 4: 77.3, 7: 64.8, 8: 74.9}),
    (33000, 7168, 256, {1: 263, 2: 225, 4: 221, 7: 253, 8: 264}),
    (40000, 7168, 128, {1: 181, 2: 164, 4: 171, 7: 198, 8: 201}),
    (12000, 4096, 96, {1: 43.2, 2: 31.9, 4: 41.4, 8: 44.7}),
    (6000, 768, 256, {1: 30.4, 2: 25.8, 3: 26.2, 4: 28.4, 6: 32.9}),
    (32700, 4096, 200, {1: 106, 2: 123, 4: 138, 8: 197}),
    (65536, 7168, 256, {1: 323, 2: 363, 4: 402, 7: 483, 8: 492}),
    (50000, 1536, 128, {1: 59.9, 2: 73.2, 3: 77, 4: 87.7, 6: 104, 8: 121}),
    (16384, 1024, 200, {1: 41.6, 2: 37.7, 4: 46, 8: 61.7}),
    (2100, 2048, 200, {1: 43, 2: 28.2, 4: 24.4, 8: 27.1}),
    (16384, 7168, 256, {1: 121, 2: 89.3, 4: 99.1, 7: 126, 8: 119}),
    (24000, 4096, 256, {1: 88.3, 2: 102, 4: 106, 8: 133}),
])
def test_slices_near_the_fastest(T, d, E, us):
    assert us[slices(T, d, E)] <= 1.15 * min(us.values())


def test_slices_divide_the_chunks():
    for E in (65, 100, 128, 256):
        for d in (256, 768, 1280, 1792, 7168, 16384):
            for T in (1, 129, 1000, 5000, 20000, 33000, 100_000, 1 << 24):
                s = slices(T, d, E)
                assert 1 <= s <= 8 and d // 64 % s == 0
    assert slices(1000, 7168, 64) == 0
