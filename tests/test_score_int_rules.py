"""The size rules of routing by scores and of the int8 experts choose the faster
side where both were measured (us on one MI355X; CPU: the rules alone)."""
import pytest

from tests import dispatch
from tests.score_int_rules import rule

pytestmark = pytest.mark.skipif(not dispatch.HAVE_CXX, reason="needs a host compiler")


@pytest.mark.parametrize("T,d,E,k,f,fs,stream,tile", [
    (16, 2048, 128, 8, 768, 0, 87.6, 127), (256, 2048, 128, 8, 768, 0, 162, 189), (768, 2048, 128, 8, 768, 0, 191, 205),
    (1536, 2048, 128, 8, 768, 0, 270, 251), (192, 4096, 32, 8, 1536, 0, 175, 199), (384, 4096, 32, 8, 1536, 0, 244, 210),
    (256, 7168, 16, 4, 2048, 0, 208, 213), (384, 7168, 16, 4, 2048, 0, 266, 220),
    (800, 2048, 200, 4, 768, 2048, 262, 345),
    # few tiles
    (384, 4096, 8, 2, 1536, 0, 87, 91), (768, 4096, 8, 2, 1536, 0, 113, 97), (384, 2048, 16, 4, 768, 0, 52, 58),
    (768, 2048, 16, 4, 768, 0, 76, 65), (128, 7168, 8, 8, 2048, 2048, 172, 239), (192, 7168, 8, 8, 2048, 2048, 223, 246),
    (256, 7168, 8, 8, 2048, 2048, 303, 254), (192, 5120, 12, 12, 512, 1024, 101, 173), (384, 2048, 8, 8, 768, 0, 65, 58),
])
def test_streaming_or_tile_products(T, d, E, k, f, fs, stream, tile):
    assert bool(rule("tiles", T, d, E, k, f, fs)) == (stream < tile)


@pytest.mark.parametrize("T,d,E,k,f,eight,four", [
    (40, 2048, 48, 8, 1024, 79, 88), (40, 5120, 48, 8, 1024, 166, 178), (40, 2048, 28, 8, 1536, 74, 82),
    (40, 2048, 48, 8, 768, 73, 76), (64, 4096, 32, 8, 1536, 146, 159), (64, 2048, 128, 8, 768, 148, 140),
    (40, 2048, 64, 8, 1024, 102, 97), (14, 2048, 48, 8, 768, 61, 58), (14, 5120, 48, 8, 768, 130, 120),
    (4, 4096, 64, 4, 512, 41.4, 36.6), (64, 7168, 64, 8, 2048, 539, 529),
])
def test_waves_of_the_up_product(T, d, E, k, f, eight, four):
    assert rule("up_waves", T, d, E, k, f, 0) == (8 if eight < four else 4)


def test_waves_fit_the_columns():
    for E, k, fs in ((1, 1, 0), (8, 8, 0), (8, 8, 2048), (12, 12, 256), (16, 16, 512), (32, 4, 256), (200, 8, 1024)):
        for T in (1, 2, 16, 17, 64):
            for f in (256, 768, 1280, 2048):
                if not rule("tiles", T, 512, E, k, f, fs):
                    continue
                up, down = (rule(n, T, 512, E, k, f, fs) for n in ("up_waves", "down_waves"))
                assert 4 <= up <= 15 and down == 4
                if not rule("up_dense", T, 512, E, k, f, fs):
                    assert f % (8 * up) == 0 and fs % (8 * up) == 0


def test_one_token():
    assert rule("token", 1, 8192, 64, 8, 2048, 2048) == 1
    assert rule("token", 2, 2048, 64, 8, 2048, 0) == 0
    assert rule("token", 1, 8448, 64, 8, 2048, 0) == 0             # the token's codes
    assert rule("token", 1, 2048, 64, 16, 3328, 256) == 1          # sixteen rows of H
    assert rule("token", 1, 2048, 64, 16, 3584, 256) == 0
    assert rule("token", 1, 2048, 64, 1, 1024, 256 * 111) == 1 and rule("token", 1, 2048, 64, 1, 1024, 256 * 112) == 0


@pytest.mark.parametrize("T,d,E,here,others", [
    (1, 7168, 256, 11.5, 22.4), (512, 7168, 256, 21.5, 27), (1500, 7168, 256, 38, 29), (1024, 4096, 256, 20.7, 21.1),
    (1500, 4096, 256, 26, 22.5), (3000, 2048, 256, 26, 23), (1024, 7168, 128, 16.5, 18.2), (1500, 7168, 128, 20.7, 18.6),
    (4096, 2048, 128, 16.4, 19), (6000, 2048, 128, 23.6, 20), (1024, 7168, 64, 14.5, 42), (6000, 7168, 64, 50, 73),
    (8192, 7168, 64, 59, 53), (1, 4096, 32, 8, 15), (8192, 4096, 32, 22, 28), (16384, 4096, 32, 49, 41),
    (4096, 2048, 16, 14.3, 16), (8192, 2048, 16, 19.4, 18.5),
])
def test_router_slices(T, d, E, here, others):
    assert bool(rule("slices", T, d, E)) == (here < others)


@pytest.mark.parametrize("d,E", [(256, 1), (256, 16), (1024, 96), (7168, 256), (2048, 33), (16384, 64), (7168, 200), (256, 64), (512, 32)])
def test_partial_logits_fit_their_rows(d, E):
    """The partial sums of every batch up to T tokens fit what T tokens reserve."""
    rows = 0
    for T in [*range(0, 200), *range(200, 5000, 13), 4096, 4097, 8192, 8193, 16384, 100000]:
        S = rule("slices", T, d, E)
        assert 0 <= S <= rule("slice_steps", d, E)
        assert rule("slice_rows", T, d, E) >= rows
        rows = rule("slice_rows", T, d, E)
        assert S <= 1 or S * T <= rows
