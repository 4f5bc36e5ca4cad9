"""Pins of the residual join's oracle: the generator's published outputs, norms
in closed form, and gradients against differences (CPU)."""
import itertools

import numpy as np
import pytest

from oracle import join_oracle as J


@pytest.mark.parametrize("counter,key,words", [
    ((0,) * 4, (0,) * 2, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_known_answers(counter, key, words):
    """The known-answer vectors that its authors publish."""
    assert tuple(int(w) for w in J.philox(counter, key)) == words


def test_mask_layout_and_share():
    seed, offset = (0xA4093822) | (0x299F31D0 << 32), (5 << 32) | 9
    m = J.keep_mask(7, 48, 0.25, seed, offset)
    w = J.philox((3, 6, 9, 5), (seed & J.M32, seed >> 32))
    bits = [int(w[i // 2]) >> (16 * (i % 2)) & 0xFFFF for i in range(8)]
    assert np.array_equal(m[6, 24:32], [(b >= 16384) / 0.75 for b in bits])
    assert (J.keep_mask(3, 8, 0.0, 1, 2) == 1).all()
    big = J.keep_mask(400, 800, 0.1, 12345, 7)
    # 320000 draws with p = 6554 / 65536: five deviations of the share
    assert abs((big == 0).mean() - 6554 / 65536) < 5 * np.sqrt(0.1 * 0.9 / big.size)
    assert abs(big.max() - 65536 / (65536 - 6554)) < 1e-12


def test_norms_in_closed_form():
    v = np.array([[3.0, -3.0, 3.0, -3.0, 1.0, 1.0, 1.0, 1.0]])
    assert np.allclose(J.norm("rms", v, eps=0.0), v / np.sqrt(5.0))
    assert np.allclose(J.norm("layer", v, np.full(8, 2.0), np.full(8, 1.0), eps=0.0),
                       1.0 + 2.0 * (v - 0.5) / np.sqrt(4.75))
    assert np.allclose(J.norm("rms", np.zeros((2, 8)), eps=1e-6), 0.0)
    assert J.norm("none", v) is v


@pytest.mark.parametrize("y_norm,r_norm,block", [
    *[(a, b, True) for a, b in itertools.product(("none", "rms", "layer"), repeat=2)],
    ("none", "rms", False), ("none", "layer", False)])
def test_gradient_against_differences(y_norm, r_norm, block):
    rng = np.random.default_rng(3)
    T, d, eps, scale = 3, 16, 1e-3, 0.7
    x, y = rng.standard_normal((T, d)), rng.standard_normal((T, d)) + 0.3
    p = {n: 1.0 + 0.3 * rng.standard_normal(T if n == "token_gate" else d) for n in J.PARAMS}
    if y_norm == "none":
        p["y_weight"] = p["y_bias"] = None
    if r_norm == "none":
        p["r_weight"] = p["r_bias"] = None
    if not block:
        p["gate"] = p["token_gate"] = None
    keep = J.keep_mask(T, d, 0.3, 99, 1) if block else 1.0
    gr, gh = rng.standard_normal((T, d)), rng.standard_normal((T, d))

    def loss(x, y, p):
        r = J.join_r(x, y, p, y_norm, eps, scale, keep) if block else x
        return (gr * r).sum() + (gh * J.norm(r_norm, r, p["r_weight"], p["r_bias"], eps)).sum()

    r = J.join_r(x, y, p, y_norm, eps, scale, keep) if block else x
    st = np.stack((*J.stats(y_norm, y, eps), *J.stats(r_norm, r, eps)), 1)
    g = J.backward(y if block else None, r, st, p, gr, gh, y_norm, r_norm, scale, keep)
    for name in ("x", *(["y"] if block else []), *[n for n in J.PARAMS if p[n] is not None]):
        base = {"x": x, "y": y}.get(name, p.get(name))
        got = g["d" + name if name in "xy" else name]
        for at in [np.unravel_index(i, base.shape) for i in rng.choice(base.size, min(base.size, 12), False)]:
            h = 1e-5
            diff = []
            for s in (h, -h):
                v = base.copy()
                v[at] += s
                args = {"x": (v, y, p), "y": (x, v, p)}.get(name, (x, y, {**p, name: v}))
                diff.append(loss(*args))
            # the truncation of a central difference is of order h^2 = 1e-10, its rounding of
            # order 1e-16 * |loss| / h = 1e-9
            assert abs((diff[0] - diff[1]) / (2 * h) - got[at]) < 1e-6 * (1 + abs(got[at])), (name, at)


def test_magnitudes_bound_the_gradients():
    rng = np.random.default_rng(5)
    T, d = 4, 24
    y, r, dr, dh = (rng.standard_normal((T, d)) for _ in range(4))
    p = {n: rng.standard_normal(T if n == "token_gate" else d) for n in J.PARAMS}
    st = np.stack((*J.stats("layer", y, 1e-6), *J.stats("rms", r, 1e-6)), 1)
    g, m = (J.backward(y, r, st, p, dr, dh, "layer", "rms", -0.5, mag=q) for q in (False, True))
    assert set(g) == set(m)
    for n in g:
        assert (np.abs(g[n]) <= m[n] * (1 + 1e-12)).all(), n
