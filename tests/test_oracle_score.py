"""Pins of the scored router's oracle: brute force, closed forms, differences."""
import itertools

import numpy as np
import pytest

from oracle import int_oracle as I
from oracle import score_oracle as S

CASES = [dict(score=s, groups=g, top_groups=tg, group_score=m)
         for s in ("softmax", "sigmoid") for g, tg in ((1, 1), (4, 2), (6, 6)) for m in ("max", "pair")]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(map(str, c.values())))
def test_selection_is_the_best_of_all_subsets(c):
    rng = np.random.default_rng(1)
    E, k, n = 12, 3, 12 // c["groups"]
    Z, bal = rng.normal(size=(20, E)), rng.normal(size=E) * 0.2
    idx = S.select(Z, bal, k, **c)
    sc = S.scores(Z, S.in_play(Z, bal), c["score"]) + bal
    for t in range(20):
        def group_value(gs):
            tops = [np.sort(sc[t, g * n:(g + 1) * n])[::-1] for g in gs]
            return [x[0] + x[1] if c["group_score"] == "pair" else x[0] for x in tops]
        kept = max(itertools.combinations(range(c["groups"]), c["top_groups"]),
                   key=lambda gs: sum(group_value(gs)))
        allowed = [e for g in kept for e in range(g * n, (g + 1) * n)]
        best = max(itertools.combinations(allowed, k), key=lambda es: sc[t, list(es)].sum())
        assert list(best) == list(idx[t])


def test_ties_masks_and_empty_rows():
    Z = np.zeros((3, 8))
    Z[1, [0, 3, 5]] = [-np.inf, np.finfo(np.float32).min, np.nan]
    Z[2] = -np.inf
    for score in ("softmax", "sigmoid"):
        assert S.select(Z, None, 3, score).tolist() == [[0, 1, 2], [1, 2, 4], [0, 1, 2]]
        w = S.weights(Z, None, S.select(Z, None, 3, score), score, True, 2.0)
        assert np.allclose(w[:2], 2 / 3) and (w[2] == 0).all()
    bal = np.array([0, 0, -np.inf, 0, 0, 0, 0, 1.0])
    assert S.select(Z[:1], bal, 7, "sigmoid").tolist() == [[0, 1, 3, 4, 5, 6, 7]]
    assert S.select(Z[:1], bal, 8, "sigmoid").tolist() == [list(range(8))]
    assert S.weights(Z[:1], bal, np.arange(8)[None], "sigmoid", False, 1.0)[0, 2] == 0
    # masked experts of kept groups come before any expert of the others
    Z = np.array([[5.0, -np.inf, 4.0, 4.0]])
    assert S.select(Z, None, 2, "sigmoid", 2, 1, "max").tolist() == [[0, 1]]
    assert S.select(Z, None, 2, "sigmoid", 2, 1, "pair").tolist() == [[2, 3]]


def test_closed_forms():
    Z = np.log(np.array([[1.0, 2.0, 5.0]]))
    idx = np.array([[1, 2]])
    assert np.allclose(S.weights(Z, None, idx, "softmax", False, 1.0), [[2 / 8, 5 / 8]])
    assert np.allclose(S.weights(Z, None, idx, "softmax", True, 3.0), [[6 / 7, 15 / 7]])
    assert np.allclose(S.weights(Z, None, idx, "sigmoid", False, 1.0), [[2 / 3, 5 / 6]])
    # scores that underflow keep their ratio
    Z = np.array([[-900.0, -901.0]])
    u = S.weights(Z, None, np.array([[0, 1]]), "sigmoid", True, 1.0)
    assert np.allclose(u, [[1 / (1 + np.exp(-1)), 1 / (1 + np.exp(1))]])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [False, True])
def test_gradient_against_differences(score, renormalise):
    rng = np.random.default_rng(2)
    T, E, k = 6, 9, 4
    Z, dw = rng.normal(size=(T, E)), rng.normal(size=(T, k))
    Z[1, 2] = -np.inf
    bal = np.zeros(E)
    bal[7] = -np.inf
    idx = np.sort(rng.permuted(np.tile(np.arange(E), (T, 1)), axis=1)[:, :k], 1)
    idx[1] = [0, 2, 5, 7]
    loss = lambda z: (S.weights(z, bal, idx, score, renormalise, 1.7) * dw).sum(1)   # noqa: E731
    dZ = S.score_backward(Z, bal, idx, dw, score, renormalise, 1.7)
    step = 1e-6
    for e in range(E):
        up, dn = Z.copy(), Z.copy()
        up[:, e] += step
        dn[:, e] -= step
        assert np.allclose((loss(up) - loss(dn)) / (2 * step), dZ[:, e], atol=1e-8)


def test_codes():
    x = np.array([[1.0, -127.0, 0.5, 126.6, 2.5], [0, 0, 0, 0, 0], [1, np.inf, 0, 0, 0], [1, np.nan, 0, 0, 0]],
                 np.float32)
    q, s = I.quantize_rows(x)
    assert q.tolist() == [[1, -127, 0, 127, 2], [0] * 5, [0] * 5, [0] * 5]
    assert s[0] == 1.0 and s[1] == 0.0 and np.isnan(s[2:]).all()
    rng = np.random.default_rng(0)
    v = rng.normal(size=(50, 300)).astype(np.float32)
    q, s = I.quantize_rows(v)
    assert np.abs(q).max(1).tolist() == [127] * 50
    assert (np.abs(q * s[:, None].astype(np.float64) - v) <= s[:, None] * (0.5 + 1e-5)).all()


def test_int_forward_is_the_layer_up_to_quantisation():
    from oracle import moe_oracle as O
    from paper_2609_36070_amd.workloads import Workload, make_inputs
    w = Workload("q", T=20, d=256, E=4, k=2, f=256, f_s=256)
    inp = make_inputs(w, 3)
    idx = O.topk_select(O.router_logits(inp["X"], inp["W_r"]), 2)
    wt = O.gate_weights(O.router_logits(inp["X"], inp["W_r"]), idx)
    W = {n: inp[n] for n in ("W_gate", "W_up", "W_down", "Wg_s", "Wu_s", "Wd_s")}
    ref = O.moe_forward(inp["X"], W, idx, wt)
    ref = ref[0] if isinstance(ref, tuple) else ref["Y"] if isinstance(ref, dict) else ref
    q = {n: [I.quantize_weights(m) for m in inp[f]] for n, f in (("g", "W_gate"), ("u", "W_up"), ("d", "W_down"))}
    q.update(gs=I.quantize_weights(inp["Wg_s"]), us=I.quantize_weights(inp["Wu_s"]), ds=I.quantize_weights(inp["Wd_s"]))
    Y, tol = I.moe_forward_int(inp["X"], q, idx, wt)
    # three quantisations, each off by at most half of 1/127 of a row's largest
    # value: a few percent of the norm, far from either operand being wrong
    assert np.linalg.norm(Y - ref) <= 0.05 * np.linalg.norm(ref)
    assert np.linalg.norm(tol) <= 0.02 * np.linalg.norm(ref)
