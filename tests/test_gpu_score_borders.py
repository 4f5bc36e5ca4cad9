"""Scored routing where the compared values are closest: the choice is that of
the definition in 64 bits, on the GPU's own logits."""
import numpy as np
import pytest
import torch

from oracle import score_oracle as S
from tests.parity import say, to_np
from tests.test_gpu_score import Case, Run

pytestmark = pytest.mark.gpu


def routed(c, X, W_r, bias, balance):
    r = Run(c, X, W_r, bias, balance)
    r.route()
    torch.cuda.synchronize()
    return to_np(r.logits)[:c.T], to_np(r.idx)[:c.T]


def one_hot_rows(T, d, rows):
    """Tokens whose logits are the rows, exactly, in turn."""
    W_r = np.zeros((d, rows.shape[1]), np.float32)
    W_r[:len(rows)] = rows
    X = np.zeros((T, d), np.float32)
    X[np.arange(T), np.arange(T) % len(rows)] = 1.0
    return X, W_r


@pytest.mark.parametrize("balance", [0.0, 0.25, 1.0, -0.75])
@pytest.mark.parametrize("groups,top_groups", [(1, 1), (8, 3)])
@pytest.mark.parametrize("score,low,high", [("sigmoid", 28.0, 38.0), ("softmax", -38.0, -31.0)])
def test_scores_apart_by_their_last_bits(score, low, high, groups, top_groups, balance):
    """Saturated sigmoids, and softmax scores far below one expert's, beside the
    same balance: values that differ by a few units in the last place of 64 bits,
    the larger ones at the higher ids, and exact ties."""
    E, T = 16, 24
    rng = np.random.default_rng(1)
    rows = np.sort(rng.integers(int(4 * low), int(4 * high), (12, E)), axis=1).astype(np.float32) / 4
    rows[:4] = low + (high - low) / E * np.arange(E) // 1
    if score == "softmax":
        rows[:, 0] = 0.0
    c = Case(T, 256, E, 4, score, groups, top_groups, "pair", balance=balance)
    Z, idx = routed(c, *one_hot_rows(T, 256, rows), None, np.full(E, balance, np.float32))
    assert np.array_equal(Z, rows[np.arange(T) % 12])
    assert np.array_equal(idx, S.select(Z, np.full(E, balance, np.float32), c.k, **c.sel))


def select_rows(Z, balance, c):
    """oracle.score_oracle.select for many rows without masks or exact ties."""
    V = S.ranking_values(Z, balance, c.score, c.groups, c.group_score)
    T, E = V.shape
    if c.groups > 1:
        best = np.sort(V.reshape(T, c.groups, -1), axis=2)
        gs = best[:, :, -1] + (best[:, :, -2] if c.group_score == "pair" else 0.0)
        keep = np.argsort(-gs, axis=1, kind="stable")[:, :c.top_groups]
        kept = np.zeros((T, c.groups), bool)
        np.put_along_axis(kept, keep, True, axis=1)
        V = np.where(np.repeat(kept, E // c.groups, axis=1), V, -np.inf)
    return np.sort(np.argsort(-V, axis=1, kind="stable")[:, :c.k], axis=1)


NEAR = [(score, z, width, bal) for score, z, width in
        (("sigmoid", -8.0, 1e-3), ("sigmoid", -20.0, 1e-3), ("sigmoid", -40.0, 1e-3), ("sigmoid", -60.0, 1e-3),
         ("sigmoid", -87.0, 1e-3), ("sigmoid", -95.0, 1.0), ("sigmoid", 2.0, 1e-4), ("softmax", 0.0, 1e-4),
         ("softmax", 0.0, 4.0))
        for bal in (False, True)]


@pytest.mark.parametrize("score,z,width,bal", NEAR)
def test_close_rows_are_those_of_the_definition(score, z, width, bal):
    """100000 rows of 64 experts whose logits lie close together around z, in
    groups ranked by sums of two, without a balance and with one as small as the
    differences between the scores."""
    say(f"[gpu] {score} {z} {width} {bal}")
    T, d, E = 100_000, 256, 64
    c = Case(T, d, E, 8, score, 8, 4, "pair")
    rng = np.random.default_rng(7)
    X = torch.from_numpy(rng.standard_normal((T, d), dtype=np.float32)).bfloat16().float().numpy()
    W_r = torch.from_numpy(rng.standard_normal((d, E), dtype=np.float32) * np.float32(width / 16)).bfloat16()
    size = 1.0 / (1.0 + np.exp(-z)) if score == "sigmoid" else 1.0 / E
    balance = (rng.standard_normal(E) * size * min(width, 0.1)).astype(np.float32) if bal else None
    Z, idx = routed(c, X, W_r.float().numpy(), np.full(E, z, np.float32), balance)
    wrong = (idx != select_rows(Z, balance, c)).any(1)
    assert wrong.sum() == 0
