"""Scored routing where the compared values are closest: the choice is that of
the definition in 64 bits, on the GPU's own logits."""
import numpy as np
import pytest
import torch

from oracle import score_oracle as S
from tests.parity import to_np
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
