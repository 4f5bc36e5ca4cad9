"""The gradient of routing by scores for ids that are listed twice or lie outside
the experts, each form of the scores, every row against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import score_oracle as S
from tests.parity import to_np
from tests.test_gpu_score import DEV, Case, Run, inputs, spread

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_rows_of_repeated_and_wrong_ids(score, renormalise):
    E, k = 24, 4
    c = Case(40, 256, E, k, score, renormalise=renormalise, scale=1.5)
    X, W_r, bias, balance = inputs(c)
    r = Run(c, X, W_r, bias, balance)
    r.route()
    rows = {3: [5, 5, 5, 5], 7: [3, 3, 5, 3], 8: [-1, 24, 1 << 30, -(1 << 31)], 9: [-1, 4, 24, 4], 11: [0, -7, 23, 255],
            38: [256, 1, 2, 3], 39: [24, -1, -1, 2]}
    for t, ids in rows.items():
        r.idx[t] = torch.tensor(ids, dtype=torch.int32, device=DEV)
    dw = torch.randn(c.T, k, device=DEV, generator=torch.Generator(DEV).manual_seed(2))
    r.grad(dw)
    torch.cuda.synchronize()
    Z, idx, _, dZ = r.outputs()
    g = to_np(dw).astype(np.float64)
    live = S.in_play(Z, balance)
    # as in the rounding of the weights, and of sums of k terms each rounded
    rel = (3 * (24 + 2 * spread(Z, live)) + 16 + 2 * k) * 2.0 ** -24
    for t in range(c.T):
        on = (idx[t] >= 0) & (idx[t] < E)
        ref = np.zeros(E)
        if on.any():
            ref = S.score_backward(Z[t:t + 1], balance, idx[t:t + 1, on], g[t:t + 1, on], score, renormalise, 1.5)[0]
        tol = rel[t] * 1.5 * k * np.abs(g[t]).max()
        assert (np.abs(dZ[t] - ref) <= tol).all(), (t, idx[t], np.abs(dZ[t] - ref).max(), tol)
        if score == "sigmoid" or renormalise:
            off = np.ones(E, bool)
            off[idx[t, on]] = False
            assert (dZ[t, off] == 0).all()
    assert (dZ[8] == 0).all()
    r.check_guards()
