"""Partial logits of every number of slices, added by threads with one piece of a
row and with two: logits against the oracle, the choice on the GPU's own logits."""
import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from tests import dispatch, score_int_rules as R
from tests.parity import say, to_np
from tests.test_gpu_score import DEV, Case, Run, check, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E", [(1, 256), (16, 256), (5, 65), (1, 24), (130, 128)])
@pytest.mark.parametrize("d", [256, 512, 768, 1280, 2304, 4096, 4352, 7168, 8192, 8448, 12544, 20480])
def test_every_number_of_slices(T, E, d):
    c = Case(T, d, E, 6, "softmax", bias=0.5)
    if dispatch.HAVE_CXX:
        say(f"[gpu] T={T} E={E} d={d}: {R.rule('slices', T, d, E)} slices")
    X, W_r, bias, balance = inputs(c)
    r = Run(c, X, W_r, bias, balance)
    r.route()
    dw = torch.from_numpy(np.random.default_rng(5).standard_normal((T, 6), dtype=np.float32)).to(DEV)
    r.grad(dw)
    torch.cuda.synchronize()
    assert np.abs(to_np(r.logits)[:T] - O.router_logits(X, W_r, bias)).max() <= 1e-4
    check(r, dw)
