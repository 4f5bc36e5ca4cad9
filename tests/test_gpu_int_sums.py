"""The int8 experts' outputs in small batches: summed in fp32 and rounded once, so
that no output is off by more than half a bf16 step of its own, beside the codes
that the 32-bit evaluation of the activation can move."""
import numpy as np
import pytest
import torch

from oracle import int_oracle as I
from paper_2609_36070_amd.layer import DeviceLayer
from paper_2609_36070_amd.workloads import Workload, make_inputs
from tests import dispatch, score_int_rules as R
from tests.parity import say, to_np
from tests.test_gpu_int import oracle_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w", [
    Workload("one token", T=1, d=512, E=8, k=4, f=256, f_s=256),
    Workload("few tokens", T=7, d=768, E=9, k=3, f=512),
    Workload("sixteen", T=16, d=1024, E=12, k=4, f=512, f_s=256),
    Workload("forty", T=40, d=512, E=16, k=8, f=256),
    Workload("dense and shared", T=61, d=512, E=4, k=4, f=512, f_s=512),
    Workload("dense, two tiles of rows", T=150, d=256, E=4, k=4, f=256, f_s=256),
    Workload("several tiles of an expert", T=300, d=256, E=8, k=2, f=256, bias_std=2.0),
    Workload("many experts", T=257, d=256, E=128, k=8, f=256, f_s=256),
], ids=lambda w: w.name)
def test_one_rounding(w):
    say(f"[gpu] {w.name}")
    inp = make_inputs(w, 31)
    L = DeviceLayer(w, inp, int8=True)
    if dispatch.HAVE_CXX:
        assert R.layer("token", w) or R.layer("tiles", w)      # the path of small batches
    L.step_int()
    torch.cuda.synchronize()
    q, idx, wt = oracle_weights(w, inp), to_np(L.topk_idx), to_np(L.topk_w).astype(np.float64)
    xq, xs = I.quantize_rows(inp["X"])
    Y, off = np.zeros((w.T, w.d)), np.zeros((w.T, w.d))

    def add(t, weight, g, u, d):
        y, a, h, hq, hs = I.ffn_rows(xq[t], xs[t], g, u, d)
        moved = I.tie_codes(a, h, hs, 0.0).astype(np.float64) @ np.abs(d[0]).T.astype(np.float64)
        moved *= hs[:, None].astype(np.float64) * d[1].astype(np.float64)
        # the scale hs carries the error of the largest value, in 32 bits
        moved += (np.abs(y) + moved) * 200 * 2.0 ** -24
        np.add.at(Y, t, weight[:, None] * y)
        np.add.at(off, t, np.abs(weight)[:, None] * (moved + np.abs(y) * (w.k + 3) * 2.0 ** -24))

    for e in range(w.E):
        t, s = np.nonzero(idx == e)
        if len(t):
            add(t, wt[t, s], q["g"][e], q["u"][e], q["d"][e])
    if w.f_s:
        add(np.arange(w.T), np.ones(w.T), q["gs"], q["us"], q["ds"])
    err = np.abs(to_np(L.Y) - Y)
    assert (err <= off + (np.abs(Y) + off) * 2.0 ** -8).all(), (err / (off + np.abs(Y) * 2.0 ** -8 + 1e-30)).max()
