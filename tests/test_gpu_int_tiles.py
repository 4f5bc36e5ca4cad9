"""The int8 experts' outputs in large batches, held in fp16 with a power of two per
expert until they are summed: off by half an fp16 step each, whatever the scales."""
import numpy as np
import pytest
import torch

from oracle import int_oracle as I
from paper_2609_36070_amd.layer import DeviceLayer
from paper_2609_36070_amd.workloads import Workload, make_inputs, to_bf16
from tests import dispatch, score_int_rules as R
from tests.parity import say, to_np
from tests.test_gpu_int import oracle_weights

pytestmark = pytest.mark.gpu


def reference(w, inp, idx, wt, kf):
    """Y in float64, and what an implementation may be off by before Y is rounded."""
    q = oracle_weights(w, inp)
    xq, xs = I.quantize_rows(inp["X"])
    Y, off = np.zeros((w.T, w.d)), np.zeros((w.T, w.d))

    def add(t, weight, g, u, d, K):
        y, a, h, hq, hs = I.ffn_rows(xq[t], xs[t], g, u, d)
        moved = I.tie_codes(a, h, hs, 0.0).astype(np.float64) @ np.abs(d[0]).T.astype(np.float64)
        moved *= hs[:, None].astype(np.float64) * d[1].astype(np.float64)
        moved += (np.abs(y) + moved) * 200 * 2.0 ** -24     # the scale, from 32-bit values
        # half an fp16 step: 2^-11 of the value; near 0, 2^(dot - 39) of the largest
        # channel's unit, the products of K codes being at most 2^dot
        dot = int(np.ceil(np.log2(127 * 127 * K)))
        unit = hs[:, None].astype(np.float64) * np.nanmax(d[1]).astype(np.float64)
        step = np.maximum((np.abs(y) + moved) * 2.0 ** -11, unit * 2.0 ** (dot - 39))
        np.add.at(Y, t, weight[:, None] * y)
        np.add.at(off, t, np.abs(weight)[:, None] * (moved + step + np.abs(y) * (w.k + 5) * 2.0 ** -24))

    for e in range(w.E):
        t, s = np.nonzero(idx == e)
        if len(t):
            add(t, wt[t, s], q["g"][e], q["u"][e], q["d"][e], w.f)
    if w.f_s:
        add(np.arange(w.T), np.ones(w.T), q["gs"], q["us"], q["ds"], w.f_s)
    return Y, off


def check(w, inp, L, rows=slice(None)):
    if dispatch.HAVE_CXX:
        assert not R.layer("token", w) and not R.layer("tiles", w)      # the tile products
    Y, off = reference(w, inp, to_np(L.topk_idx), to_np(L.topk_w).astype(np.float64), w.f)
    err, tol = np.abs(to_np(L.Y) - Y)[rows], (off + (np.abs(Y) + off) * 2.0 ** -8 + 1e-38)[rows]
    say(f"  worst share of the bound {(err / tol).max():.3f}")
    assert (err <= tol).all()
    # and by far less than with the outputs in bf16, whose step is eight times as long
    small = to_np(torch.from_numpy(Y).bfloat16()).astype(np.float64) - Y
    assert np.sqrt((err ** 2).mean()) <= 1.1 * np.sqrt((small[rows] ** 2).mean()) + np.sqrt((off[rows] ** 2).mean())


SHAPES = [
    Workload("ragged", T=777, d=512, E=16, k=4, f=768, f_s=1024),
    Workload("skewed", T=600, d=256, E=8, k=2, f=512, bias_std=2.0),
    Workload("dense", T=400, d=256, E=3, k=3, f=256, f_s=256),
    Workload("one expert", T=300, d=1024, E=1, k=1, f=2304),
    Workload("several tiles per workgroup", T=700, d=2560, E=16, k=8, f=256, f_s=512),
    Workload("long rows", T=500, d=8448, E=2, k=2, f=512),
]


@pytest.mark.parametrize("w", SHAPES, ids=lambda w: w.name)
def test_outputs(w):
    say(f"[gpu] {w.name}")
    inp = make_inputs(w, 41)
    L = DeviceLayer(w, inp, int8=True)
    L.step_int()
    torch.cuda.synchronize()
    check(w, inp, L)


def test_scales_far_apart():
    """Experts and channels whose scales differ by up to 2^60, channels of zeros and
    tiny tokens: every output to its own size."""
    w = Workload("far apart", T=450, d=512, E=6, k=2, f=256, f_s=256)
    say(f"[gpu] {w.name}")
    inp = make_inputs(w, 43)
    inp["W_down"][1] *= np.float32(2.0 ** 40)
    inp["W_down"][2] *= np.float32(2.0 ** -60)
    inp["W_down"][3] = 0.0
    for e in (0, 1, 4):
        inp["W_down"][e][:, 7] *= np.float32(2.0 ** 12)
        inp["W_down"][e][:, 9] *= np.float32(2.0 ** -15)
        inp["W_down"][e][:, 11] = 0.0
    inp["Wd_s"][:, 13] *= np.float32(2.0 ** -20)
    inp["X"][5] = 0.0
    inp["X"][6] *= np.float32(2.0 ** -40)
    inp["X"] = to_bf16(inp["X"])
    L = DeviceLayer(w, inp, int8=True)
    L.step_int()
    torch.cuda.synchronize()
    Y, off = reference(w, inp, to_np(L.topk_idx), to_np(L.topk_w).astype(np.float64), w.f)
    err, tol = np.abs(to_np(L.Y) - Y), off + (np.abs(Y) + off) * 2.0 ** -8 + 1e-38
    assert np.isfinite(to_np(L.Y)).all() and (err <= tol).all(), (err / tol).max()


def test_routes_without_a_place_and_stale_workspace():
    """Weights go by slot and outputs by plan position: ids outside the experts leave
    slots without one, whatever the workspace held."""
    w = Workload("holes", T=500, d=256, E=8, k=3, f=256, f_s=256)
    inp = make_inputs(w, 44)
    L = DeviceLayer(w, inp, int8=True)
    L.ws.fill_(0xFF)                       # NaN wherever nothing was written
    L.route()
    bad = torch.randperm(w.T, generator=torch.Generator().manual_seed(1))[:200]
    L.topk_idx[bad[:100], 1] = -1
    L.topk_idx[bad[50:150], 2] = 8
    L.topk_idx[bad[150:]] = 1 << 20
    L.plan()
    L.forward_int()
    torch.cuda.synchronize()
    idx, wt = to_np(L.topk_idx), to_np(L.topk_w).astype(np.float64)
    Y, off = reference(w, inp, idx, wt, w.f)
    assert (np.abs(to_np(L.Y) - Y) <= off + (np.abs(Y) + off) * 2.0 ** -8 + 1e-38).all()


def test_nan_channels_leave_the_others_their_range():
    w = Workload("nan channel", T=450, d=256, E=4, k=2, f=256, f_s=256)
    inp = make_inputs(w, 45)
    L = DeviceLayer(w, inp, int8=True)
    L.step_int()
    torch.cuda.synchronize()
    clean = L.Y.clone()
    L.W_down[1, 3, 20], L.Wd_s[5, 30] = float("nan"), float("inf")
    L.quantize_int()
    L.forward_int()
    torch.cuda.synchronize()
    hit = (L.topk_idx == 1).any(1)
    assert torch.isnan(L.Y[hit, 20]).all() and torch.isnan(L.Y[:, 30]).all()
    keep = torch.ones_like(clean, dtype=torch.bool)
    keep[hit, 20] = False
    keep[:, 30] = False
    assert torch.equal(L.Y[keep], clean[keep])
