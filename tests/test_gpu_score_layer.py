"""The backward passes of a layer routed by scores: the router's gradient from the
layer's own dL/dw, and every other gradient against the backward it shares them with."""
import numpy as np
import pytest
import torch

from oracle import score_oracle as S
from paper_2609_36070_amd import binding as B
from paper_2609_36070_amd.layer import DeviceLayer
from paper_2609_36070_amd.workloads import Workload, make_inputs
from tests.parity import assert_close, say, to_np
from tests.test_gpu_score import LAYERS

pytestmark = pytest.mark.gpu

MORE = [
    (Workload("scored mx, dense", T=130, d=512, E=4, k=4, f=256, f_s=256, backward=True),
     B.routing("softmax", renormalise=False, scale=2.0), dict(mx=True)),
    (Workload("scored mx weight gradients", T=300, d=256, E=8, k=2, f=256, f_s=512, backward=True),
     B.routing("sigmoid", renormalise=False), dict(mx=True, mx_wgrad=True)),
    (Workload("scored one token", T=1, d=256, E=8, k=3, f=256, backward=True), B.routing("sigmoid", 4, 3), dict()),
    (Workload("scored many experts", T=700, d=512, E=96, k=6, f=256, backward=True),
     B.routing("softmax", 8, 3, "pair"), dict()),
]


@pytest.mark.parametrize("w,routing,kw", LAYERS + MORE, ids=lambda v: getattr(v, "name", ""))
def test_gradients(w, routing, kw):
    say(f"[gpu] {w.name}")
    balance = (np.random.default_rng(4).standard_normal(w.E) * 0.1).astype(np.float32)
    L = DeviceLayer(w, dict(make_inputs(w, 21), balance=balance), routing=routing, **kw)
    (L.step_mx if L.mx else L.step)()
    torch.cuda.synchronize()
    names = ["dW_gate", "dW_up", "dW_down"] + (["dWg_s", "dWu_s", "dWd_s"] if w.f_s else [])
    first = {n: getattr(L, n).clone() for n in names + ["dX", "dZ", "dW_r"]}
    Z, idx = to_np(L.logits), to_np(L.topk_idx)
    wts = dict(score=B.SCORES[routing.score], renormalise=bool(routing.renormalise), scale=routing.scale)

    dZ = to_np(first["dZ"]).astype(np.float64)
    if L.ring_rows is None:
        # the layer's own dL/dw: what the router's gradient starts from.  Bound as in
        # the operator's own test: the weights' rounding and sums of k terms
        read = L.mx_ws_tensor if L.mx else L.ws_tensor
        dg = to_np(read(B.WS_DG, torch.float32, (w.T * w.k,)))[to_np(L.route_pos)].reshape(w.T, w.k).astype(np.float64)
        ref = S.score_backward(Z, balance, idx, dg, **wts)
        spread = np.ptp(Z.astype(np.float64), axis=1)[:, None]
        tol = (3 * (24 + 2 * spread) + 16 + 2 * w.k) * 2.0 ** -24 * routing.scale * np.abs(dg).max(1, keepdims=True)
        assert (np.abs(dZ - ref) <= tol).all(), (np.abs(dZ - ref) / tol).max()
    # dW_r = X^T dZ in fp32 sums of T terms, dZ in two bf16 parts: the first is off by
    # half a step, 2^-8 of dZ, the second by 2^-8 of that rest
    X = to_np(L.X).astype(np.float64)
    tol = (np.abs(X).T @ np.abs(dZ)) * (2.0 ** -16 + (2 * w.T + 4) * 2.0 ** -24)
    assert (np.abs(to_np(first["dW_r"]) - X.T @ dZ) <= tol + 1e-12).all()

    # the same call with the other router's gradient: the experts' gradients bit for
    # bit, dX but for its router term (both sides round to bf16)
    L.routing = None
    if L.ring_rows is not None:
        L.forward()        # a ring's backward follows a forward: it uses up the last window
    (L.backward_mx if L.mx else L.backward)()
    torch.cuda.synchronize()
    for n in names:
        assert torch.equal(first[n], getattr(L, n)), n
    a, b = to_np(first["dX"]).astype(np.float64), to_np(L.dX).astype(np.float64)
    term = (dZ - to_np(L.dZ).astype(np.float64)) @ to_np(L.W_r).astype(np.float64).T
    assert (np.abs(a - b - term) <= 2.0 ** -8 * (np.abs(a) + np.abs(b)) + 2e-4 * np.abs(term).max() + 1e-6).all()
    assert_close("router term", a - b, term, max(2e-2, 4 * 2.0 ** -8 * np.abs(a).max() / np.abs(term).max()))
