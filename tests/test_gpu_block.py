"""A layer between the norms of a residual block: the join's calls and the layer's together, forward
and backward, against the float64 oracles with the GPU's own selection."""
import numpy as np
import pytest
import torch

from oracle import join_oracle as J
from oracle import moe_oracle as O
from paper_2609_36070_amd import binding as B
from paper_2609_36070_amd.layer import DeviceBlock, DeviceLayer
from paper_2609_36070_amd.workloads import Workload, make_inputs, to_bf16
from tests.parity import REL_TOL, assert_close, say, to_np, weights_dict

pytestmark = pytest.mark.gpu
EPS = 1e-6


def f64(t):
    return to_np(t).astype(np.float64)


def make(T, stream, y_norm, r_norm, drop, backward, d=512, E=8, k=2, f_s=256, seed=0, **kw):
    w = Workload("block", T=T, d=d, E=E, k=k, f=256, f_s=f_s, bias_std=0.5, backward=backward)
    inp = make_inputs(w, seed)
    inp["dY"] = None
    rng = np.random.default_rng(seed + 1)
    draw = lambda n: 1 + 0.2 * rng.standard_normal(n)   # noqa: E731
    p = dict(in_weight=draw(d), gate=draw(d), token_gate=draw(T), r_weight=draw(d))
    if r_norm == "layer":
        p["r_bias"] = draw(d)
    if y_norm != "none":
        p["y_weight"] = draw(d)
    block = DeviceBlock(w, inp, p, stream, "rms", y_norm, r_norm, EPS, 0.5, drop, seed=77, **kw)
    return w, inp, {n: np.asarray(v, np.float32).astype(np.float64) for n, v in p.items()}, block


def reference(w, inp, p, block, y_norm, r_norm, drop, dr=None, dh=None):
    """The whole block in float64 on the GPU's selection; with dr and dh its gradients."""
    x = f64(block.x)
    W = weights_dict(inp, True)
    idx = to_np(block.layer.topk_idx)
    h0 = J.norm("rms", x, p["in_weight"], None, EPS)
    Z = h0 @ inp["W_r"].astype(np.float64) + inp["bias"]
    wt = O.gate_weights(Z, idx)
    y = O.moe_forward_dense(h0, W, idx, wt)
    keep = J.keep_mask(w.T, w.d, drop, 77, int(block.rng[1]) if drop else 0)
    r = J.join_r(x, y, p, y_norm, EPS, 0.5, keep)
    out = dict(h0=h0, y=y, r=r, h=J.norm(r_norm, r, p["r_weight"], p.get("r_bias"), EPS), idx=idx, Z=Z)
    if dr is None:
        return out
    st = np.stack((*J.stats(y_norm, y, EPS), *J.stats(r_norm, r, EPS)), 1)
    g = J.backward(y, r, st, p, dr, dh, y_norm, r_norm, 0.5, keep)
    layer = O.moe_backward(h0, inp["W_r"], W, idx, wt, g["dy"])
    m, s = J.stats("rms", x, EPS)
    first = J.backward(None, x, np.stack((m, s, m, s), 1), {"r_weight": p["in_weight"]}, g["dx"], layer["dX"],
                       "none", "rms")
    out.update(g=g, layer=layer, dx=first["dx"], in_weight=first["r_weight"])
    return out


def gap(Z, k):
    """Smallest distance of a token's k-th logit to the next."""
    top = np.sort(Z, 1)[:, ::-1]
    return (top[:, k - 1] - top[:, k]).min() if Z.shape[1] > k else np.inf


@pytest.mark.parametrize("stream,y_norm,r_norm,drop", [("bf16", "rms", "rms", 0.0), ("f32", "none", "layer", 0.1),
                                                       ("f32", "layer", "rms", 0.25)])
@pytest.mark.parametrize("T", [7, 300])
def test_training_block(T, stream, y_norm, r_norm, drop):
    say(f"[gpu] block T={T} {stream} {y_norm} {r_norm} {drop}")
    w, inp, p, block = make(T, stream, y_norm, r_norm, drop, True)
    rng = np.random.default_rng(9)
    dr, dh = (to_bf16(rng.standard_normal((T, w.d), dtype=np.float32)) for _ in range(2))
    block.dr.copy_(torch.from_numpy(dr))
    block.dh.copy_(torch.from_numpy(dh))
    block.forward()
    block.backward()
    torch.cuda.synchronize()
    ref = reference(w, inp, p, block, y_norm, r_norm, drop, dr.astype(np.float64), dh.astype(np.float64))
    L = block.layer
    for name, got, want in (("h0", L.X, ref["h0"]), ("y", L.Y, ref["y"]), ("r", block.r, ref["r"]),
                            ("h", block.h, ref["h"]), ("dy", L.dY, ref["g"]["dy"]), ("dx", block.dx, ref["dx"]),
                            ("dW_gate", L.dW_gate, ref["layer"]["dW_gate"]),
                            ("dW_r", L.dW_r, ref["layer"]["dW_r"]),
                            ("in_weight", block.first_grads["r_weight"], ref["in_weight"])):
        assert_close(name, f64(got), want)
    for name, t in block.grads.items():
        assert_close(name, f64(t), ref["g"][name])


def test_training_block_captured_and_replayed():
    """A graph of a whole step, replayed with the offset moved on: every replay is the eager step."""
    T = 200
    blocks = [make(T, "f32", "rms", "rms", 0.2, True)[3] for _ in range(2)]
    rng = np.random.default_rng(9)
    for name in ("dr", "dh"):
        v = torch.from_numpy(rng.standard_normal((T, 512), dtype=np.float32))
        for b in blocks:
            getattr(b, name).copy_(v)
    a, b = blocks
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.forward()
        a.backward()
    seen = []
    for step in range(3):
        for q in blocks:
            q.rng[1] = step
        graph.replay()
        b.forward()
        b.backward()
        torch.cuda.synchronize()
        for name in ("r", "h", "dx"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (step, name)
        for name in a.grads:
            assert torch.equal(a.grads[name], b.grads[name]), (step, name)
        assert torch.equal(a.layer.dW_down, b.layer.dW_down)
        seen.append(a.r.clone())
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


@pytest.mark.parametrize("T", [1, 5, 16])
def test_decoding_block(T):
    """Up to 16 tokens: norm, the layer in two launches, join; two blocks one after the other."""
    routing = B.routing("sigmoid", scale=1.5)
    w, inp, p, block = make(T, "bf16", "rms", "rms", 0.0, False, E=16, k=4, routing=routing)
    assert block.few
    block.forward()
    torch.cuda.synchronize()
    plain = DeviceLayer(w, {**inp, "X": to_np(block.layer.X)}, routing=routing, with_backward=False)
    plain.step()
    torch.cuda.synchronize()
    if gap(to_np(plain.logits), w.k) > 1e-4:
        assert torch.equal(plain.topk_idx, block.layer.topk_idx)
        # there H and each expert's output are rounded to bf16 too
        assert_close("y", f64(block.layer.Y), f64(plain.Y), REL_TOL)
    want = J.join_r(f64(block.x), f64(block.layer.Y), {n: p.get(n) for n in J.PARAMS}, "rms", EPS, 0.5)
    assert_close("r", f64(block.r), want)
    first_r = block.r.clone()
    block.x.copy_(block.r)
    block.forward()
    torch.cuda.synchronize()
    h0 = J.norm("rms", f64(first_r), p["in_weight"], None, EPS)
    assert_close("h0 of the second block", f64(block.layer.X), h0)
    assert torch.isfinite(block.h).all()


def test_few_of_a_layer_and_its_refusal():
    w = Workload("few", T=6, d=256, E=8, k=2, f=256)
    L = DeviceLayer(w, make_inputs(w, 3), few=True)
    L.step()
    torch.cuda.synchronize()
    Y, idx = L.Y.clone(), L.topk_idx.clone()
    L.step_few()
    torch.cuda.synchronize()
    assert torch.equal(idx, L.topk_idx)
    assert_close("Y", f64(L.Y), f64(Y))
    with pytest.raises(ValueError):
        DeviceLayer(w.scaled(T=17), make_inputs(w.scaled(T=17), 3), few=True)
