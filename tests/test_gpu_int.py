"""The experts in 8-bit integers on the GPU against the oracle, element by
element: codes exactly, outputs within the codes that the 32-bit evaluation of
the activation can move across a tie and the roundings to bf16."""
import numpy as np
import pytest
import torch

from oracle import int_oracle as I
from paper_2609_36070_amd import binding as B
from paper_2609_36070_amd.layer import DeviceLayer
from paper_2609_36070_amd.workloads import Workload, make_inputs, to_bf16
from tests import dispatch, score_int_rules as R
from tests.parity import say, to_np

pytestmark = pytest.mark.gpu
EXTRA_CODES = 0.0     # codes that a different rounding of H could move beyond the oracle's own count


def oracle_weights(w, inp):
    q = {n: [I.quantize_weights(m) for m in inp[k]] for n, k in (("g", "W_gate"), ("u", "W_up"), ("d", "W_down"))}
    if w.f_s:
        q.update(gs=I.quantize_weights(inp["Wg_s"]), us=I.quantize_weights(inp["Wu_s"]),
                 ds=I.quantize_weights(inp["Wd_s"]))
    return q


def check_weights(L, q, w):
    """Every code and scale, bit for bit."""
    for i, n in enumerate("gud"):
        assert np.array_equal(to_np(L.int_bufs[i]), np.stack([c for c, _ in q[n]])), n
        assert np.array_equal(to_np(L.int_bufs[3 + i]), np.stack([s for _, s in q[n]]), equal_nan=True), n
        if w.f_s:
            assert np.array_equal(to_np(L.int_bufs[6 + i]), q[n + "s"][0]), n
            assert np.array_equal(to_np(L.int_bufs[9 + i]), q[n + "s"][1], equal_nan=True), n


def parity(w, seed=0, inp=None, codes=True):
    say(f"[gpu] {w.name} T={w.T} d={w.d} E={w.E} k={w.k} f={w.f} f_s={w.f_s}")
    inp = make_inputs(w, seed) if inp is None else inp
    L = DeviceLayer(w, inp, int8=True)
    L.step_int()
    torch.cuda.synchronize()
    q = oracle_weights(w, inp)
    if codes:
        check_weights(L, q, w)
    Y, tol = I.moe_forward_int(inp["X"], q, to_np(L.topk_idx), to_np(L.topk_w), extra=EXTRA_CODES)
    err = np.abs(to_np(L.Y) - Y)
    say(f"  |err| {err.max():.3e} of {np.abs(Y).max():.3e}, worst share of the bound {(err / tol).max():.3f}")
    assert (err <= tol).all()
    # the bound is no blank cheque: on average the error is far below it
    assert np.sqrt((err ** 2).mean()) <= 8e-3 * np.sqrt((Y ** 2).mean()) + 1e-30
    return L, inp


SHAPES = [
    Workload("one token", T=1, d=256, E=8, k=2, f=256),
    Workload("one token, one expert", T=1, d=512, E=1, k=1, f=256),
    Workload("one token, shared", T=1, d=1024, E=16, k=4, f=512, f_s=256),
    Workload("few tokens", T=7, d=768, E=9, k=3, f=512),
    Workload("16 tokens", T=16, d=2048, E=12, k=4, f=768),
    Workload("17 tokens", T=17, d=2048, E=12, k=4, f=768),
    Workload("61 dense", T=61, d=1280, E=4, k=4, f=512, f_s=512),
    Workload("64 on one", T=64, d=256, E=2, k=1, f=256, bias_std=3.0),
    Workload("65", T=65, d=512, E=8, k=8, f=256),
    Workload("128 experts", T=100, d=512, E=128, k=8, f=256, bias_std=0.5),
    Workload("300, skewed", T=300, d=256, E=8, k=2, f=512, bias_std=2.0),
    Workload("ragged", T=777, d=512, E=16, k=4, f=768, f_s=1024),
    Workload("wide", T=40, d=256, E=4, k=2, f=2304),
    Workload("long rows", T=33, d=8448, E=2, k=2, f=256),
    Workload("k 16 of 200", T=520, d=256, E=200, k=16, f=256),
    Workload("whole tiles", T=1024, d=256, E=4, k=1, f=256),
]


@pytest.mark.parametrize("w", SHAPES, ids=lambda w: w.name)
def test_forward(w):
    parity(w, seed=2)


PATHS = [
    # (what the rules say, checked where a host compiler is there)
    (Workload("token, longest row", T=1, d=8192, E=4, k=2, f=256, f_s=256), dict(token=1)),
    (Workload("token, 17 routes", T=1, d=256, E=32, k=16, f=256, f_s=512), dict(token=1)),
    (Workload("token, f past the registers", T=1, d=256, E=3, k=2, f=2816, f_s=2304), dict(token=1)),
    (Workload("token, wide Y", T=1, d=4352, E=3, k=3, f=256), dict(token=1)),
    (Workload("one long token", T=1, d=8448, E=4, k=2, f=256, f_s=256), dict(token=0, tiles=1)),
    (Workload("one token, long f", T=1, d=256, E=16, k=16, f=3584), dict(token=0, tiles=1)),
    (Workload("dense, uneven waves", T=16, d=512, E=12, k=12, f=768, f_s=256), dict(up_dense=1, up_waves=5)),
    (Workload("dense, waves across experts", T=33, d=256, E=8, k=8, f=1280, f_s=256), dict(up_dense=1, up_waves=6)),
    (Workload("dense, two tiles of rows", T=100, d=256, E=4, k=4, f=512, f_s=256), dict(up_dense=0, tiles=4)),
    (Workload("dense, 192 rows", T=192, d=256, E=3, k=3, f=256), dict(up_dense=0, tiles=4)),
    (Workload("dense, tiles", T=193, d=256, E=3, k=3, f=256), dict(tiles=0)),
    (Workload("eight waves", T=60, d=256, E=12, k=4, f=512, f_s=256), dict(tiles=4, up_waves=8)),
    (Workload("four waves", T=60, d=256, E=64, k=8, f=1024), dict(tiles=4, up_waves=4)),
    (Workload("sixteen on one", T=16, d=256, E=8, k=1, f=256, bias_std=9.0), dict(tiles=1, up_waves=4)),
    (Workload("many up tiles", T=600, d=256, E=16, k=8, f=1280, bias_std=0.5), dict(tiles=0)),
    (Workload("many down tiles", T=600, d=2560, E=16, k=8, f=256, f_s=512), dict(tiles=0)),
    (Workload("shared and hot", T=1500, d=512, E=8, k=1, f=256, f_s=768, bias_std=2.0), dict(tiles=0)),
]


@pytest.mark.parametrize("w,path", PATHS, ids=lambda v: getattr(v, "name", ""))
def test_paths(w, path):
    """Shapes at the edges of every path, and several tiles per workgroup."""
    if dispatch.HAVE_CXX:
        assert {n: R.layer(n, w) for n in path} == path
    parity(w, seed=3, codes=False)


@pytest.mark.parametrize("T", [1, 9, 40, 700])
def test_an_expert_listed_twice(T):
    """A token may list an expert twice: it counts twice, each with its weight."""
    w = Workload("twice", T=T, d=256, E=6, k=3, f=256, f_s=256)
    inp = make_inputs(w, 14)
    L = DeviceLayer(w, inp, int8=True)
    L.route()
    L.topk_idx[0] = torch.tensor([4, 4, 1], dtype=torch.int32, device="cuda")
    L.topk_idx[T - 1] = torch.tensor([2, 2, 2], dtype=torch.int32, device="cuda")
    L.plan()
    L.forward_int()
    torch.cuda.synchronize()
    Y, tol = I.moe_forward_int(inp["X"], oracle_weights(w, inp), to_np(L.topk_idx), to_np(L.topk_w),
                               extra=EXTRA_CODES)
    assert (np.abs(to_np(L.Y) - Y) <= tol).all()


def test_one_workspace_under_two_graphs():
    """Two captured layers that share a workspace, replayed in turn on one
    stream, with eager work on the same workspace between."""
    w = Workload("shared ws", T=24, d=256, E=8, k=2, f=256, f_s=256)
    layers = [DeviceLayer(w, make_inputs(w, s), int8=True) for s in (1, 2)]
    layers[1].ws = layers[0].ws
    want, graphs = [], []
    for L in layers:
        L.step_int()
        torch.cuda.synchronize()
        want.append(L.Y.clone())
    for L in layers:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            L.step_int()
    for i in (0, 1, 0, 1, 1, 0):
        layers[i].Y.zero_()
        layers[1 - i].step_int()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(layers[i].Y, want[i]) and torch.equal(layers[1 - i].Y, want[1 - i])


@pytest.mark.parametrize("T", [1, 40, 500])
def test_stage_events(T):
    """Every stage's event is recorded, in order, and the results stay."""
    w = Workload("events", T=T, d=512, E=8, k=2, f=512, f_s=256)
    L = DeviceLayer(w, make_inputs(w, 2), int8=True)
    L.step_int()
    torch.cuda.synchronize()
    want = L.Y.clone()
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(7)]
    for e in ev:
        e.record()                          # creates the events
    stages = B.MoeStageEvents()
    for i, e in enumerate(ev):
        stages.ev[i] = e.cuda_event
    L.step_int(fwd_events=stages)
    torch.cuda.synchronize()
    assert all(a.elapsed_time(b) >= 0 for a, b in zip(ev, ev[1:])) and ev[0].elapsed_time(ev[6]) > 0
    assert torch.equal(L.Y, want)


def test_special_values():
    """Zero tokens, zero channels, channels and tokens of tiny and huge values,
    and values that tie between two codes."""
    w = Workload("special", T=50, d=256, E=4, k=2, f=256, f_s=256)
    inp = make_inputs(w, 5)
    inp["X"][3] = 0.0
    inp["X"][4] *= np.float32(2.0 ** -100)
    inp["X"][5, ::2] = 0.5 * np.sign(inp["X"][5, ::2])
    inp["X"][5, 7] = 1.0
    for n, ax in (("W_gate", 7), ("W_up", 9), ("W_down", 11), ("Wg_s", 13), ("Wu_s", 15), ("Wd_s", 17)):
        inp[n][..., ax] = 0.0
        inp[n][..., ax + 20] *= np.float32(2.0 ** -124)    # scales and quotients near the subnormals
        inp[n][..., ax + 40] *= np.float32(2.0 ** 20)
        inp[n] = to_bf16(inp[n])          # the oracle has the values that the device has
    parity(w, inp=inp)


def test_infinite_and_nan_values_stay_in_their_rows():
    """A token that holds an infinity or a NaN has an output of NaN; the others
    keep every bit.  A channel of W_down that holds one makes its column NaN."""
    for w in (Workload("nan, few", T=12, d=256, E=4, k=2, f=256),
              Workload("nan, many", T=600, d=256, E=4, k=2, f=256, f_s=256)):
        inp = make_inputs(w, 6)
        L, _ = parity(w, inp=inp)
        clean, logits = L.Y.clone(), L.logits.clone()
        L.X[2, 5], L.X[9, 0], L.X[10, 1] = float("inf"), float("nan"), float("-inf")
        L.forward_int()
        torch.cuda.synchronize()
        bad = torch.zeros(w.T, dtype=torch.bool, device=L.Y.device)
        bad[[2, 9, 10]] = True
        assert torch.isnan(L.Y[bad]).all() and torch.equal(L.Y[~bad], clean[~bad])
        assert torch.equal(logits, L.logits)
        L.X.copy_(torch.from_numpy(inp["X"]))
        L.W_down[1, 3, 20] = float("nan")
        L.quantize_int()
        L.forward_int()
        torch.cuda.synchronize()
        hit = (L.topk_idx == 1).any(1)
        assert torch.isnan(L.Y[hit, 20]).all()
        keep = torch.ones_like(L.Y, dtype=torch.bool)
        keep[hit, 20] = False
        assert torch.equal(L.Y[keep], clean[keep])


def test_experts_without_tokens_and_no_tokens():
    w = Workload("collapsed", T=90, d=256, E=16, k=2, f=256)
    inp = make_inputs(w, 8)
    inp["W_r"][:] = 0.0                    # every token takes experts 0 and 1
    L, _ = parity(w, inp=inp)
    assert to_np(L.counts)[2:].sum() == 0
    L = DeviceLayer(Workload("none", T=0, d=256, E=4, k=2, f=256, f_s=256),
                    make_inputs(Workload("none", T=0, d=256, E=4, k=2, f=256, f_s=256)), int8=True)
    L.step_int()
    torch.cuda.synchronize()


def test_unplaced_routes_are_left_out():
    """Ids outside [0, E) get no plan position; they contribute nothing."""
    for T in (9, 400):
        w = Workload("bad ids", T=T, d=256, E=8, k=2, f=256)
        inp = make_inputs(w, 4)
        L = DeviceLayer(w, inp, int8=True)
        L.route()
        L.topk_idx[3, 0], L.topk_idx[5, 1] = -1, 8
        L.plan()
        L.forward_int()
        torch.cuda.synchronize()
        idx, wt = to_np(L.topk_idx), to_np(L.topk_w)
        Y, tol = I.moe_forward_int(inp["X"], oracle_weights(w, inp), idx, wt, extra=EXTRA_CODES)
        assert (np.abs(to_np(L.Y) - Y) <= tol).all()


@pytest.mark.parametrize("T", [1, 40, 500])
def test_repeats_streams_and_graph(T):
    """Routing by scores, plan and int8 experts as a serving loop runs them:
    the same bits eagerly, on another stream and from a replayed graph."""
    w = Workload("served", T=T, d=512, E=16, k=4, f=512, f_s=256)
    inp = dict(make_inputs(w, 12), balance=np.zeros(16, np.float32))
    L = DeviceLayer(w, inp, int8=True, routing=B.routing("sigmoid", 4, 2, "pair", True, 2.5))
    L.step_int()
    torch.cuda.synchronize()
    want = L.Y.clone()
    side = torch.cuda.Stream()
    L.Y.zero_()
    torch.cuda.synchronize()
    L.step_int(side)
    torch.cuda.synchronize()
    assert torch.equal(L.Y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.step_int()
    for _ in range(3):
        L.Y.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(L.Y, want)


def test_two_layers_on_two_streams():
    w = Workload("pair", T=200, d=512, E=8, k=2, f=512)
    layers = [DeviceLayer(w, make_inputs(w, s), int8=True) for s in (1, 2)]
    for L in layers:
        L.step_int()
    torch.cuda.synchronize()
    want = [L.Y.clone() for L in layers]
    streams = [torch.cuda.Stream() for _ in layers]
    for L in layers:
        L.Y.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for L, s in zip(layers, streams):
            L.step_int(s)
    torch.cuda.synchronize()
    assert all(torch.equal(L.Y, y) for L, y in zip(layers, want))


def test_nothing_is_written_behind_the_output():
    w = Workload("guard", T=37, d=256, E=4, k=2, f=256)
    L = DeviceLayer(w, make_inputs(w, 1), int8=True)
    L.route()
    L.plan()
    out = torch.full((w.T + 2, w.d), 3.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((B.moe_int_workspace_bytes(L.shape) + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    B.moe_forward_int(L.shape, L.X, L.int_weights, L.topk_idx, L.topk_w, L.plan_bufs, out, ws,
                      ws_bytes=ws.numel() - 4096)
    torch.cuda.synchronize()
    assert (out[w.T:] == 3).all() and (ws[-4096:] == 0xAB).all()
