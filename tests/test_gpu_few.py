"""The whole layer for a few tokens on the GPU against the float64 oracles: the
selection is exact on the GPU's own logits, Y within the rounding of its steps.

Tolerance of Y.  A 32-bit sum over K takes K / 32 matrix products in four waves, 32
terms inside each, at most 32 slices and 10 roundings of other steps; a matrix
unit may cut off where a rounding goes to the nearest (a whole step): (K / 128 + 80)
steps of 2^-23 relative to the sum of the magnitudes.  H = silu(A) B moves with A
by at most 1.1 |B|, and is held to 2^-16 of itself (a low part of 8 bits under a
high one).  Y is rounded by half a step, 2^-8.
"""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from oracle import score_oracle as S
from paper_2609_36070_amd import binding as B
from paper_2609_36070_amd.workloads import to_bf16
from tests.parity import say, to_np

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAMES = ("W_gate", "W_up", "W_down", "Wg_s", "Wu_s", "Wd_s")


@dataclasses.dataclass(frozen=True)
class Case:
    T: int
    d: int
    E: int
    k: int
    f: int = 256
    fs: int = 0
    score: str = "softmax"
    groups: int = 1
    top_groups: int = 1
    group_score: str = "max"
    renormalise: bool = True
    scale: float = 1.0
    balance: float = 0.0
    bias: float = 0.0

    @property
    def sel(self):
        return dict(score=self.score, groups=self.groups, top_groups=self.top_groups,
                    group_score=self.group_score)

    @property
    def wts(self):
        return dict(score=self.score, renormalise=self.renormalise, scale=self.scale)

    def routing(self):
        return B.routing(renormalise=self.renormalise, scale=self.scale, **self.sel)

    def shape(self):
        return B.make_shape(self.T, self.d, self.E, self.k, self.f, self.fs)


CASES = [
    Case(1, 256, 1, 1), Case(1, 256, 1, 1, fs=256), Case(16, 256, 1, 1, 512), Case(2, 1024, 8, 1, 512, 0, "sigmoid", bias=0.5),
    Case(1, 2048, 128, 8, 768), Case(4, 7168, 256, 8, 256, 512, "sigmoid", 8, 4, "pair", scale=2.5, balance=0.1),
    Case(7, 1024, 8, 8, 512, 1024), Case(16, 512, 32, 8, 1536), Case(3, 512, 5, 2, 256, 256, renormalise=False),
    Case(16, 256, 256, 16, 256, 0, "sigmoid", 64, 4, "max", False, 1.0, 0.1), Case(15, 768, 255, 7, bias=0.5),
    Case(13, 512, 51, 16, 256, 768, "softmax", 3, 2, "pair", True, 0.5, 0.0), Case(5, 4096, 12, 4, 512, 0, "sigmoid"),
    Case(16, 1280, 20, 4, 1024, 512, "softmax", 4, 2, balance=0.1), Case(9, 256, 160, 6, 512, 256, "sigmoid", 8, 3, "pair"),
    Case(16, 256, 4, 4, 256, 256), Case(6, 2304, 60, 1, 768), Case(11, 1792, 96, 6, 256, 2048, "sigmoid", renormalise=False),
    Case(9, 2048, 16, 8, 1536),      # more weights than the caches hold
    Case(16, 1024, 2, 1, 2048, bias=1.0), Case(10, 512, 7, 7, 256, 0, "sigmoid", 7, 7, "pair"),
]
IDS = ["-".join(str(v) for v in dataclasses.astuple(c)) for c in CASES]


def inputs(c, seed=0):
    rng = np.random.default_rng(seed)
    n = lambda *s, std=1.0: to_bf16(rng.standard_normal(s, dtype=np.float32) * np.float32(std))   # noqa: E731
    inp = dict(X=n(c.T, c.d), W_r=n(c.d, c.E, std=c.d ** -0.5),
               W_gate=n(c.E, c.d, c.f, std=c.d ** -0.5), W_up=n(c.E, c.d, c.f, std=c.d ** -0.5),
               W_down=n(c.E, c.f, c.d, std=c.f ** -0.5))
    for name, s in (("Wg_s", (c.d, c.fs)), ("Wu_s", (c.d, c.fs)), ("Wd_s", (c.fs, c.d))):
        inp[name] = n(*s, std=s[0] ** -0.5) if c.fs else None
    inp["bias"] = rng.standard_normal(c.E, dtype=np.float32) * np.float32(c.bias) if c.bias else None
    inp["balance"] = rng.standard_normal(c.E, dtype=np.float32) * np.float32(c.balance) if c.balance else None
    return inp


class Run:
    """The call's buffers, outputs with untouched rows behind them, and a workspace of rubbish."""

    def __init__(self, c, inp):
        self.c, self.inp, self.sh, self.routing = c, inp, c.shape(), c.routing()
        up = lambda a, t: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(t).to(DEV)   # noqa: E731
        self.t = {n: up(inp[n], torch.bfloat16) for n in ("X", "W_r", *NAMES)}
        self.bias, self.balance = up(inp["bias"], torch.float32), up(inp["balance"], torch.float32)
        self.weights = B.weights_struct(*(self.t[n] for n in NAMES))
        self.logits = torch.full((c.T + 2, c.E), 777.0, device=DEV)
        self.idx = torch.full((c.T + 2, c.k), -7, dtype=torch.int32, device=DEV)
        self.w = torch.full((c.T + 2, c.k), 777.0, device=DEV)
        self.Y = torch.full((c.T + 2, c.d), 777.0, dtype=torch.bfloat16, device=DEV)
        self.nbytes = B.moe_few_workspace_bytes(self.sh)
        self.ws = torch.full((self.nbytes + 256,), 0xA5, dtype=torch.uint8, device=DEV)

    def call(self, stream=None):
        B.moe_forward_few(self.sh, self.routing, self.t["X"], self.t["W_r"], self.bias, self.balance, self.weights,
                          self.logits, self.idx, self.w, self.Y, self.ws, ws_bytes=self.nbytes, stream=stream)

    def outputs(self):
        return [t.clone() for t in (self.logits, self.idx, self.w, self.Y)]

    def check_guards(self):
        T = self.c.T
        assert (self.logits[T:] == 777).all() and (self.w[T:] == 777).all() and (self.idx[T:] == -7).all()
        assert (self.Y[T:] == 777).all() and (self.ws[self.nbytes:] == 0xA5).all()
        assert T == 0 or int(self.ws[:4].view(torch.int32).item()) == 0


def expert(x, Wg, Wu, Wd):
    """Output of an expert and the bound of its error (without Y's own rounding)."""
    x, Wg, Wu, Wd = (np.asarray(v, np.float64) for v in (x, Wg, Wu, Wd))
    d, f = Wg.shape
    ed, ef = ((n / 128 + 80) * 2.0 ** -23 for n in (d, f))
    a, b = x @ Wg, x @ Wu
    ma, mb = (ed * (np.abs(x) @ np.abs(w)) for w in (Wg, Wu))
    s = a / (1 + np.exp(-a))
    h = s * b
    eh = 1.1 * ma * (np.abs(b) + mb) + (np.abs(s) + 1.1 * ma) * mb + 2.0 ** -16 * np.abs(h)
    return h @ Wd, (eh + ef * np.abs(h)) @ np.abs(Wd)


def check(r, tokens=None):
    c, inp, T = r.c, r.inp, r.c.T
    Z, idx, w, Y = (to_np(t)[:T] for t in (r.logits, r.idx, r.w, r.Y))
    Zo = O.router_logits(inp["X"], inp["W_r"], inp["bias"])
    # fp32 sums over d, at most d / 8 + 60 roundings one after the other
    mag = np.abs(inp["X"]).astype(np.float64) @ np.abs(inp["W_r"]) + (0 if inp["bias"] is None else np.abs(inp["bias"]))
    assert (np.abs(Z - Zo) <= (c.d / 8 + 60) * 2.0 ** -24 * mag).all()
    assert np.array_equal(idx, S.select(Z, inp["balance"], c.k, **c.sel))
    ref = S.weights(Z, inp["balance"], idx, **c.wts)
    z = Z.astype(np.float64)
    # as the scored router's weights: differences of logits, exponentials, a sum and a quotient
    rel = (24 + 2 * np.minimum(z.max(1) - z.min(1), 100.0)[:, None]) * 2.0 ** -24
    assert (np.abs(w - ref) <= rel * np.abs(ref) + 1e-37).all()
    want, tol = np.zeros((T, c.d)), np.zeros((T, c.d))
    for e in np.unique(idx):
        t, slot = np.nonzero(idx == e)
        y, err = expert(inp["X"][t], *(inp[n][e] for n in NAMES[:3]))
        wt = w[t, slot].astype(np.float64)[:, None]
        want[t] += wt * y
        tol[t] += wt * err
    if c.fs:
        y, err = expert(inp["X"], *(inp[n] for n in NAMES[3:]))
        want, tol = want + y, tol + err
    err = np.abs(Y - want) / (2.0 ** -8 * (1 + 2.0 ** -8) * np.abs(want) + tol)
    say(f"  Y: {err.max():.3f} of the bound, {(np.abs(Y - want) / np.abs(want).max()).max():.2e} of the largest")
    assert err.max() <= 1.0
    r.check_guards()


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_against_the_definition(c):
    say(f"[gpu] few {dataclasses.astuple(c)}")
    r = Run(c, inputs(c))
    r.call()
    torch.cuda.synchronize()
    check(r)


def test_every_number_of_tokens():
    for T in range(1, 17):
        c = Case(T, 256, 24, 3, 256, 256, balance=0.1)
        say(f"[gpu] few {T} tokens")
        r = Run(c, inputs(c, T))
        r.call()
        torch.cuda.synchronize()
        check(r)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("groups", [1, 4])
def test_masks_infinities_and_ties(score, renormalise, groups):
    """Logits of exact ties, +-inf, the lowest finite values, NaN, and nothing in play: the
    scored router's rows, chosen as its oracle does."""
    E, d, k = 32, 256, 5
    c = Case(16, d, E, k, 256, 0, score, groups, min(groups, 2), "pair", renormalise, 1.5)
    inp = inputs(c, 9)
    rng = np.random.default_rng(9)
    W_r = np.zeros((d, E), np.float32)
    W_r[:8] = to_bf16(rng.standard_normal((8, E), dtype=np.float32))
    W_r[1] = 1.0
    W_r[2] = np.where(np.arange(E) % 3 == 0, 2.0, -2.0)
    X = np.zeros((c.T, d), np.float32)
    for t in range(c.T):
        X[t, t % 8] = 30.0 if t >= 8 else 1.0
    X[5] = 0.0
    bias = np.zeros(E, np.float32)
    bias[[3, 9]] = -np.inf, np.finfo(np.float32).min
    bias[4] = np.inf
    balance = (rng.standard_normal(E) * 0.05).astype(np.float32)
    balance[[1, 12, 30]] = -np.inf, np.inf, np.nan
    inp.update(X=X, W_r=W_r)
    for bal, bi in ((balance, bias), (None, bias), (None, None), (np.zeros(E, np.float32), None),
                    (np.zeros(E, np.float32), np.full(E, -np.inf, np.float32))):
        inp.update(bias=bi, balance=bal)
        r = Run(c, inp)
        r.call()
        torch.cuda.synchronize()
        Z, idx, w = (to_np(t)[:c.T] for t in (r.logits, r.idx, r.w))
        assert np.array_equal(idx, S.select(Z, bal, k, **c.sel))
        ref = S.weights(Z, bal, idx, **c.wts)
        live = S.in_play(Z, bal)
        z = np.clip(np.where(live, Z, 0), -1e4, 1e4).astype(np.float64)
        rel = (24 + 2 * np.minimum(z.max(1) - z.min(1), 100.0)[:, None]) * 2.0 ** -24
        assert np.isfinite(w).all() and (np.abs(w - ref) <= rel * np.abs(ref) + 1e-37).all()
        assert torch.isfinite(r.Y[:c.T]).all()
        if bi is not None and np.isneginf(bi).all():
            assert (w == 0).all() and (r.Y[:c.T] == 0).all()
        r.check_guards()


def test_close_scores_are_ranked_in_64_bits():
    """Saturated sigmoids plus a balance differ by less than 2^-24; equal ones go by id."""
    c = Case(8, 256, 128, 6, score="sigmoid", balance=1.0)
    inp = inputs(c)
    inp["W_r"] = np.zeros((c.d, c.E), np.float32)
    inp["W_r"][0, 100:] = to_bf16(17.0 + 0.125 * np.arange(28, dtype=np.float32))
    inp["X"] = np.zeros((c.T, c.d), np.float32)
    inp["X"][:4, 0] = 1.0
    inp["balance"] = np.full(c.E, 0.25, np.float32)
    r = Run(c, inp)
    r.call()
    torch.cuda.synchronize()
    idx = to_np(r.idx)
    assert (idx[:4] == np.arange(122, 128)).all() and (idx[4:8] == np.arange(6)).all()


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_an_expert_reaches_its_tokens_alone(value):
    """Infinite or NaN weights of an expert, and values of a token, stay where they belong."""
    c = Case(6, 256, 8, 2, 512, 256)
    inp = inputs(c)
    good = Run(c, inp)
    good.call()
    torch.cuda.synchronize()
    idx = to_np(good.idx)[:c.T]
    e = int(idx[0, 0])
    hit = (idx == e).any(1)
    assert hit.any() and not hit.all()
    for name in NAMES[:3]:
        bad = Run(c, inp)
        bad.t[name][e] = value
        bad.call()
        torch.cuda.synchronize()
        miss = torch.from_numpy(~hit).to(DEV)
        assert torch.equal(bad.Y[:c.T][miss], good.Y[:c.T][miss]), name
        assert not torch.isfinite(bad.Y[:c.T][~miss]).any(), name
    bad = Run(c, inp)
    bad.t["X"][3, 7] = value
    bad.call()
    torch.cuda.synchronize()
    keep = [0, 1, 2, 4, 5]
    assert torch.equal(bad.Y[keep], good.Y[keep]) and torch.equal(bad.idx[keep], good.idx[keep])
    assert not torch.isfinite(bad.Y[3]).any()
    bad.check_guards()


def test_repeats_streams_and_several_at_once():
    """The same bits again, on other streams, with three other calls running beside (more workgroups
    than the GPU holds at once)."""
    cases = (Case(16, 2048, 64, 4, 768, 512, balance=0.1), Case(3, 4096, 16, 4, 1024), Case(16, 1024, 32, 8, 1536),
             Case(9, 512, 128, 8, 512, 256, "sigmoid"))
    runs = [(Run(c, inputs(c, 3)), Run(c, inputs(c, 3))) for c in cases]
    for r, _ in runs:
        r.call()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for (_, r), s in zip(runs, streams):
            r.call(s)
    torch.cuda.synchronize()
    for r, other in runs:
        for x, y in zip(r.outputs(), other.outputs()):
            assert torch.equal(x, y)
        other.check_guards()


@pytest.mark.parametrize("offset", [16, 64, 112, 240])
def test_workspaces_of_any_alignment(offset):
    """A workspace from any multiple of 16 bytes: the same bits, and nothing past its end."""
    for c in (Case(7, 1024, 32, 4, 512, 256), Case(3, 2048, 16, 4, 768)):
        inp = inputs(c, 6)
        r, other = Run(c, inp), Run(c, inp)
        other.ws = torch.full((other.nbytes + 512,), 0xA5, dtype=torch.uint8, device=DEV)[offset:]
        assert other.ws.data_ptr() % 256 == offset
        r.call()
        for _ in range(3):
            other.call()
            torch.cuda.synchronize()
            for a, b in zip(r.outputs(), other.outputs()):
                assert torch.equal(a, b)
            other.check_guards()


def test_captured_and_replayed():
    c = Case(5, 1024, 40, 5, 512, 256, "sigmoid", 4, 2, "pair", True, 2.0, 0.1)
    r, ref = Run(c, inputs(c)), Run(c, inputs(c))
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        r.call()
    for step in range(3):
        x = inputs(c, 10 + step)["X"]
        for q in (r, ref):
            q.t["X"].copy_(torch.from_numpy(x))
        graph.replay()
        ref.call()
        torch.cuda.synchronize()
        for x, y in zip(r.outputs(), ref.outputs()):
            assert torch.equal(x, y), step


def test_no_tokens():
    c = Case(0, 256, 16, 2)
    r = Run(c, inputs(c))
    r.t["X"] = torch.empty(8, 256, dtype=torch.bfloat16, device=DEV)
    r.call()
    torch.cuda.synchronize()
    r.check_guards()


def test_agrees_with_the_separate_calls():
    """Route, plan and forward of the same layer: one bf16 step of their roundings of H apart."""
    c = Case(16, 1024, 32, 4, 512, 512, "sigmoid", scale=1.5)
    inp = inputs(c, 4)
    r = Run(c, inp)
    r.call()
    sh, T, R = c.shape(), c.T, c.T * c.k
    ws = torch.empty(B.moe_workspace_bytes(sh, False), dtype=torch.uint8, device=DEV)
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)   # noqa: E731
    logits, idx, w = torch.empty(T, c.E, device=DEV), i32((T, c.k)), torch.empty(T, c.k, device=DEV)
    plan = B.plan_bufs(*(bufs := (i32(c.E), i32(c.E + 1), i32(R), i32(R))))
    Y = torch.empty(T, c.d, dtype=torch.bfloat16, device=DEV)
    B.moe_route_scored(sh, c.routing(), r.t["X"], r.t["W_r"], None, None, logits, idx, w, ws)
    B.moe_plan(sh, idx, plan, ws)
    B.moe_forward(sh, r.t["X"], r.weights, idx, w, plan, Y, False, ws)
    torch.cuda.synchronize()
    assert bufs[1][c.E] == R and torch.equal(idx, r.idx[:T])
    assert (w - r.w[:T]).abs().max() < 1e-5
    # H, each expert's output and Y rounded to bf16 there, Y alone here
    assert (Y.float() - r.Y[:T].float()).abs().max() <= 4 * 2.0 ** -8 * Y.float().abs().max()


def test_workgroups_that_start_late():
    """Beside joins whose workgroups leave no room on a CU (143 KB of its LDS): workgroups of a call start in
    dribs, after others have done the items that they would have begun with; none is done twice or left."""
    T, d = 6144, 7168
    j = B.join(T, d, y_norm="layer", r_norm="layer")
    x, y, out, h = (torch.zeros(T, d, dtype=torch.bfloat16, device=DEV) for _ in range(4))
    weights = {n: torch.ones(d, device=DEV) for n in B.JOIN_PARAMS if n != "token_gate"}
    params = B.join_params(**weights)
    # items of the up product fewer than the workgroups, about as many, and more
    cases = (Case(2, 512, 16, 2, 512), Case(16, 1024, 32, 4, 768, 256), Case(16, 2048, 64, 4, 1536))
    runs = [(Run(c, inputs(c, 5)), Run(c, inputs(c, 5))) for c in cases]
    for r, _ in runs:
        r.call()
    torch.cuda.synchronize()
    joins, few = torch.cuda.Stream(), torch.cuda.Stream()
    for turn in range(10):
        for r, other in runs:
            other.Y[:other.c.T].fill_(777.0)
            for s in (joins, few):
                s.wait_stream(torch.cuda.current_stream())
            for _ in range(3):
                B.moe_join_forward(j, x, y, params, None, out, h, None, stream=joins)
                other.call(few)
            for s in (joins, few):
                torch.cuda.current_stream().wait_stream(s)
            torch.cuda.synchronize()
            for a, b in zip(r.outputs(), other.outputs()):
                assert torch.equal(a, b), (turn, r.c)
            other.check_guards()
