"""Joining a block to the residual stream on the GPU against the float64 oracle.

Tolerances.  A rounding to a type is off by half a step, eps / 2 of the value.  A
32-bit sum over a row adds at most 32 values in a thread, 6 exchanges in a wave and
16 waves, and a term has at most 10 roundings of its own: 64 half steps of 2^-24,
relative to the sum of the magnitudes.  Sums over T rows add T / 256 (+ 1) of them in
a thread, 3 exchanges in a wave, at most 8 of a workgroup's rows, the at most 768
workgroups in 32 lists of 24, and the lists: T / 256 + 68 more.
"""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import join_oracle as J
from paper_2609_36070_amd import binding as B
from tests.parity import say, to_np

pytestmark = pytest.mark.gpu
DEV = "cuda"
U32, U16 = 2.0 ** -24, 2.0 ** -8
EPS = 1e-5


@dataclasses.dataclass(frozen=True)
class Case:
    T: int
    d: int
    stream: str = "bf16"
    y_norm: str = "rms"
    r_norm: str = "rms"
    gate: bool = False
    token_gate: bool = False
    scale: float = 1.0
    drop: float = 0.0
    block: bool = True
    weights: bool = True
    seed: int = 0

    def join(self):
        return B.join(self.T, self.d, self.stream, self.y_norm, self.r_norm, EPS, EPS, self.scale, self.drop)


CASES = [
    # every instance of the kernels, few rows and many; rows that no thread count divides
    Case(1, 8), Case(1, 7168, y_norm="layer", gate=True), Case(3, 1000, "f32", "layer", "layer", True, True, 0.5, 0.1),
    Case(257, 8, "f32", "none", "layer", drop=0.5), Case(300, 504, gate=True, token_gate=True),
    Case(700, 1024, "f32", "rms", "layer", drop=0.1), Case(258, 1032, y_norm="layer", r_norm="layer", gate=True),
    Case(1001, 2048, "f32", "none", "rms", True, False, -2.0, 0.25), Case(513, 2056, token_gate=True, drop=0.9),
    Case(600, 4096, y_norm="layer", r_norm="none"), Case(259, 4104, "f32", "rms", "rms", True, True, 0.3, 0.01),
    Case(520, 7168, gate=True, drop=0.1), Case(261, 8192, "f32", "layer", "layer"), Case(16, 8200, y_norm="none"),
    Case(301, 16384, "f32", "layer", "layer", True, True, 0.7, 0.1), Case(300, 12296, gate=True, drop=0.5),
    # workgroups that take many rows of the forward, a ragged number of them
    Case(24577, 520, y_norm="none", drop=0.1), Case(12289, 1032, "f32", "layer", "layer", True), Case(6145, 2056, gate=True),
    Case(6150, 4104, "f32", "none", "rms", token_gate=True, drop=0.1),
    Case(1025, 9224, "f32", "none", "layer", True, False, 0.5), Case(2, 16384, y_norm="layer", r_norm="none", drop=0.2),
    Case(300, 8200, block=False, y_norm="none"), Case(70, 12288, "f32", "rms", "rms", weights=False),
    Case(256, 2048, r_norm="none", y_norm="none", drop=0.1), Case(5, 24, "f32", "rms", "none", weights=False),
    # the norm before the first block; norms without weights
    Case(1, 2048, block=False, y_norm="none"), Case(400, 4096, "f32", "none", "layer", block=False),
    Case(77, 128, weights=False, y_norm="layer", r_norm="layer", token_gate=True),
    Case(64, 256, block=False, y_norm="none", weights=False),
]
IDS = ["-".join(str(v) for v in dataclasses.astuple(c)) for c in CASES]


def dev(a, t=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(t).to(DEV)


def f64(t):
    return None if t is None else to_np(t).astype(np.float64)


class Run:
    """The buffers of a case, outputs with untouched rows behind them."""

    def __init__(self, c):
        self.c, rng = c, np.random.default_rng(c.seed)
        T, d = c.T, c.d
        self.type = torch.float32 if c.stream == "f32" else torch.bfloat16
        make = lambda t, shift=0.0: dev(rng.standard_normal((T, d)) + shift, t)   # noqa: E731
        self.x, self.dr = make(self.type), make(self.type)
        self.y = make(torch.bfloat16, 0.25) if c.block else None
        self.dh = make(torch.bfloat16)
        has = dict(y_weight=c.weights and c.y_norm != "none", y_bias=c.weights and c.y_norm == "layer",
                   r_weight=c.weights and c.r_norm != "none", r_bias=c.weights and c.r_norm == "layer",
                   gate=c.gate, token_gate=c.token_gate)
        self.p = {n: dev(1 + 0.3 * rng.standard_normal(T if n == "token_gate" else d)) if has[n] else None
                  for n in J.PARAMS}
        self.key = [int(v) for v in rng.integers(0, 2 ** 62, 2)]
        self.rng = torch.tensor(self.key, dtype=torch.int64, device=DEV) if c.drop else None
        like = lambda t, rows, cols: torch.full((rows + 2, cols), 77.0, dtype=t, device=DEV)   # noqa: E731
        self.r = like(self.type, T, d) if c.block else None
        self.h, self.stats = like(torch.bfloat16, T, d), like(torch.float32, T, 4)
        self.dx, self.dy = like(self.type, T, d), like(torch.bfloat16, T, d) if c.block else None
        self.g = {n: torch.full((len(v) + 8,), 77.0, device=DEV) for n, v in self.p.items() if v is not None}
        self.join, self.params, self.grads = c.join(), B.join_params(**self.p), B.join_grads(**self.g)
        self.ws = torch.empty(B.moe_join_workspace_bytes(self.join), dtype=torch.uint8, device=DEV)

    def forward(self, stream=None):
        B.moe_join_forward(self.join, self.x, self.y, self.params, self.rng, self.r, self.h, self.stats,
                           stream=stream)

    def backward(self, stream=None):
        B.moe_join_backward(self.join, self.y, self.x if self.r is None else self.r, self.stats, self.params,
                            self.rng, self.dr, self.dh, self.dx, self.dy, self.grads, self.ws, stream=stream)

    def outputs(self):
        out = dict(r=self.r, h=self.h, stats=self.stats, dx=self.dx, dy=self.dy, **self.g)
        return {n: t for n, t in out.items() if t is not None}

    def check_guards(self):
        for n, t in self.outputs().items():
            m = len(self.p[n]) if n in J.PARAMS else self.c.T
            assert (t[m:] == 77).all(), n


def within(name, got, want, tol):
    err = np.abs(got - want)
    worst = float((err / np.maximum(tol, 1e-300)).max()) if err.size else 0.0
    say(f"  {name}: {worst:.3f} of the bound")
    assert np.isfinite(got).all() and worst <= 1.0, name


def check(run):
    c, T = run.c, run.c.T
    half = U16 if c.stream == "bf16" else U32
    keep = J.keep_mask(T, c.d, c.drop, *run.key)
    p = {n: f64(v) for n, v in run.p.items()}
    x, y = f64(run.x), f64(run.y)
    st = f64(run.stats[:T])
    if c.block:
        r = f64(run.r[:T])
        m, s = J.stats(c.y_norm, y, EPS)
        within("y's mean", st[:, 0], m, 64 * U32 * np.abs(y).mean(1))
        within("y's 1/deviation", st[:, 1], s, 2 * 64 * U32 * s)
        want = J.join_r(x, y, p, c.y_norm, EPS, c.scale, keep)
        # magnitudes: the mean is an addend of its own
        u = y if c.y_norm == "none" else (np.abs(y) + np.abs(y).mean(1, keepdims=True)) * s[:, None]
        mag = J.join_r(np.abs(x), np.abs(u), {n: None if v is None else np.abs(v) for n, v in p.items()},
                       "none", EPS, abs(c.scale), keep)
        if p["y_weight"] is not None:
            u = np.abs(u * p["y_weight"]) + (0 if p["y_bias"] is None else np.abs(p["y_bias"]))
            q = {n: np.abs(p[n]) for n in ("gate", "token_gate") if p[n] is not None}
            mag = J.join_r(np.abs(x), u, q, "none", EPS, abs(c.scale), keep)
        within("r", r, want, half * np.abs(want) * (1 + 2.0 ** -8) + 3 * 64 * U32 * mag)
    else:
        r = x
    m, s = J.stats(c.r_norm, r, EPS)
    within("r's mean", st[:, 2], m, 64 * U32 * np.abs(r).mean(1))
    within("r's 1/deviation", st[:, 3], s, 2 * 64 * U32 * s)
    want = J.norm(c.r_norm, r, p["r_weight"], p["r_bias"], EPS)
    u = np.abs(r) if c.r_norm == "none" else (np.abs(r) + np.abs(r).mean(1, keepdims=True)) * s[:, None]
    mag = np.abs(u * (1 if p["r_weight"] is None else p["r_weight"])) + (0 if p["r_bias"] is None else np.abs(p["r_bias"]))
    within("h", f64(run.h[:T]), want, U16 * np.abs(want) * (1 + 2.0 ** -8) + 3 * 64 * U32 * mag)

    args = (y, r, st, p, f64(run.dr), f64(run.dh), c.y_norm, c.r_norm)
    g, mag = (J.backward(*args, abs(c.scale) if q else c.scale, keep, mag=q) for q in (False, True))
    within("dx", f64(run.dx[:T]), g["dx"], half * np.abs(g["dx"]) * (1 + 2.0 ** -8) + 2 * 64 * U32 * mag["dx"])
    if c.block:
        within("dy", f64(run.dy[:T]), g["dy"],
               U16 * np.abs(g["dy"]) * (1 + 2.0 ** -8) + 4 * 64 * U32 * mag["dy"])
    for n, t in run.g.items():
        got = f64(t)[:len(run.p[n])]
        terms = 3 * 64 + (T / 256 + 68 if n != "token_gate" else 0)
        within("d" + n, got, g[n], terms * U32 * mag[n])
    run.check_guards()


@pytest.mark.parametrize("c", CASES, ids=IDS)
def test_against_the_definition(c):
    say(f"[gpu] join {dataclasses.astuple(c)}")
    run = Run(c)
    run.forward()
    run.backward()
    torch.cuda.synchronize()
    check(run)


@pytest.mark.parametrize("T, d", [(32, 64), (33, 64), (64, 64), (65, 64), (16, 256), (17, 256), (2, 2048), (3, 2048),
                                  (2, 4096), (3, 4096), (1, 7168), (2, 7168), (1023, 1000), (1027, 1000), (512, 2048),
                                  (513, 2048), (384, 4096), (385, 4096), (384, 7168), (385, 7168), (300, 8200)])
def test_a_workgroup_a_round_or_more(T, d):
    """Rows that one workgroup takes, which leaves the sums itself, those for which there is one round, and
    those past them; nothing is written past the workspace."""
    run = Run(Case(T, d, "bf16", "layer", "layer", True, True, 0.5, 0.1))
    n = B.moe_join_workspace_bytes(run.join)
    run.ws = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    run.forward()
    run.backward()
    torch.cuda.synchronize()
    assert (run.ws[n:] == 0xA5).all()
    check(run)


def test_repeats_bit_for_bit_and_on_another_stream():
    for c in (Case(1111, 2048, "f32", "layer", "rms", True, True, 0.5, 0.1), Case(600, 8400, token_gate=True, drop=0.1)):
        repeat(c)


def repeat(c):
    first = Run(c)
    first.forward()
    first.backward()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    again = Run(c)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again.forward()
        again.backward()
    side.synchronize()
    for n, t in first.outputs().items():
        assert torch.equal(t, again.outputs()[n]), n


@pytest.mark.parametrize("c", [Case(300, 1000, "bf16", "rms", "layer", True, False, 1.0, 0.2),
                               Case(270, 9000, "bf16", "rms", "layer", True, True, 1.0, 0.2)], ids=("1000", "9000"))
def test_in_place_gives_the_same(c):
    a, b = Run(c), Run(c)
    a.forward()
    a.backward()
    b.r = b.x
    b.forward()
    b.dx = b.dr
    b.backward()
    torch.cuda.synchronize()
    assert torch.equal(a.r[:c.T], b.x) and torch.equal(a.dx[:c.T], b.dr)
    for n in ("h", "stats", "dy"):
        assert torch.equal(getattr(a, n), getattr(b, n)), n
    for n in a.g:
        assert torch.equal(a.g[n], b.g[n]), n


@pytest.mark.parametrize("which", ("dr", "dh"))
def test_one_gradient_only(which):
    """The last block has no further stream, a join without h no norm: zeros give the same."""
    c = Case(65, 520, "f32", "layer", "rms", True, True, 0.5, 0.3)
    a, b = Run(c), Run(c)
    a.forward()
    b.forward()
    getattr(a, which).zero_()
    a.backward()
    setattr(b, which, None)
    b.backward()
    torch.cuda.synchronize()
    for n, t in a.outputs().items():
        assert torch.equal(t, b.outputs()[n]), n


def test_frozen_parameters_and_sum_only():
    c = Case(129, 256, "f32", "rms", "none", True, False, 0.5)
    a = Run(c)
    a.forward()
    a.backward()
    b = Run(c)
    B.moe_join_forward(b.join, b.x, b.y, b.params, None, b.r, None, b.stats)
    grads = B.join_grads(gate=b.g["gate"])
    b.dh = None
    B.moe_join_backward(b.join, b.y, b.r, b.stats, b.params, None, b.dr, None, b.dx, b.dy, grads, b.ws)
    torch.cuda.synchronize()
    assert torch.equal(a.r, b.r) and (b.h == 77).all() and (b.g["y_weight"] == 77).all()
    want = J.backward(f64(b.y), f64(b.r)[:c.T], f64(b.stats)[:c.T], {n: f64(v) for n, v in b.p.items()},
                      f64(b.dr), None, c.y_norm, "none", c.scale)
    within("gate", f64(b.g["gate"])[:c.d], want["gate"], 300 * U32 * np.abs(
        J.backward(f64(b.y), f64(b.r)[:c.T], f64(b.stats)[:c.T], {n: f64(v) for n, v in b.p.items()},
                   f64(b.dr), None, c.y_norm, "none", c.scale, mag=True)["gate"]))


def test_mask_of_a_large_offset_and_seed():
    """64-bit seeds and offsets, as the generator's counter has them, negative ones too."""
    c = Case(9, 64, "f32", "none", "none", drop=0.5)
    run = Run(c)
    for key in ((-1, -(1 << 63)), ((1 << 62) + 5, (1 << 33) + 1)):
        run.rng.copy_(torch.tensor(key, dtype=torch.int64))
        run.forward()
        torch.cuda.synchronize()
        gone = (run.r[:c.T] == run.x).cpu().numpy()
        assert np.array_equal(gone, J.keep_mask(c.T, c.d, 0.5, key[0] % 2 ** 64, key[1] % 2 ** 64) == 0)


def test_rows_that_are_zero_infinite_or_nan():
    """A row's values stay in its row; what dropout takes out is 0 whatever it was."""
    c = Case(300, 520, "f32", "rms", "rms", True, False, 1.0, 0.5)
    run = Run(c)
    run.y[0] = 0
    run.x[0] = 0
    run.y[1, 3] = float("inf")
    run.x[2, 5] = float("nan")
    run.forward()
    run.backward()
    torch.cuda.synchronize()
    assert (run.r[0] == 0).all() and (run.h[0] == 0).all() and abs(run.stats[0, 3].item() * EPS ** 0.5 - 1) < 1e-5
    assert run.r[2].isnan().sum() == 1 and run.h[2].isnan().all()
    assert run.r[3:c.T].isfinite().all() and run.h[3:c.T].isfinite().all() and run.dx[3:c.T].isfinite().all()
    d = Case(4, 64, "f32", "none", "none", drop=0.5)
    run = Run(d)
    run.y[:] = float("nan")
    run.forward()
    torch.cuda.synchronize()
    gone = torch.from_numpy(J.keep_mask(4, 64, 0.5, *run.key) == 0).to(DEV)
    assert torch.equal(run.r[:4][gone], run.x[gone]) and run.r[:4][~gone].isnan().all()


@pytest.mark.parametrize("c", [Case(37, 64, "f32", "none", "rms", True, True, drop=0.5),
                               Case(300, 1000, "bf16", "none", "layer", True, True, 0.7, 0.25),
                               Case(20, 7000, "bf16", "none", "rms", True, True, 0.7, 0.25),
                               Case(20, 9000, "bf16", "none", "none", True, True, 1.0, 0.5)],
                         ids=lambda c: str(c.d))
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_dropped_values_reach_no_gradient(c, value):
    """What dropout takes out of y is nothing to the gates' gradients either, whatever it was."""
    runs = [Run(c), Run(c)]
    gone = torch.from_numpy(J.keep_mask(c.T, c.d, c.drop, *runs[0].key) == 0).to(DEV)
    for run, v in zip(runs, (0.0, value)):
        run.y[gone] = v
        run.forward()
        run.backward()
    torch.cuda.synchronize()
    zero, other = (run.outputs() for run in runs)
    assert other["gate"].isfinite().all() and other["token_gate"].isfinite().all()
    for n in zero:
        assert torch.equal(zero[n], other[n]), n


@pytest.mark.parametrize("d", [512, 5000])
@pytest.mark.parametrize("where", ["y", "y_weight", "y_bias"])
def test_dropped_values_of_a_norm(d, where):
    """A NaN that y's norm spreads over a row, or its weights over a column, reaches the gates' sums of the
    elements that were kept and no others."""
    c = Case(9, d, "f32", "layer", "none", True, True, 1.0, 0.5)
    run = Run(c)
    gone = J.keep_mask(c.T, d, 0.5, *run.key) == 0
    if where == "y":
        run.y[4, 17] = float("nan")
        bad = np.zeros((9, d), bool)
        bad[4] = True
    else:
        run.p[where][17] = float("inf")
        bad = np.zeros((9, d), bool)
        bad[:, 17] = True
    run.forward()
    run.backward()
    torch.cuda.synchronize()
    bad &= ~gone
    for n, axis in (("gate", 0), ("token_gate", 1)):
        got = ~np.isfinite(to_np(run.g[n])[:bad.shape[1 - axis]])
        assert np.array_equal(got, bad.any(axis)), n


def test_no_rows():
    c = Case(0, 64, "f32", "layer", "layer", True)
    run = Run(c)
    for t in (run.x, run.y, run.dr, run.dh):
        assert t.numel() == 0
    pad = torch.zeros(64, device=DEV)
    B.moe_join_forward(run.join, pad, pad, run.params, None, run.r, run.h, run.stats)
    B.moe_join_backward(run.join, pad, pad, run.stats, run.params, None, pad, pad, run.dx, run.dy, run.grads,
                        run.ws)
    torch.cuda.synchronize()
    for n, t in run.g.items():
        assert (t[:c.d] == 0).all(), n
    run.check_guards()


def test_captured_steps_draw_new_masks():
    """A graph of both calls, replayed with another offset each time."""
    c = Case(200, 512, "bf16", "rms", "rms", True, False, 1.0, 0.3)
    run, ref = Run(c), Run(c)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run.forward()
        run.backward()
    for step in range(3):
        for q in (run, ref):
            q.rng[1] = 1000 + step
        graph.replay()
        ref.forward()
        ref.backward()
        torch.cuda.synchronize()
        for n, t in run.outputs().items():
            assert torch.equal(t, ref.outputs()[n]), (step, n)


def test_many_rows_of_few_values():
    """More rows than one launch's first blocks hold at 32 bits of a byte offset."""
    T, d = (1 << 29) // 64 + 3, 64                 # 2 GiB of fp32 rows
    j = B.join(T, d, "f32", "none", "rms", EPS, EPS)
    x = torch.zeros(T, d, device=DEV)
    x[-3:] = torch.arange(3 * d, device=DEV).view(3, d).float()
    h = torch.full((T + 1, d), 77.0, dtype=torch.bfloat16, device=DEV)
    B.moe_join_forward(j, x, None, B.join_params(), None, None, h)
    torch.cuda.synchronize()
    want = torch.from_numpy(J.norm("rms", f64(x[-3:]), eps=EPS)).to(DEV)
    assert (h[-4:-1].double() - want).abs().max() <= 1.01 * U16 * want.abs().max()
    assert (h[:-4] == 0).all() and (h[-1] == 77).all()
