"""The residual join's gradient in every instance that the size rules choose between up to 8192 columns, norms
with every mix of weight and bias, and rows past the forward's first launch.  Tolerances are those of the
join's other tests."""
import numpy as np
import pytest
import torch

from oracle import join_oracle as J
from paper_2609_36070_amd import binding as B
from tests.parity import say, to_np
from tests.test_gpu_join import DEV, EPS, U16, U32, Case, Run, check, f64, within

pytestmark = pytest.mark.gpu

# columns: a row count for one round of workgroups, one for more (32, 16, 8, 4, 2, 1 .. rows to a workgroup and
# 512 of them, 384 past 2048 columns), neither a multiple of a workgroup's rows
SIZES = {56: (77, 16399), 128: (37, 8205), 248: (19, 4103), 512: (11, 2051), 1000: (7, 1025), 2040: (5, 515),
         4088: (5, 387), 8184: (5, 387)}
# what the gradient has to sum and whether a layer norm is there, by which the instance is chosen
FORMS = {
    "rms, weights alone": dict(y_norm="rms", r_norm="rms", gate=True),
    "biases of the sum's norm": dict(y_norm="rms", r_norm="layer", gate=True, y_weight=False),
    "all": dict(y_norm="layer", r_norm="layer", gate=True),
}


class Weights(Run):
    """A case whose norms have the weights and biases that are named, whatever their kind."""

    def __init__(self, c, **has):
        super().__init__(c)
        rng = np.random.default_rng(c.seed + 99)
        for n, there in has.items():
            draw = torch.from_numpy((1 + 0.3 * rng.standard_normal(c.d)).astype(np.float32)).to(DEV)
            self.p[n] = draw if there else None
            self.g.pop(n, None)
            if there:
                self.g[n] = torch.full((c.d + 8,), 77.0, device=DEV)
        self.params, self.grads = B.join_params(**self.p), B.join_grads(**self.g)


def run(r):
    n = B.moe_join_workspace_bytes(r.join)
    r.ws = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    r.forward()
    r.backward()
    torch.cuda.synchronize()
    assert (r.ws[n:] == 0xA5).all()
    check(r)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("rounds", ["one", "more"])
@pytest.mark.parametrize("d", SIZES)
def test_every_instance(d, rounds, stream, form):
    T, kw = SIZES[d][rounds == "more"], dict(FORMS[form])
    has = {"y_weight": kw.pop("y_weight")} if "y_weight" in kw else {}
    say(f"[gpu] instance {T} x {d} {stream}: {form}")
    # (the mask takes the oracle longest: not with every size)
    run(Weights(Case(T, d, stream, scale=0.5, drop=0.1 if T < 1000 else 0.0, token_gate=d > 1000, **kw), **has))


@pytest.mark.parametrize("has", [dict(y_bias=True, r_bias=True), dict(y_weight=False, y_bias=True),
                                 dict(r_weight=False, r_bias=True), dict(y_bias=True), dict(r_bias=True)],
                         ids=lambda h: " ".join(n for n in h if h[n]))
@pytest.mark.parametrize("T,d", [(33, 264), (700, 1000), (390, 5000), (20, 9000)])
def test_rms_norms_with_biases(T, d, has):
    """A norm's weight and bias are there or not on their own, without a mean too."""
    say(f"[gpu] rms with biases {T} x {d} {has}")
    run(Weights(Case(T, d, "bf16" if T % 2 else "f32", "rms", "rms", True, False, 0.5), **has))


@pytest.mark.parametrize("norms", [("rms", "none"), ("none", "rms"), ("layer", "rms")])
def test_rows_past_the_first_launch(norms):
    """The forward's 2^26 rows of 8 values are a launch's 2^21 workgroups of 32; 37 more rows are the next one's.
    Rows on either side of the border and the last ones, their statistics and mask, against the oracle;
    every row's sum by what it can be."""
    y_norm, r_norm = norms
    first, d, drop, key = 1 << 26, 8, 0.5, (11, 5)
    T = first + 37
    say(f"[gpu] {T} rows, {norms}")
    g = torch.Generator(device=DEV).manual_seed(3)
    x, y = (torch.randn(T, d, generator=g, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    r, h = (torch.full((T + 1, d), 77.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    stats = torch.full((T + 1, 4), 77.0, device=DEV)
    rng = torch.tensor(key, dtype=torch.int64, device=DEV)
    B.moe_join_forward(B.join(T, d, "bf16", y_norm, r_norm, EPS, EPS, 1.0, drop), x, y, B.join_params(), rng, r, h, stats)
    torch.cuda.synchronize()
    for t in (r, h, stats):
        assert (t[T:] == 77).all()
    kept = 0                               # an element that moved was kept: half of them
    for part in range(0, T, 1 << 24):
        moved = r[part:min(part + (1 << 24), T)] != x[part:part + (1 << 24)]
        kept += int(moved.sum())
    # Bernoulli trials of 1/2: 20 deviations of sqrt(n) / 2; an addend below half a step of x leaves it too
    n = T * d
    assert kept <= n / 2 + 10 * n ** 0.5 and kept >= 0.45 * n
    rows = np.r_[0:3, first - 40:T]
    at = torch.from_numpy(rows).to(DEV)
    xs, ys = f64(x[at]), f64(y[at])
    words = J.philox((np.zeros(len(rows), np.uint64), rows, key[1], 0), (key[0], 0))
    bits = np.stack([(words[i // 2] >> np.uint64(16 * (i % 2))) & np.uint64(0xFFFF) for i in range(8)], 1)
    keep = (bits >= 32768) * 2.0
    want = J.join_r(xs, ys, {}, y_norm, EPS, 1.0, keep)
    rs, st = f64(r[at]), f64(stats[at])
    m, s = J.stats(y_norm, ys, EPS)
    u = np.abs(ys) if y_norm == "none" else (np.abs(ys) + np.abs(ys).mean(1, keepdims=True)) * s[:, None]
    within("r", rs, want, U16 * np.abs(want) * (1 + 2.0 ** -8) + 3 * 64 * U32 * (np.abs(xs) + u * keep))
    within("y's 1/deviation", st[:, 1], s, 2 * 64 * U32 * s)
    m, s = J.stats(r_norm, rs, EPS)
    within("r's 1/deviation", st[:, 3], s, 2 * 64 * U32 * s)
    want = J.norm(r_norm, rs, eps=EPS)
    u = np.abs(rs) if r_norm == "none" else np.abs(rs) * s[:, None]
    within("h", to_np(h[at]).astype(np.float64), want, U16 * np.abs(want) * (1 + 2.0 ** -8) + 3 * 64 * U32 * u)
