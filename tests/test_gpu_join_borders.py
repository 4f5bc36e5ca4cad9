"""Values and sizes at the borders of the residual join's forms."""
import numpy as np
import pytest
import torch

from oracle import join_oracle as J
from tests.parity import say
from tests.test_gpu_join import U32, Case, Run, f64, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("y_norm,weight,bias", [("rms", 2e37, 0.0), ("layer", 2e37, 0.0), ("layer", 6e36, 2e38)])
@pytest.mark.parametrize("T,d", [(400, 5000), (400, 8192), (20, 5000), (600, 2048)])
def test_dropped_values_that_overflow_reach_no_gradient(T, d, stream, y_norm, weight, bias):
    """Finite weights that take a normed value past the largest float: where dropout takes it out, the
    gates' sums are those of the elements that were kept, as for one that is infinite before the norm.

    Column 17 is 60 where it is dropped, 35 to 50 deviations: 7e38 or more with the first weight, 2.1e38 + 2e38 or
    more with the last.  Kept values are finite, and the scale keeps the sums in range, which the oracle's
    magnitudes have to show first."""
    say(f"[gpu] dropped {T} {d} {stream} {y_norm} {weight} {bias}")
    c = Case(T, d, stream, y_norm, "none", True, True, 1e-4, 0.5)
    run = Run(c)
    gone = J.keep_mask(T, d, 0.5, *run.key)[:, 17] == 0
    run.y[torch.from_numpy(gone).to(run.y.device), 17] = 60.0
    run.p["y_weight"][17] = weight
    if y_norm == "layer":
        run.p["y_bias"][17] = bias
    run.forward()
    run.backward()
    torch.cuda.synchronize()
    p = {n: f64(v) for n, v in run.p.items()}
    keep = J.keep_mask(T, d, 0.5, *run.key)
    args = (f64(run.y), f64(run.r[:T]), f64(run.stats[:T]), p, f64(run.dr), f64(run.dh), y_norm, "none", c.scale, keep)
    want, mag = J.backward(*args), J.backward(*args, mag=True)
    for n in ("gate", "token_gate"):
        assert (mag[n] < np.finfo(np.float32).max).all()
        terms = 3 * 64 + (T / 256 + 68 if n == "gate" else 0)      # as the join's other sums
        within("d" + n, f64(run.g[n])[:len(p[n])], want[n], terms * U32 * mag[n])
