"""A block whose layer runs in bounded memory, with few tokens too."""
import pytest
import torch

from oracle import join_oracle as J
from paper_2609_36070_amd import binding as B
from paper_2609_36070_amd.layer import DeviceLayer
from tests.parity import assert_close, say, to_np
from tests.test_gpu_block import EPS, f64, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,ring_rows", [(5, 20), (16, 64), (16, 17), (40, 160)])
def test_the_ring_is_what_runs(T, ring_rows):
    """With a window of all routes the layer's output is that of the one-pass path, bit for bit; with several it
    differs by the order of its sums."""
    say(f"[gpu] block of {T} tokens in a ring of {ring_rows}")
    routing = B.routing("sigmoid", scale=1.5)
    w, inp, p, block = make(T, "bf16", "rms", "rms", 0.0, False, E=16, k=4, routing=routing, ring_rows=ring_rows)
    assert not block.few
    block.forward()
    torch.cuda.synchronize()
    plain = DeviceLayer(w, {**inp, "X": to_np(block.layer.X)}, routing=routing, with_backward=False)
    plain.step()
    torch.cuda.synchronize()
    assert torch.equal(plain.topk_idx, block.layer.topk_idx)
    if ring_rows >= T * w.k:
        assert torch.equal(plain.Y, block.layer.Y)
    else:
        assert_close("y", f64(block.layer.Y), f64(plain.Y))
    want = J.join_r(f64(block.x), f64(block.layer.Y), {n: p.get(n) for n in J.PARAMS}, "rms", EPS, 0.5)
    assert_close("r", f64(block.r), want)
