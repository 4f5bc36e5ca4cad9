"""The few-token path of a layer is for inference: it leaves no plan and no activations and takes the
workspace that a backward reads (CPU: nothing is launched)."""
import pytest

from paper_2609_36070_amd.layer import DeviceLayer
from paper_2609_36070_amd.workloads import Workload, make_inputs

W = Workload("few", T=6, d=256, E=8, k=2, f=256)


def test_a_layer_with_a_backward_has_no_few_token_path():
    with pytest.raises(ValueError, match="backward"):
        DeviceLayer(W, make_inputs(W, 0), device="cpu", with_backward=True, few=True)
    # a training layer's workspace is large enough for the call, which would write over its activations
    with pytest.raises(ValueError, match="backward"):
        DeviceLayer(W, make_inputs(W, 0), device="cpu", with_backward=True).step_few(stream=0)


def test_one_without_has():
    assert DeviceLayer(W, make_inputs(W, 0), device="cpu", with_backward=False, few=True).ws.nbytes > 0
