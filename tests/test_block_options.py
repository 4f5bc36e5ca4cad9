"""What a block does with the options of its layer (CPU: nothing is launched)."""
import pytest

from paper_2609_36070_amd.layer import DeviceBlock
from paper_2609_36070_amd.workloads import Workload, make_inputs

W = Workload("few", T=6, d=256, E=8, k=2, f=256)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("option", ["mx", "mx_wgrad", "int8"])
def test_experts_that_a_block_does_not_run_are_refused(option, backward):
    with pytest.raises(ValueError, match=option):
        DeviceBlock(W, {}, device="cpu", with_backward=backward, **{option: True})


def test_options_that_are_off_are_none():
    block = DeviceBlock(W, make_inputs(W, 0), device="cpu", mx=False, int8=False)
    assert block.few and not block.layer.mx and not block.layer.int8


@pytest.mark.parametrize("backward", [False, True])
def test_bounded_memory_is_what_runs_where_it_is_asked_for(backward):
    """Few tokens too: the layer holds a ring of rows, and the block takes the path that stays in it."""
    block = DeviceBlock(W, make_inputs(W, 0), device="cpu", with_backward=backward, ring_rows=256)
    assert not block.few and block.layer.ring_rows == 256
    assert DeviceBlock(W, make_inputs(W, 0), device="cpu", with_backward=False).few
