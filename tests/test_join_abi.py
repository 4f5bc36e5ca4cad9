"""Host-side checks of the residual join's entry points (CPU only: nothing is launched)."""
import ctypes
import math

import pytest

from paper_2609_36070_amd import binding as B

FAKE, MISALIGNED, BIG = 0x10000, 0x10008, 1 << 40
FULL = dict(y_weight=FAKE, y_bias=FAKE, gate=FAKE, token_gate=FAKE, r_weight=FAKE, r_bias=FAKE)


def _join(**kw):
    return B.join(**{**dict(T=4, d=64, y_norm="layer", r_norm="rms", drop=0.1), **kw})


def _forward(join=None, params=None, **kw):
    a = {**dict(x=FAKE, y=FAKE, rng=FAKE, r=FAKE, h=FAKE, stats=FAKE), **kw}
    return B.moe_join_forward(_join() if join is None else join, a["x"], a["y"],
                              B.join_params(**(FULL if params is None else params)), a["rng"], a["r"], a["h"],
                              a["stats"], stream=0, raise_on_error=False)


def _backward(join=None, params=None, grads=None, **kw):
    a = {**dict(y=FAKE, r=FAKE, stats=FAKE, rng=FAKE, dr=FAKE, dh=FAKE, dx=FAKE, dy=FAKE, ws=FAKE,
                ws_bytes=BIG), **kw}
    return B.moe_join_backward(_join() if join is None else join, a["y"], a["r"], a["stats"],
                               B.join_params(**(FULL if params is None else params)), a["rng"], a["dr"],
                               a["dh"], a["dx"], a["dy"], B.join_grads(**(FULL if grads is None else grads)),
                               a["ws"], a["ws_bytes"], stream=0, raise_on_error=False)


@pytest.mark.parametrize("call", (_forward, _backward))
def test_join_ranges(call):
    for field, value in [("T", -1), ("d", 0), ("stream_type", 2), ("stream_type", -1), ("y_norm", 3),
                         ("r_norm", -1), ("y_eps", 0.0), ("y_eps", math.nan), ("r_eps", -1e-6),
                         ("r_eps", math.inf), ("scale", math.nan), ("scale", math.inf), ("drop", 1.0),
                         ("drop", -0.1), ("drop", math.nan), ("drop", 1 - 2.0 ** -20)]:
        j = _join()
        setattr(j, field, value)
        assert call(j) == B.MOE_EINVAL, (field, value)
    for kw in (dict(d=60), dict(d=16392), dict(T=1 << 31)):
        assert call(_join(**kw)) == B.MOE_EUNSUPPORTED, kw
        assert B.moe_join_workspace_bytes(_join(**kw)) == 0


@pytest.mark.parametrize("call", (_forward, _backward))
def test_parameters_belong_to_what_is_there(call):
    assert call(params={**FULL, "gate": MISALIGNED}) == B.MOE_EINVAL
    assert call(_join(y_norm="none")) == B.MOE_EINVAL          # weights of no norm
    assert call(_join(r_norm="none")) == B.MOE_EINVAL
    assert call(_join(drop=0.0)) == B.MOE_EINVAL               # a generator without dropout
    assert call(rng=None) == B.MOE_EINVAL
    assert call(rng=MISALIGNED) == B.MOE_EINVAL
    # a norm before the first block: nothing that belongs to a block
    alone = dict(y_norm="none", drop=0.0)
    p = dict(r_weight=FAKE)
    none = dict(y=None, rng=None, r=None) if call is _forward else dict(y=None, rng=None, dy=None, grads={})
    assert call(_join(**alone), {**p, "gate": FAKE}, **none) == B.MOE_EINVAL
    assert call(_join(**alone), {**p, "token_gate": FAKE}, **none) == B.MOE_EINVAL
    assert call(_join(y_norm="rms", drop=0.0), p, **none) == B.MOE_EINVAL
    assert call(_join(y_norm="none"), p, **{**none, "rng": FAKE}) == B.MOE_EINVAL


def test_forward_pointers():
    for name in ("x", "y", "r", "h", "stats"):
        assert _forward(**{name: MISALIGNED}) == B.MOE_EINVAL, name
    assert _forward(x=None) == B.MOE_EINVAL
    assert _forward(r=None) == B.MOE_EINVAL                    # a block's sum goes somewhere
    assert _forward(h=None) == B.MOE_EINVAL                    # a norm without its output
    assert _forward(_join(y_norm="none", drop=0.0), {}, y=None, rng=None) == B.MOE_EINVAL   # r of no block
    L, ref = B.lib(), ctypes.byref
    assert L.moe_join_forward(None, *[FAKE] * 2, ref(B.join_params()), *[FAKE] * 4, None) == B.MOE_EINVAL
    assert L.moe_join_forward(ref(_join()), *[FAKE] * 2, None, *[FAKE] * 4, None) == B.MOE_EINVAL


def test_backward_pointers():
    for name in ("y", "r", "stats", "dr", "dh", "dx", "dy", "ws"):
        assert _backward(**{name: MISALIGNED}) == B.MOE_EINVAL, name
    for name in ("r", "stats", "dx", "ws", "dy", "y"):
        assert _backward(**{name: None}) == B.MOE_EINVAL, name
    assert _backward(dr=None, dh=None) == B.MOE_EINVAL
    for name in FULL:
        assert _backward(params={**FULL, name: None}) == B.MOE_EINVAL, name    # gradient of nothing
        assert _backward(grads={**FULL, name: MISALIGNED}) == B.MOE_EINVAL, name
    assert _backward(ws_bytes=B.moe_join_workspace_bytes(_join()) - 1) == B.MOE_ENOSPACE


@pytest.mark.parametrize("d", (8, 512, 1000, 2048, 7168, 16384))
def test_workspace_never_falls(d):
    sizes = [B.moe_join_workspace_bytes(B.join(T, d)) for T in (0, 1, 7, 255, 256, 257, 5000, 1 << 30)]
    assert sizes[0] > 0 and sizes == sorted(sizes)


def test_empty_forward_is_accepted():
    assert _forward(_join(T=0)) == B.MOE_OK


def test_a_block_refuses_parameters_that_it_does_not_have():
    from paper_2609_36070_amd.layer import DeviceBlock
    from paper_2609_36070_amd.workloads import Workload
    with pytest.raises(ValueError, match="y_wieght"):
        DeviceBlock(Workload("few", T=6, d=256, E=8, k=2, f=256), {}, {"y_wieght": None, "gate": None}, device="cpu")
