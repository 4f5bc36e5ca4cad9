"""Host-side checks of the scored router's and the int8 experts' entry points
(CPU only: nothing is launched)."""
import ctypes
import math

import pytest

from paper_2609_36070_amd import binding as B
from paper_2609_36070_amd.workloads import WORKLOADS

FAKE, MISALIGNED, BIG = 0x10000, 0x10008, 1 << 40
OK = B.make_shape(64, 256, 8, 2, 256)


def _route(shape=OK, routing=None, **kw):
    a = dict(X=FAKE, W_r=FAKE, bias=None, balance=None, logits=FAKE, topk_idx=FAKE, topk_w=FAKE, ws=FAKE,
             ws_bytes=BIG)
    a.update(kw)
    r = B.routing() if routing is None else routing
    return B.lib().moe_route_scored(ctypes.byref(shape), ctypes.byref(r), a["X"], a["W_r"], a["bias"],
                                    a["balance"], a["logits"], a["topk_idx"], a["topk_w"], a["ws"],
                                    a["ws_bytes"], None)


def _grad(shape=OK, routing=None, **kw):
    a = dict(logits=FAKE, balance=None, topk_idx=FAKE, dw=FAKE, dZ=FAKE)
    a.update(kw)
    r = B.routing() if routing is None else routing
    return B.lib().moe_score_backward(ctypes.byref(shape), ctypes.byref(r), a["logits"], a["balance"],
                                      a["topk_idx"], a["dw"], a["dZ"], None)


def _bad_routings():
    for field, value in [("score", 2), ("score", -1), ("group_score", 2), ("renormalise", 2),
                         ("groups", 0), ("groups", 3), ("groups", -1), ("top_groups", 0),
                         ("top_groups", 2), ("scale", math.nan), ("scale", math.inf)]:
        r = B.routing()
        setattr(r, field, value)
        yield field, value, r
    yield "experts of the kept groups", 1, B.routing(groups=8, top_groups=1)   # 1 expert, k = 2


@pytest.mark.parametrize("field,value,r", _bad_routings(), ids=lambda v: str(v) if not isinstance(v, B.MoeRouting) else "")
def test_routing_ranges(field, value, r):
    for call in (_route, _grad):
        assert call(routing=r) == B.MOE_EINVAL
    sh = B.make_shape(64, 256, 128, 2, 256)
    many = B.routing(groups=128)
    assert _route(sh, many) == B.MOE_EUNSUPPORTED
    assert _grad(sh, many) == B.MOE_EUNSUPPORTED


def test_route_scored_validation():
    for name in ("X", "W_r", "logits", "topk_idx", "topk_w", "ws"):
        assert _route(**{name: None}) == B.MOE_EINVAL, name
    for name in ("X", "W_r", "bias", "balance", "logits", "topk_idx", "topk_w", "ws"):
        assert _route(**{name: MISALIGNED}) == B.MOE_EINVAL, name
    assert _route(ws_bytes=16) == B.MOE_ENOSPACE
    assert _route(B.make_shape(64, 192, 8, 2, 256)) == B.MOE_EUNSUPPORTED
    assert _route(B.make_shape(64, 256, 8, 9, 256)) == B.MOE_EINVAL
    assert B.lib().moe_route_scored(ctypes.byref(OK), None, *[FAKE] * 8, BIG, None) == B.MOE_EINVAL


def test_score_backward_validation():
    for name in ("logits", "topk_idx", "dw", "dZ"):
        assert _grad(**{name: None}) == B.MOE_EINVAL, name
        assert _grad(**{name: MISALIGNED}) == B.MOE_EINVAL, name
    assert _grad(balance=MISALIGNED) == B.MOE_EINVAL
    assert _grad(B.make_shape(64, 256, 300, 2, 256)) == B.MOE_EUNSUPPORTED


def test_scored_backwards_validate_routing_and_logits():
    L = B.lib()
    plan = B.MoePlanBufs(FAKE, FAKE, FAKE, FAKE)
    w = B.MoeWeights(FAKE, FAKE, FAKE, None, None, None)
    mx = B.MoeMxBwdWeights(*[FAKE] * 6)
    g = B.MoeGrads(FAKE, FAKE, FAKE, FAKE, None, None, None, None)
    ref = ctypes.byref

    def calls(routing, logits, balance, ws_bytes):
        head = [ref(OK), ref(routing), logits, balance, FAKE, FAKE, FAKE, ref(w)]
        tail = [FAKE, FAKE, ref(plan), FAKE, ref(g)]
        yield L.moe_backward_scored(*head, *tail, FAKE, ws_bytes, None, None)
        yield L.moe_backward_ring_scored(*head, *tail, 64, FAKE, ws_bytes, None)
        yield L.moe_backward_mx_scored(*head, ref(mx), *tail, 0, FAKE, ws_bytes, None)

    bad = B.routing()
    bad.score = 7
    assert set(calls(bad, FAKE, None, BIG)) == {B.MOE_EINVAL}
    assert set(calls(B.routing(), None, None, BIG)) == {B.MOE_EINVAL}
    assert set(calls(B.routing(), FAKE, MISALIGNED, BIG)) == {B.MOE_EINVAL}
    assert set(calls(B.routing(), FAKE, None, 64)) == {B.MOE_ENOSPACE}


def _ints(shared=False):
    return [FAKE] * 6 + [FAKE if shared else None] * 6


def _forward(shape=OK, weights=None, **kw):
    a = dict(X=FAKE, topk_idx=FAKE, topk_w=FAKE, Y=FAKE, ws=FAKE, ws_bytes=BIG)
    a.update(kw)
    w = B.MoeIntWeights(*(_ints() if weights is None else weights))
    plan = B.MoePlanBufs(*kw.get("plan", [FAKE] * 4))
    return B.lib().moe_forward_int(ctypes.byref(shape), a["X"], ctypes.byref(w), a["topk_idx"], a["topk_w"],
                                   ctypes.byref(plan), a["Y"], a["ws"], a["ws_bytes"], None, None)


def test_forward_int_validation():
    for name in ("X", "topk_idx", "topk_w", "Y", "ws"):
        assert _forward(**{name: None}) == B.MOE_EINVAL, name
        assert _forward(**{name: MISALIGNED}) == B.MOE_EINVAL, name
    for i in range(6):
        w = _ints()
        w[i] = None
        assert _forward(weights=w) == B.MOE_EINVAL
    shared = B.make_shape(64, 256, 8, 2, 256, 256)
    assert _forward(shared) == B.MOE_EINVAL                        # no shared weights
    assert _forward(OK, _ints(True)) == B.MOE_EINVAL               # shared weights of no shared expert
    assert _forward(plan=[FAKE, None, FAKE, FAKE]) == B.MOE_EINVAL
    need = B.moe_int_workspace_bytes(OK)
    assert need > 0 and _forward(ws_bytes=need - 1) == B.MOE_ENOSPACE
    assert _forward(B.make_shape(64, 1 << 18, 8, 2, 256)) == B.MOE_EUNSUPPORTED    # d > 2^17
    assert _forward(B.make_shape(1 << 23, 512, 8, 2, 256)) == B.MOE_EUNSUPPORTED   # T d >= 2^32


def test_quantize_weights_validation():
    call = B.lib().moe_int_quantize_weights
    w = B.MoeWeights(FAKE, FAKE, FAKE, None, None, None)
    q = B.MoeIntWeights(*_ints())
    ref = ctypes.byref
    assert call(ref(OK), ref(B.MoeWeights(FAKE, None, FAKE, None, None, None)), ref(q), None) == B.MOE_EINVAL
    assert call(ref(OK), ref(w), ref(B.MoeIntWeights(*_ints(True))), None) == B.MOE_EINVAL
    assert call(ref(OK), None, ref(q), None) == B.MOE_EINVAL
    assert call(ref(OK), ref(w), None, None) == B.MOE_EINVAL
    assert call(ref(B.make_shape(64, 1 << 20, 8, 2, 256)), ref(w), ref(q), None) == B.MOE_EUNSUPPORTED


@pytest.mark.parametrize("name", sorted(WORKLOADS))
def test_int_workspace(name):
    """Holds what a one-pass bf16 forward's routes need, never falls with T, and
    serves the router and the plan."""
    w = WORKLOADS[name]
    sizes = [B.moe_int_workspace_bytes(B.make_shape(t, w.d, w.E, w.k, w.f, w.f_s))
             for t in sorted((0, 1, 16, 17, 64, 65, 1000, w.T))]
    assert sizes == sorted(sizes)
    sh = B.make_shape(w.T, w.d, w.E, w.k, w.f, w.f_s)
    assert B.moe_int_workspace_bytes(sh) >= w.T * w.d + w.T * w.k * (w.f + 2 * w.d)
    assert _route(sh, ws_bytes=0) == B.MOE_ENOSPACE
    assert B.moe_int_workspace_bytes(B.make_shape(16, 100, 8, 2, 256)) == 0
    assert B.moe_int_workspace_bytes(B.make_shape(16, 1 << 18, 8, 2, 256)) == 0
