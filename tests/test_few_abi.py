"""Host-side checks of the few-token layer's entry point (CPU only: nothing is launched)."""
import ctypes

import pytest

from paper_2609_36070_amd import binding as B

FAKE, MISALIGNED, BIG = 0x10000, 0x10008, 1 << 40
OK = B.make_shape(4, 256, 8, 2, 256)


def _few(shape=OK, routing=None, weights=None, **kw):
    a = {**dict(X=FAKE, W_r=FAKE, bias=None, balance=None, logits=FAKE, topk_idx=FAKE, topk_w=FAKE, Y=FAKE,
                ws=FAKE, ws_bytes=BIG), **kw}
    w = B.weights_struct(*([FAKE] * 3 if weights is None else weights))
    return B.moe_forward_few(shape, B.routing() if routing is None else routing, a["X"], a["W_r"], a["bias"],
                             a["balance"], w, a["logits"], a["topk_idx"], a["topk_w"], a["Y"], a["ws"],
                             a["ws_bytes"], stream=0, raise_on_error=False)


def test_pointers():
    for name in ("X", "W_r", "logits", "topk_idx", "topk_w", "Y", "ws"):
        assert _few(**{name: None}) == B.MOE_EINVAL, name
    for name in ("X", "W_r", "bias", "balance", "logits", "topk_idx", "topk_w", "Y", "ws"):
        assert _few(**{name: MISALIGNED}) == B.MOE_EINVAL, name
    for i in range(3):
        w = [FAKE] * 3
        w[i] = None
        assert _few(weights=w) == B.MOE_EINVAL
    assert _few(weights=[FAKE] * 6) == B.MOE_EINVAL                 # a shared expert that is not there
    assert _few(B.make_shape(4, 256, 8, 2, 256, 256)) == B.MOE_EINVAL
    L, ref = B.lib(), ctypes.byref
    w = B.weights_struct(FAKE, FAKE, FAKE)
    tail = [FAKE] * 4 + [FAKE, BIG, None]
    assert L.moe_forward_few(ref(OK), None, FAKE, FAKE, None, None, ref(w), *tail) == B.MOE_EINVAL
    assert L.moe_forward_few(None, ref(B.routing()), FAKE, FAKE, None, None, ref(w), *tail) == B.MOE_EINVAL
    assert L.moe_forward_few(ref(OK), ref(B.routing()), FAKE, FAKE, None, None, None, *tail) == B.MOE_EINVAL


def test_shapes_and_routings():
    for kw in (dict(T=17), dict(T=1 << 20), dict(d=192), dict(f=100), dict(E=300), dict(k=17, E=20)):
        s = {**dict(T=4, d=256, E=8, k=2, f=256), **kw}
        assert _few(B.make_shape(*s.values())) == B.MOE_EUNSUPPORTED, kw
        assert B.moe_few_workspace_bytes(B.make_shape(*s.values())) == 0
    assert _few(B.make_shape(4, 256, 8, 9, 256)) == B.MOE_EINVAL
    assert _few(B.make_shape(-1, 256, 8, 2, 256)) == B.MOE_EINVAL
    bad = B.routing()
    bad.score = 9
    assert _few(routing=bad) == B.MOE_EINVAL
    assert _few(routing=B.routing(groups=8, top_groups=1)) == B.MOE_EINVAL      # 1 expert, k = 2


@pytest.mark.parametrize("layer", [(256, 1, 1, 256, 0), (2048, 128, 8, 768, 0), (7168, 256, 8, 512, 512),
                                   (7168, 8, 8, 2048, 2048), (1 << 20, 4, 2, 256, 256), (256, 256, 16, 1 << 20, 0)])
def test_workspace(layer):
    sizes = [B.moe_few_workspace_bytes(B.make_shape(T, *layer)) for T in range(17)]
    assert sizes[0] > 0 and sizes == sorted(sizes)
    sh = B.make_shape(16, *layer)
    w = [FAKE] * (6 if layer[4] else 3)
    assert _few(sh, weights=w, ws_bytes=sizes[16] - 1) == B.MOE_ENOSPACE
    d, E, k, f, fs = layer
    # H of every route in two bf16 parts
    assert sizes[16] >= 16 * 4 * (min(E, 16 * k) * f + fs)
    assert _few(B.make_shape(0, *layer), weights=w, ws_bytes=sizes[0]) == B.MOE_OK
