"""The experts in 8-bit integers, in float64 but for what the definition fixes
in float32: a row's scale amax / 127 and the quotient x / scale that is rounded
to a code (see include/moe.h).
"""
from __future__ import annotations

import numpy as np

from . import moe_oracle as O


def quantize_rows(x):
    """(codes int64, scales float32) of the rows (last axis) of x; the codes of
    values given in float64 come from the float32-rounded quotient."""
    x = np.asarray(x)
    with np.errstate(all="ignore"):
        amax = np.abs(x).max(-1, keepdims=True) if x.shape[-1] else np.zeros(x.shape[:-1] + (1,))
        s = (np.float32(1) * amax.astype(np.float32)) / np.float32(127)
        bad = ~np.isfinite(amax)
        s = np.where(bad, np.float32(np.nan), s).astype(np.float32)
        den = np.where(s > 0, s, np.float32(1))
        q = x.astype(np.float32) / den if x.dtype == np.float32 else (x / den.astype(np.float64)).astype(np.float32)
        q = np.where(s > 0, np.clip(np.rint(q), -127, 127), 0.0)
    return q.astype(np.int64), s[..., 0]


def quantize_weights(W):
    """Per-channel codes [N, K] and scales [N] of W [K, N] (float32)."""
    return quantize_rows(np.ascontiguousarray(np.asarray(W, np.float32).T))


def ffn_rows(xq, xs, g, u, d):
    """(y, h, near): outputs of rows of codes through one expert, its gated
    activation, and the codes' distance-to-a-tie data used by bounds.
    g, u, d: (codes [N, K], scales [N])."""
    a = (xq @ g[0].T).astype(np.float64) * xs[:, None].astype(np.float64) * g[1].astype(np.float64)
    b = (xq @ u[0].T).astype(np.float64) * xs[:, None].astype(np.float64) * u[1].astype(np.float64)
    h = O.silu(a) * b
    hq, hs = quantize_rows(h)
    y = (hq @ d[0].T).astype(np.float64) * hs[:, None].astype(np.float64) * d[1].astype(np.float64)
    return y, a, h, hq, hs


def tie_codes(a, h, hs, extra):
    """[rows, f] bool: codes that a relative error of the 32-bit evaluation can
    move to the neighbouring integer, besides an absolute error of `extra` codes."""
    q = np.abs(h) / np.maximum(hs[:, None].astype(np.float64), 1e-300)
    rel = lambda v: (32 + 4 * np.abs(v)) * 2.0 ** -24   # noqa: E731
    top = np.take_along_axis(a, np.abs(h).argmax(1)[:, None], 1)
    eps = q * (rel(a) + rel(top)) + extra
    return np.abs(q - np.floor(q) - 0.5) <= eps


def moe_forward_int(X, Wq, idx, w, extra=0.0):
    """Y [T, d] and an elementwise bound on an implementation's distance from
    it.  Wq: codes and scales per expert, {"g": [...], "u": [...], "d": [...]},
    and "gs", "us", "ds" of the shared expert if there is one."""
    X = np.asarray(X, np.float32)
    T, d = X.shape
    xq, xs = quantize_rows(X)
    Y, tol = np.zeros((T, d)), np.zeros((T, d))

    def add(t, wt, g, u, dn):
        y, a, h, hq, hs = ffn_rows(xq[t], xs[t], g, u, dn)
        near = tie_codes(a, h, hs, extra)
        flip = near.astype(np.float64) @ np.abs(dn[0]).T.astype(np.float64)
        off = flip * hs[:, None].astype(np.float64) * dn[1].astype(np.float64)
        # the scale hs carries the error of the largest value; the output rounds to
        # bf16: half a step of the computed value, which is at most |y| + off
        off += (np.abs(y) + off) * (2.0 ** -8 + 200 * 2.0 ** -24)
        np.add.at(Y, t, wt[:, None] * y)      # a token may list an expert twice
        np.add.at(tol, t, np.abs(wt)[:, None] * off)

    for e in range(len(Wq["g"])):
        t, s = np.nonzero(idx == e)
        if len(t):
            add(t, w[t, s].astype(np.float64), Wq["g"][e], Wq["u"][e], Wq["d"][e])
    if "gs" in Wq:
        add(np.arange(T), np.ones(T), Wq["gs"], Wq["us"], Wq["ds"])
    return Y, tol + (np.abs(Y) + tol) * 2.0 ** -8 + 1e-30
