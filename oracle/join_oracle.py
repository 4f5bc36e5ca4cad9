"""Joining a block to the residual stream in float64, from the definition (see
include/moe.h): norms, dropout, gates, the sum and its gradient.

Params are a dict of y_weight, y_bias, gate, token_gate, r_weight, r_bias; what
is missing or None is 1 (biases: 0).  Row statistics [T, 4] are mean and
1 / deviation of y's row, then of r's.
"""
from __future__ import annotations

import numpy as np

PARAMS = ("y_weight", "y_bias", "gate", "token_gate", "r_weight", "r_bias")
M32 = 0xFFFFFFFF


def philox(counter, key):
    """Philox4x32-10: counter of 4 and key of 2 32-bit words (arrays broadcast) -> 4 words."""
    c = [np.asarray(v, np.uint64) for v in counter]
    k = [int(v) for v in key]
    s = np.uint64(32)
    m = np.uint64(M32)
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> s) ^ c[1] ^ np.uint64(k[0]), b & m, (a >> s) ^ c[3] ^ np.uint64(k[1]), a & m]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def keep_mask(T, d, drop, seed, offset):
    """[T, d] multipliers: 0 where dropped, 1 / (share kept) elsewhere."""
    n = int(np.floor(float(np.float32(drop)) * 65536 + 0.5))
    if n == 0:
        return np.ones((T, d))
    j, t = np.meshgrid(np.arange(d // 8), np.arange(T))
    words = philox((j, t, offset & M32, offset >> 32 & M32), (seed & M32, seed >> 32 & M32))
    bits = np.empty((T, d // 8, 8), np.int64)
    for i in range(8):
        bits[:, :, i] = (np.broadcast_to(words[i // 2], j.shape) >> np.uint64(16 * (i % 2))) & np.uint64(0xFFFF)
    return (bits.reshape(T, d) >= n) * (65536 / (65536 - n))


def stats(kind, v, eps):
    """Mean and 1 / deviation of each row; zeros without a norm."""
    if kind == "none":
        return np.zeros(len(v)), np.zeros(len(v))
    m = v.mean(1) if kind == "layer" else np.zeros(len(v))
    return m, 1.0 / np.sqrt(((v - m[:, None]) ** 2).mean(1) + eps)


def _unit(kind, v, m, s):
    return v if kind == "none" else (v - m[:, None]) * s[:, None]


def _affine(u, w, b):
    u = u if w is None else u * w
    return u if b is None else u + b


def _gates(p, scale):
    a = np.full((1, 1), float(scale))
    if p.get("gate") is not None:
        a = a * p["gate"]
    return a if p.get("token_gate") is None else a * p["token_gate"][:, None]


def join_r(x, y, p, y_norm="none", eps=1e-6, scale=1.0, keep=1.0):
    """The sum, not rounded."""
    u = _unit(y_norm, y, *stats(y_norm, y, eps))
    return x + _gates(p, scale) * (_affine(u, p.get("y_weight"), p.get("y_bias")) * keep)


def norm(kind, r, w=None, b=None, eps=1e-6):
    return _affine(_unit(kind, r, *stats(kind, r, eps)), w, b)


def _norm_grad(kind, u, s, w, g, mag):
    """Gradient wrt the values under the norm; mag: of the magnitudes, nothing cancelling."""
    g = g if w is None else g * w
    if kind == "none":
        return g
    sign = 1.0 if mag else -1.0
    out = g + sign * u * (g * u).mean(1, keepdims=True)
    if kind == "layer":
        out = out + sign * g.mean(1, keepdims=True)
    return s[:, None] * out


def backward(y, r, st, p, dr, dh, y_norm="none", r_norm="rms", scale=1.0, keep=1.0, mag=False):
    """Gradients {dx, dy, parameters} of dr and dh (either None).  With mag every
    term enters with its magnitude: what the errors of a 32-bit evaluation are relative to."""
    a = np.abs if mag else (lambda v: v)
    p = {n: None if v is None else a(v) for n, v in p.items()}
    u = a(_unit(r_norm, r, st[:, 2], st[:, 3]))
    out = {}
    D = 0.0 if dr is None else a(dr)
    if dh is not None:
        D = D + _norm_grad(r_norm, u, st[:, 3], p.get("r_weight"), a(dh), mag)
        out.update(r_weight=(a(dh) * u).sum(0), r_bias=a(dh).sum(0))
    else:
        out.update(r_weight=np.zeros(r.shape[1]), r_bias=np.zeros(r.shape[1]))
    out["dx"] = D
    if y is not None:
        u = a(_unit(y_norm, y, st[:, 0], st[:, 1]))
        v = _affine(u, p.get("y_weight"), p.get("y_bias")) * keep
        dn = a(_gates(p, scale)) * D * keep
        one = {**p, "gate": None}
        out["gate"] = (a(_gates(one, scale)) * v * D).sum(0)
        one = {**p, "token_gate": None}
        out["token_gate"] = (a(_gates(one, scale)) * v * D).sum(1)
        out.update(y_weight=(dn * u).sum(0), y_bias=dn.sum(0) * np.ones(r.shape[1]))
        out["dy"] = _norm_grad(y_norm, u, st[:, 1], p.get("y_weight"), dn, mag)
    return out
