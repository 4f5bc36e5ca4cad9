"""Routing by scores in float64, from the definition (see include/moe.h).

Z [T, E] logits; balance [E] or None; score "softmax" or "sigmoid"; groups of
E / groups consecutive experts, the best top_groups of which are kept
(group_score "max" or "pair"); weights scale * s, over the chosen scores' sum
if renormalise.  Loops over tokens: plain, not fast.
"""
from __future__ import annotations

import numpy as np

MASKED = -1e38
FLT_MAX = float(np.finfo(np.float32).max)


def in_play(Z, balance=None):
    """[T, E] bool: experts that are not masked."""
    Z = np.asarray(Z, np.float64)
    live = Z >= MASKED               # NaN compares false
    if balance is not None:
        live = live & (np.asarray(balance, np.float64) >= MASKED)[None]
    return live


def _clamped(Z, live):
    return np.where(live, np.minimum(np.asarray(Z, np.float64), FLT_MAX), 0.0)


def scores(Z, live, score):
    """[T, E] scores; 0 for masked experts."""
    z = _clamped(Z, live)
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return np.where(live, 1.0 / (1.0 + np.exp(-z)), 0.0)
    top = np.where(live, z, -np.inf).max(1, keepdims=True)
    e = np.where(live, np.exp(z - np.where(np.isfinite(top), top, 0.0)), 0.0)
    total = e.sum(1, keepdims=True)
    return np.where(total > 0, e / np.where(total > 0, total, 1.0), 0.0)


def ranking_values(Z, balance, score, groups, group_score):
    """The values experts are ranked by; -inf where masked."""
    live = in_play(Z, balance)
    if balance is None and not (groups > 1 and group_score == "pair"):
        v = _clamped(Z, live)
    else:
        v = scores(Z, live, score)
        if balance is not None:
            v = v + np.where(np.asarray(balance) >= MASKED, np.asarray(balance, np.float64), 0.0)[None]
    return np.where(live, v, -np.inf)


def select(Z, balance, k, score, groups=1, top_groups=1, group_score="max"):
    """[T, k] chosen ids, ascending."""
    V = ranking_values(Z, balance, score, groups, group_score)
    T, E = V.shape
    n = E // groups
    out = np.empty((T, k), np.int32)
    for t in range(T):
        kept = np.ones(E, bool)
        if groups > 1:
            gs = []
            for g in range(groups):
                best = np.sort(V[t, g * n:(g + 1) * n])[::-1]
                pair = group_score == "pair" and n > 1 and best[1] > -np.inf
                gs.append(best[0] + best[1] if pair else best[0])
            order = sorted(range(groups), key=lambda g: (-gs[g], g))[:top_groups]
            kept[:] = False
            for g in order:
                kept[g * n:(g + 1) * n] = True
        order = sorted((e for e in range(E) if kept[e]), key=lambda e: (-V[t, e], e))
        out[t] = sorted(order[:k])
    return out


def _log_scores(Z, live, score):
    z = _clamped(Z, live)
    if score == "sigmoid":
        return -np.logaddexp(0.0, -z)
    top = np.where(live, z, -np.inf).max(1, keepdims=True)
    top = np.where(np.isfinite(top), top, 0.0)
    total = np.where(live, np.exp(z - top), 0.0).sum(1, keepdims=True)
    return z - top - np.log(np.where(total > 0, total, 1.0))


def unscaled_weights(Z, balance, idx, score, renormalise):
    live = in_play(Z, balance)
    logs = np.take_along_axis(np.where(live, _log_scores(Z, live, score), -np.inf), idx, 1)
    if renormalise:      # ratios, so that scores that underflow together keep theirs
        top = logs.max(1, keepdims=True)
        logs = logs - np.where(np.isfinite(top), top, 0.0)
    u = np.exp(logs)
    if renormalise:
        total = u.sum(1, keepdims=True)
        u = np.where(total > 0, u / np.where(total > 0, total, 1.0), 0.0)
    return u


def weights(Z, balance, idx, score, renormalise, scale):
    return scale * unscaled_weights(Z, balance, idx, score, renormalise)


def score_backward(Z, balance, idx, dw, score, renormalise, scale):
    """dZ [T, E]: gradient wrt the logits for dw [T, k] = dL/dweights."""
    live = in_play(Z, balance)
    T, E = live.shape
    u = unscaled_weights(Z, balance, idx, score, renormalise)
    s, z = scores(Z, live, score), _clamped(Z, live)
    dZ = np.zeros((T, E))
    for t in range(T):
        on = live[t, idx[t]]
        g = np.where(on, dw[t], 0.0)
        dot = float((u[t] * g).sum())
        d = scale * u[t] * (g - dot if renormalise else g)
        if score == "sigmoid":
            with np.errstate(over="ignore"):
                d = d / (1.0 + np.exp(z[t, idx[t]]))
        elif not renormalise:
            dZ[t] = -s[t] * scale * dot
        for i, e in enumerate(idx[t]):
            if on[i]:
                dZ[t, e] += d[i]
    return dZ
