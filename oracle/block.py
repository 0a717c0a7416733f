"""The operators around the layer in float64: block norms, router, expert order, clipping.

Written from the definitions, row by row, for small sizes. Where a function returns pairs, the
second of each is the sum of the magnitudes of the terms that the first adds up: rounding errors
of a sum are bounded by a multiple of it (not of the value, which may cancel).
"""
from __future__ import annotations

import math

import numpy as np


def _or_ones(a, n):
    return np.ones(n) if a is None else np.asarray(a, dtype=np.float64)


def norm_forward(X, Y, *, pre, post, w_pre=None, w_post=None, gate_c=None, gate_t=None, res_scale=1.0, eps=1e-6):
    """(X_out, scale), (N, scale) or None."""
    T, d = X.shape
    gt, u = _or_ones(gate_t, T), _or_ones(w_post, d) * _or_ones(gate_c, d)
    X_out, X_scale = res_scale * X, np.abs(res_scale * X)
    if Y is not None:
        ry = 1 / np.sqrt((Y * Y).mean(1) + eps) if post else np.ones(T)
        P = (gt * ry)[:, None] * u * Y
        X_out, X_scale = X_out + P, X_scale + np.abs(P)
    if not pre:
        return (X_out, X_scale), None
    rx = 1 / np.sqrt((X_out * X_out).mean(1) + eps)
    w = _or_ones(w_pre, d)
    # an error of X_out moves N directly and through the mean square, by at most as much again
    N_scale = np.abs(w) * rx[:, None] * (X_scale + np.abs(X_out) * ((np.abs(X_out) * X_scale).mean(1) * rx * rx)[:, None])
    return (X_out, X_scale), (w * rx[:, None] * X_out, N_scale)


def norm_backward(X_out, Y, dX_out, dN, *, pre, post, w_pre=None, w_post=None, gate_c=None, gate_t=None, res_scale=1.0,
                  eps=1e-6):
    """{name: (gradient, scale)} of sum(dX_out * X_out) + sum(dN * N)."""
    like = dX_out if dX_out is not None else X_out
    T, d = like.shape
    gt, gc, wp = _or_ones(gate_t, T), _or_ones(gate_c, d), _or_ones(w_post, d)
    D = np.zeros((T, d)) if dX_out is None else dX_out.copy()
    S = np.abs(D)
    out = {}
    if pre:
        rx = 1 / np.sqrt((X_out * X_out).mean(1) + eps)
        xh = X_out * rx[:, None]
        dn = np.zeros((T, d)) if dN is None else dN
        g = dn * _or_ones(w_pre, d)
        D = D + rx[:, None] * (g - xh * (g * xh).mean(1)[:, None])
        S = S + rx[:, None] * (np.abs(g) + np.abs(xh) * np.abs(g * xh).mean(1)[:, None])
        out["dw_pre"] = (dn * xh).sum(0), np.abs(dn * xh).sum(0)
    out["dX"] = res_scale * D, abs(res_scale) * S
    if Y is not None:
        ry = 1 / np.sqrt((Y * Y).mean(1) + eps) if post else np.ones(T)
        yh = Y * ry[:, None]
        h, hs = gt[:, None] * gc * wp * D, np.abs(gt[:, None] * gc * wp) * S
        dY, ds = ry[:, None] * h, ry[:, None] * hs
        if post:
            dY = dY - ry[:, None] * yh * (h * yh).mean(1)[:, None]
            ds = ds + ry[:, None] * np.abs(yh) * (hs * np.abs(yh)).mean(1)[:, None]
        out["dY"] = dY, ds
        s, ss = (gt[:, None] * D * yh).sum(0), (np.abs(gt)[:, None] * S * np.abs(yh)).sum(0)
        out["dw_post"] = gc * s, np.abs(gc) * ss
        out["dgate_c"] = wp * s, np.abs(wp) * ss
        out["dgate_t"] = (gc * wp * D * yh).sum(1), (np.abs(gc * wp) * S * np.abs(yh)).sum(1)
    return out


def route_forward(logits, k, normalise=True, scale=1.0):
    """expert [T][k], weight [T][k]."""
    T, E = logits.shape
    expert, weight = np.full((T, k), -1, dtype=np.int32), np.zeros((T, k))
    for t in range(T):
        free = [e for e in range(E) if logits[t, e] > -math.inf]  # NaN is not
        chosen = sorted(free, key=lambda e: (-logits[t, e], e))[:k]
        if not chosen:
            continue
        with np.errstate(invalid="ignore"):
            ex = {e: np.exp(logits[t, e] - logits[t, chosen[0]]) for e in free}
        Z = sum(ex[e] for e in (chosen if normalise else free))
        for j, e in enumerate(chosen):
            expert[t, j], weight[t, j] = e, scale * (ex[e] / Z)
    return expert, weight


def route_backward(logits, expert, dweight, normalise=True, scale=1.0):
    """(dlogits, scale)."""
    dl, sc = np.zeros(logits.shape), np.zeros(logits.shape)
    for t in range(logits.shape[0]):
        chosen = {int(e): scale * dweight[t, j] for j, e in enumerate(expert[t]) if e >= 0}
        free = [e for e in range(logits.shape[1]) if logits[t, e] > -math.inf]
        over = list(chosen) if normalise else free
        if not over:
            continue
        top = max(logits[t, e] for e in over)
        p = {e: math.exp(logits[t, e] - top) for e in over}
        Z = sum(p.values())
        mean = sum(p[e] / Z * chosen[e] for e in chosen)
        mean_abs = sum(p[e] / Z * abs(chosen[e]) for e in chosen)
        for e in over:
            dl[t, e] = p[e] / Z * (chosen.get(e, 0.0) - mean)
            sc[t, e] = p[e] / Z * (abs(chosen.get(e, 0.0)) + mean_abs)
    return dl, sc


def expert_order(expert, E):
    """pos [T][k] and offsets [E + 1]."""
    pos, offsets, row = np.full(expert.shape, -1, dtype=np.int32), np.zeros(E + 1, dtype=np.int32), 0
    flat, out = expert.reshape(-1), pos.reshape(-1)
    for e in range(E):
        offsets[e] = row
        for s in np.nonzero(flat == e)[0]:
            out[s] = row
            row += 1
    offsets[E] = row
    return pos, offsets


def expert_combine(Ys, pos, weight=None):
    """(Y, scale)."""
    T, k = pos.shape
    Y, sc = np.zeros((T, Ys.shape[1])), np.zeros((T, Ys.shape[1]))
    for t in range(T):
        for j in range(k):
            if 0 <= pos[t, j] < Ys.shape[0]:
                term = (1.0 if weight is None else weight[t, j]) * Ys[pos[t, j]]
                Y[t] += term
                sc[t] += np.abs(term)
    return Y, sc


def expert_combine_backward(dY, Ys, pos, weight=None):
    """dYs (zeros in rows that no slot names), (dweight, scale)."""
    T, k = pos.shape
    dYs, dw, sc = np.zeros(Ys.shape), np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            p = pos[t, j]
            if 0 <= p < Ys.shape[0]:
                dYs[p] = (1.0 if weight is None else weight[t, j]) * dY[t]
                dw[t, j], sc[t, j] = (dY[t] * Ys[p]).sum(), np.abs(dY[t] * Ys[p]).sum()
    return dYs, (dw, sc)


def clip(grads, max_norm):
    """norm, the scaled gradients."""
    norm = math.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads))
    by = max_norm / norm if math.isfinite(norm) and norm > max_norm else 1.0
    return norm, [np.asarray(g, dtype=np.float64) * by for g in grads]
