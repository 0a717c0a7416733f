"""Definitions, in float64 and without the library's code, of the operators for many routed experts
in 8 bits: the router with groups, numbers in 8 bits, their products, AdamW. Test infrastructure only."""
from __future__ import annotations

import numpy as np

BLOCK = 128


# ---- router -------------------------------------------------------------------------------------

def _scores(l, score):
    """Scores of one token's logits (float64), 0 where an expert is not available."""
    there = l > -np.inf  # false for NaN too
    s = np.zeros_like(l)
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            s[there] = 1 / (1 + np.exp(-l[there]))
    elif there.any():
        top = l[there].max()
        with np.errstate(invalid="ignore"):
            e = np.where(l[there] == top, 1.0, np.exp(l[there] - top))
        s[there] = e / e.sum()
    return there, s


def route_groups(logits, k, *, bias=None, score="sigmoid", groups=1, group_k=1, group_top=1, normalise=True, scale=1.0):
    """(expert [T][k], weight [T][k]) of logits [T][E]."""
    T, E = logits.shape
    size = E // groups
    b = np.zeros(E) if bias is None else np.asarray(bias, dtype=np.float64)
    expert, weight = np.full((T, k), -1, dtype=np.int32), np.zeros((T, k))
    for t in range(T):
        there, s = _scores(logits[t], score)
        with np.errstate(invalid="ignore"):
            c = (s + b).astype(np.float32)
        can = there & (c > -np.inf)
        if groups > 1:
            worth = {}
            for g in range(groups):
                best = sorted((c[e] for e in range(g * size, (g + 1) * size) if can[e]), reverse=True)[:group_top]
                if best:
                    worth[g] = best[0] if len(best) == 1 else np.float32(best[0] + best[1])
            taken = sorted(worth, key=lambda g: (-worth[g], g))[:group_k]
            can = can & np.isin(np.arange(E) // size, taken)
        chosen = sorted(np.flatnonzero(can), key=lambda e: (-c[e], e))[:k]
        share = weights_of(logits[t], s, chosen, score, normalise)
        expert[t, :len(chosen)] = chosen
        weight[t, :len(chosen)] = scale * share
    return expert, weight


def weights_of(l, s, chosen, score, normalise):
    """Weights before the scale. Quotients of sigmoids by their logarithms, which do not underflow."""
    if not normalise or not len(chosen):
        return s[chosen]
    x = l[chosen]
    if score == "sigmoid":
        x = -np.logaddexp(0, -x)
    top = x.max()
    with np.errstate(invalid="ignore"):
        e = np.where(x == top, 1.0, np.exp(x - top))
    return e / e.sum()


def route_groups_backward(logits, expert, dweight, *, score="sigmoid", normalise=True, scale=1.0):
    """dlogits [T][E] by the chain rule, one chosen expert's weight at a time."""
    T, E = logits.shape
    d = np.zeros((T, E))
    for t in range(T):
        there, s = _scores(logits[t], score)
        chosen = [e for e in expert[t] if 0 <= e < E]
        live = [e for e in chosen if there[e]]
        G = {e: scale * dweight[t, j] for j, e in enumerate(expert[t]) if e in live}
        if not live:
            continue
        if normalise:  # of the scores' logarithms
            share = dict(zip(live, weights_of(logits[t], s, live, score, True)))
            mean = sum(share[e] * G[e] for e in live)
            dlog = {e: share[e] * (G[e] - mean) for e in live}
        else:
            dlog = {e: s[e] * G[e] for e in live}
        for e in live:
            if score == "sigmoid":
                d[t, e] = dlog[e] * np.exp(-np.logaddexp(0, logits[t, e]))
            else:
                d[t, e] += dlog[e]
                d[t] -= dlog[e] * s
    return d


# ---- numbers in 8 bits -----------------------------------------------------------------------------

def e4m3_values():
    """The values of the codes 0 .. 126, ascending (127 is NaN)."""
    c = np.arange(127)
    exp, man = c >> 3, c & 7
    return np.where(exp == 0, man * 2.0 ** -9, (8 + man) * 2.0 ** (exp - 10.0))


def to_e4m3(x):
    """Codes of the nearest numbers, of equally near ones the one with an even code; NaN for what is not
    finite. |x| <= 448."""
    v = e4m3_values()
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.searchsorted(v, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    up, down = v[hi] - a, a - v[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isfinite(x), code, 127)
    return (code | (np.signbit(x) & np.isfinite(x)) << 7).astype(np.uint8)


def from_e4m3(code):
    v = np.append(e4m3_values(), np.nan)[code & 127]
    return np.where(code & 128, -v, v)


def scale_exponent(amax):
    """The smallest e from -127 on with amax <= 448 2^e, 0 for 0."""
    if amax == 0:
        return 0
    e = -127
    while amax > 448 * 2.0 ** e:
        e += 1
    return e


def quant(x):
    """Codes [..., n up to whole blocks] and exponents [..., blocks] along the last axis."""
    n = x.shape[-1]
    blocks = -(-n // BLOCK)
    wide = np.zeros(x.shape[:-1] + (blocks * BLOCK,))
    wide[..., :n] = x
    wide = wide.reshape(x.shape[:-1] + (blocks, BLOCK))
    amax = np.where(np.isfinite(wide), np.abs(wide), 0).max(-1)
    e = np.vectorize(scale_exponent, otypes=[np.int64])(amax) if amax.size else amax.astype(np.int64)
    return to_e4m3(wide / 2.0 ** e[..., None]).reshape(x.shape[:-1] + (blocks * BLOCK,)), e


def quant_columns(x, offsets):
    """Codes [d][columns] and exponents of x [T][d], each run from a whole block on."""
    codes, exps = [], []
    for a, b in zip(offsets[:-1], offsets[1:]):
        if b > a:
            q, e = quant(np.ascontiguousarray(x[a:b].T))
            codes.append(q)
            exps.append(e)
    if not codes:
        return np.zeros((x.shape[1], 0), np.uint8), np.zeros((x.shape[1], 0), np.int64)
    return np.concatenate(codes, 1), np.concatenate(exps, 1)


def quant_square(w):
    """Codes [R][C up to whole blocks] and exponents of one matrix, a scale for each 128 x 128."""
    R, C = w.shape
    r, c = -(-R // BLOCK), -(-C // BLOCK)
    wide = np.zeros((r * BLOCK, c * BLOCK))
    wide[:R, :C] = w
    e = np.array([[scale_exponent(_amax(wide[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK]))
                   for j in range(c)] for i in range(r)])
    by = np.repeat(np.repeat(2.0 ** e, BLOCK, 0), BLOCK, 1)
    return to_e4m3(wide / by)[:R], e


def _amax(x):
    return np.where(np.isfinite(x), np.abs(x), 0).max()


def held(codes, e, rows_per_scale=1):
    """The numbers that codes [rows][n] with exponents [rows / rows_per_scale][blocks] stand for."""
    by = np.repeat(np.repeat(2.0 ** e, BLOCK, 1), rows_per_scale, 0)
    return from_e4m3(codes) * by[:codes.shape[0], :codes.shape[1]]


# ---- AdamW ------------------------------------------------------------------------------------------

def adamw(p, g, m, v, t, *, lr, beta1, beta2, eps, weight_decay=0.0, c=1.0):
    """(new p, m, v)"""
    g = c * g
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    step = m / (1 - beta1 ** t) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return p - lr * (step + weight_decay * p), m, v


def mix(h):
    """MurmurHash3's finaliser on 32-bit numbers held in 64 bits."""
    h = np.asarray(h, dtype=np.uint64) & np.uint64(0xffffffff)
    for shift, by in ((16, 0x85ebca6b), (13, 0xc2b2ae35), (16, 1)):
        h = ((h ^ (h >> np.uint64(shift))) * np.uint64(by)) & np.uint64(0xffffffff)
    return h


def noise(places, t, seed):
    """(for m, for v): 16 random bits each for the elements at these places of the list."""
    places = np.asarray(places, dtype=np.uint64)
    key = mix(t + int(mix(seed)))
    h = mix(mix(key + (places >> np.uint64(32))) ^ (places & np.uint64(0xffffffff)))
    return (h & np.uint64(0xffff)).astype(np.int64), (h >> np.uint64(16)).astype(np.int64)


def drawn(x, bits, e, least):
    """(value, distance): the e4m3 number times 2^e that 16 bits of noise round x to, and how far, in
    steps between neighbours, the sum that was cut off lies from the next whole step."""
    a = np.abs(x) / 2.0 ** e
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -30))), -6) - 3)
    s = a / step + bits / 65536
    q = np.floor(s)
    if least:
        q = np.where((a > 0) & (a < 2.0 ** -6), np.maximum(q, 1), q)
    return np.sign(x) * q * step * 2.0 ** e, np.abs(s - np.round(s))
