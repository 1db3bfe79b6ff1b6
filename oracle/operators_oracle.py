"""Plain float64 statements of the router, the experts on 4-bit weights and the 8-bit
activation checkpoint, from their definitions (include/lancet_moe.h), with bounds on
what a float32 evaluation may be off by."""
from __future__ import annotations

import math

import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)
U32 = 2.0 ** -24     # half a step of float32, relative


# ------------------------------------------------------------------------ router
def route_scores(logits, score):
    """Scores of every expert; masked ones (-inf or NaN logits) 0.  And which are live."""
    l = np.asarray(logits, np.float64)
    live = l > -np.inf
    z = np.where(live, l, -np.inf)
    s = np.zeros_like(z)
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return np.where(live, 1 / (1 + np.exp(-z)), 0.0), live
    for t in range(z.shape[0]):
        if live[t].any():
            m = z[t].max()
            with np.errstate(invalid="ignore"):
                e = np.where(z[t] == m, 1.0, np.exp(z[t] - m))
            s[t] = np.where(live[t], e, 0.0) / e[live[t]].sum()
    return s, live


def route(logits, bias, k, score="softmax", renorm=1, groups=1, top_groups=1, scale=1.0):
    """idx, w, load, one choice after the other."""
    l = np.asarray(logits, np.float64)
    T, E = l.shape
    s, live = route_scores(l, score)
    if bias is None and groups == 1:
        c = np.where(live, l, -np.inf)
    else:
        c = s + (0.0 if bias is None else np.asarray(bias, np.float64))
        c = np.where(live & (c > -np.inf), c, -np.inf)
    n = E // groups
    idx, w, load = np.full((T, k), -1, np.int32), np.zeros((T, k)), np.zeros(E, np.int64)
    for t in range(T):
        ct = c[t].copy()
        if groups > 1:
            val = []
            for g in range(groups):
                top = sorted((v for v in ct[g * n:(g + 1) * n] if v > -np.inf), reverse=True)[:2]
                val.append(sum(top) if top else -np.inf)
            kept = sorted(range(groups), key=lambda g: (-val[g], g))[:top_groups]
            for g in range(groups):
                if g not in kept:
                    ct[g * n:(g + 1) * n] = -np.inf
        chosen = [e for e in sorted(range(E), key=lambda e: (-ct[e], e))[:k] if ct[e] > -np.inf]
        tot = sum(s[t, e] for e in chosen)
        for r, e in enumerate(chosen):
            idx[t, r] = e
            w[t, r] = scale * s[t, e] if not renorm else scale * s[t, e] / tot if tot > 0 else 0.0
            load[e] += 1
    return idx, w, load


def route_weights(logits, idx, score, renorm, scale):
    """The weights of given choices (idx -1: 0): what the gradient differentiates."""
    s, _ = route_scores(logits, score)
    ok = (idx >= 0) & (idx < s.shape[1])
    sel = np.where(ok, np.take_along_axis(s, np.where(ok, idx, 0), 1), 0.0)
    tot = sel.sum(1, keepdims=True)
    return scale * sel / np.where(tot > 0, tot, 1.0) if renorm else scale * sel


def route_bwd(logits, idx, dw, score, renorm, scale):
    """dL/dlogits by the chain rule through the scores, and the sum of its terms' magnitudes."""
    s, live = route_scores(logits, score)
    T, E = s.shape
    k = idx.shape[1]
    u, mag = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        rs = [r for r in range(k) if 0 <= idx[t, r] < E]
        tot = sum(s[t, idx[t, r]] for r in rs)
        if renorm and not tot > 0:
            continue
        mean = sum(dw[t, r] * s[t, idx[t, r]] for r in rs) / tot if renorm else 0.0
        amean = sum(abs(dw[t, r]) * s[t, idx[t, r]] for r in rs) / tot if renorm else 0.0
        for r in rs:
            f = scale / tot if renorm else scale
            u[t, idx[t, r]] += f * (dw[t, r] - mean)
            mag[t, idx[t, r]] += f * (abs(dw[t, r]) + amean)
    if score == "sigmoid":
        # 1 - s of a large logit, without its cancellation
        with np.errstate(over="ignore"):
            less = np.where(live, 1 / (1 + np.exp(np.where(live, logits, 0.0).astype(np.float64))), 0.0)
        return u * s * less, mag * s * less
    return s * (u - (u * s).sum(1, keepdims=True)), s * (mag + (mag * s).sum(1, keepdims=True))


# ------------------------------------------------------------ 4-bit expert weights
def w4_decode(codes, scales):
    """codes [..., K/2], scales [..., K/32] (uint8) -> float64 [..., K]."""
    q = np.stack((codes & 15, codes >> 4), axis=-1).reshape(*codes.shape[:-1], -1)
    v = np.where(q & 8, -1.0, 1.0) * E2M1[q & 7]
    sc = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(sc, 32, axis=-1)


def w4_quantize(W):
    """float [..., K] -> codes, scales: the smallest power of two with max <= 7, the nearest code."""
    W = np.asarray(W, np.float64)
    g = W.reshape(*W.shape[:-1], -1, 32)
    codes = np.zeros(g.shape, np.uint8)
    scales = np.zeros(g.shape[:-1], np.uint8)
    for at in np.ndindex(g.shape[:-1]):
        amax = np.abs(g[at]).max()
        if not np.isfinite(amax):
            scales[at] = 255
            continue
        s = -100
        if amax > 0:
            s = max(-100, min(125, math.ceil(math.log2(amax / 7))))
            while s > -100 and amax <= 7 * 2.0 ** (s - 1):   # log2's own rounding
                s -= 1
            while s < 125 and amax > 7 * 2.0 ** s:
                s += 1
        a = np.abs(g[at]) / 2.0 ** s
        d = np.abs(a[:, None] - E2M1[None, :])
        near = d.min(1)
        for i in range(32):
            best = [c for c in range(8) if d[i, c] == near[i]]
            c = best[0] if len(best) == 1 else next(c for c in best if c % 2 == 0)
            codes[at][i] = c | (8 if math.copysign(1.0, g[at][i]) < 0 else 0)
        scales[at] = s + 127
    codes = codes.reshape(*W.shape)
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8), scales


def act(h, name):
    if name == "identity":
        return h
    if name == "relu":
        return np.maximum(h, 0.0)
    if name == "gelu_erf":
        return 0.5 * h * (1 + np.vectorize(math.erf)(h / math.sqrt(2)))
    return 0.5 * h * (1 + np.tanh(math.sqrt(2 / math.pi) * (h + 0.044715 * h ** 3)))


def experts(x, idx, w, W1, W2, act_name, part=2.0 ** -16):
    """y (W1 [E][f][d], W2 [E][d][f] decoded), and a bound on a float32 evaluation's error:
    sums of K terms are off by (K + 4) half steps of the sum of magnitudes (the order is
    free), the activation by 16 half steps of |h| and, with slope up to 1.13, by what h is;
    act(h) goes on as bfloat16 parts good to `part` (one part: 2^-8, half a step)."""
    T, d = x.shape
    E, f = W1.shape[:2]
    y, err = np.zeros((T, d)), np.zeros((T, d))
    for e in range(E):
        t, r = np.nonzero(idx == e)
        if t.size == 0:
            continue
        h = x[t] @ W1[e].T
        eh = (d + 4) * U32 * (np.abs(x[t]) @ np.abs(W1[e]).T)
        a = act(h, act_name)
        ea = 1.13 * eh + 16 * U32 * np.abs(h) + part * np.abs(a)
        abs2 = np.abs(W2[e]).T
        np.add.at(y, t, w[t, r][:, None] * (a @ W2[e].T))
        np.add.at(err, t, np.abs(w[t, r])[:, None] * (ea @ abs2 + (f + 8 + idx.shape[1]) * U32 * (np.abs(a) @ abs2)))
    return y, err


# -------------------------------------------------------------------- checkpoint
def ckpt_round_trip(x):
    """Rows of a buffer [R][X] (float32 values): the float32 products integer * step."""
    x = np.asarray(x, np.float32)
    out = np.zeros_like(x)
    for j in range(0, x.shape[1], 64):
        g = x[:, j:j + 64]
        amax = np.abs(g).max(1, keepdims=True)
        bad = ~np.isfinite(g).all(1, keepdims=True)
        tiny = ~bad & (amax < np.float32(1e-30))
        safe = np.where(bad | tiny, np.float32(1), amax)
        q = np.rint(np.where(bad, 0, g).astype(np.float64) * 127 / safe.astype(np.float64)).astype(np.float32)
        v = q * (safe / np.float32(127))
        out[:, j:j + 64] = np.where(bad, np.float32(np.nan), np.where(tiny, np.float32(0), v))
    return out
