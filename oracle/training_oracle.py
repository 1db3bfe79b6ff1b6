"""Plain 64-bit forms of the operators of a training step without a capacity: rows sorted
by expert and back, the experts over them, token lookup.  Test infrastructure only;
torch in float64 on whatever device its inputs are on, no code of the library.

Every float result comes with a bound on how far a kernel may be off: half a step of
each rounding to bfloat16 (2^-8 of the value) or float (2^-24), carried through the
products that read the rounded value, and n 2^-24 of the sum of magnitudes for a float
sum of n terms.
"""
from __future__ import annotations

import math

import numpy as np
import torch

U32, UBF = 2.0 ** -24, 2.0 ** -8
TINY = 2.0 ** -126   # float's smallest normal number: what is smaller may count as 0


def half_step(dtype):
    return UBF if dtype in ("bf16", torch.bfloat16) else U32


def blocked(m):
    """[.., R, X] -> the 16 x 32 blocks of the bf16 expert buffers, flat but for the leading dimensions."""
    *lead, R, X = m.shape
    return m.reshape(*lead, R // 16, 16, X // 32, 32).transpose(-3, -2).reshape(*lead, R, X)


def unblocked(m):
    *lead, R, X = m.shape
    return m.reshape(*lead, R // 16, X // 32, 16, 32).transpose(-3, -2).reshape(*lead, R, X)


def n_rows(T, E, k, dtype):
    n = T * k
    return n if dtype == "f32" else -(-(n + 15 * min(E, n)) // 16) * 16


def sort_rows(idx, E, dtype):
    """idx [T][k] (numpy) -> row_begin, row_end [E], slot [T][k], src [R], choice by choice."""
    T, k = idx.shape
    al = 16 if dtype == "bf16" else 1
    lists = [[] for _ in range(E)]
    for i, e in enumerate(idx.reshape(-1).tolist()):
        if 0 <= e < E:
            lists[e].append(i)
    begin, end, at = np.zeros(E, np.int32), np.zeros(E, np.int32), 0
    slot, src = np.full(T * k, -1, np.int32), np.full(n_rows(T, E, k, dtype), -1, np.int32)
    for e, li in enumerate(lists):
        begin[e], end[e] = at, at + len(li)
        for j, i in enumerate(li):
            slot[i], src[at + j] = at + j, i
        at += -(-len(li) // al) * al
    return begin, end, slot.reshape(T, k), src


def back(rows, slot, w=None, gate=None):
    """sum_r w rows[slot] by token and its bound; gate = (Wg, dlogits)."""
    T, k = slot.shape
    held = (slot >= 0).unsqueeze(2)
    v = torch.where(held, rows.double()[slot.clamp(min=0).long()], 0.0)
    if w is not None:
        v = v * torch.where(held, w.double().unsqueeze(2), 0.0)
    y, size, n = v.sum(1), v.abs().sum(1), k
    if gate is not None:
        Wg, dl = gate[0].double(), gate[1].double()
        y, size, n = y + dl @ Wg, size + dl.abs() @ Wg.abs(), k + dl.shape[1]
    return y, half_step(rows.dtype) * y.abs() + (n + 1) * U32 * size


def combine_bwd(O, slot, src, w, dy, k):
    """dO [R][d] (rows that hold none: 0) and dw [T][k], with bounds."""
    held = src >= 0
    i = src.clamp(min=0).long()
    g = torch.where(held.unsqueeze(1), dy.double()[i // k], 0.0)
    wr = torch.where(held, w.double().reshape(-1)[i], 0.0).unsqueeze(1)
    dO = wr * g
    at = slot >= 0
    o = torch.where(at.unsqueeze(2), O.double()[slot.clamp(min=0).long()], 0.0)
    p = torch.where(at.unsqueeze(2), dy.double().unsqueeze(1), 0.0) * o
    return dO, (half_step(O.dtype) + U32) * dO.abs(), p.sum(2), (O.shape[1] + 8) * U32 * p.abs().sum(2)


def act(h, name):
    if name == "relu":
        return torch.relu(h)
    if name == "identity":
        return h
    if name == "gelu_erf":
        return 0.5 * h * (1 + torch.erf(h * math.sqrt(0.5)))
    return 0.5 * h * (1 + torch.tanh(math.sqrt(2 / math.pi) * (h + 0.044715 * h ** 3)))


def dact(h, name):
    if name == "relu":
        return (h > 0).double()
    if name == "identity":
        return torch.ones_like(h)
    if name == "gelu_erf":
        return 0.5 * (1 + torch.erf(h * math.sqrt(0.5))) + h * torch.exp(-0.5 * h * h) / math.sqrt(2 * math.pi)
    a = math.sqrt(2 / math.pi)
    t = torch.tanh(a * (h + 0.044715 * h ** 3))
    return 0.5 * (1 + t) + 0.5 * h * (1 - t * t) * a * (1 + 3 * 0.044715 * h * h)


# |act'| <= 1.13 and |act''| <= 0.8 for the GELUs (the largest of both curves, at sqrt 2 and at 0; the tanh form within 1 %).
SLOPE, BEND = 1.15, 0.82
# The library's activations: a few float roundings of values of the size of h and 1.
ACT_ULPS = 16


def expert(x, W1, W2, name, dO=None):
    """One expert on its rows: {name: (value, bound)} of O and, with dO, of dX, dW1, dW2."""
    u = half_step(x.dtype)
    x, W1, W2 = x.double(), W1.double(), W2.double()
    n, d, f = x.shape[0], W1.shape[1], W1.shape[0]
    h = x @ W1.t()
    th = (d + 2) * U32 * (x.abs() @ W1.abs().t())            # the float sum
    a = act(h, name)
    ta = SLOPE * th + ACT_ULPS * U32 * (1 + h.abs())
    ta_kept = ta + u * (a.abs() + ta)                        # A is kept rounded
    O = a @ W2.t()
    tO = ta_kept @ W2.abs().t() + (f + 2) * U32 * ((a.abs() + ta_kept) @ W2.abs().t())
    out = {"O": (O, tO + u * (O.abs() + tO))}
    if dO is None:
        return out
    dO = dO.double()
    dA = dO @ W2
    tdA = (d + 2) * U32 * (dO.abs() @ W2.abs())
    th_kept = th + u * (h.abs() + th)                        # act' of H as it is kept
    s = dact(h, name)
    bend = BEND if name.startswith("gelu") else 0.0
    ts = bend * th_kept + ACT_ULPS * U32 * (1 + h.abs())
    if name == "relu":                                       # the step at 0: a sum that may have either sign
        ts = ts + (h.abs() <= th).double()
    dh = dA * s
    tdh = tdA * (s.abs() + ts) + dA.abs() * ts
    tdh = tdh + u * (dh.abs() + tdh)
    dX = dh @ W1
    tX = tdh @ W1.abs() + (f + 2) * U32 * ((dh.abs() + tdh) @ W1.abs())
    dW1 = dh.t() @ x
    t1 = tdh.t() @ x.abs() + (n + 2) * U32 * ((dh.abs() + tdh).t() @ x.abs())
    dW2 = dO.t() @ a
    t2 = dO.abs().t() @ ta_kept + (n + 2) * U32 * (dO.abs().t() @ (a.abs() + ta_kept))
    out["dX"] = (dX, tX + u * (dX.abs() + tX))
    out["dW1"] = (dW1, t1 + u * (dW1.abs() + t1))
    out["dW2"] = (dW2, t2 + u * (dW2.abs() + t2))
    return out


def embed(ids, W, scale):
    ok = (ids >= 0) & (ids < W.shape[0])
    y = torch.where(ok.unsqueeze(1), scale * W.double()[torch.where(ok, ids, 0).long()], 0.0)
    return y, (half_step(W.dtype) + U32) * y.abs()


def embed_bwd(ids, dy, V, scale, old=None):
    ok = (ids >= 0) & (ids < V)
    i, g = ids[ok].long(), dy[ok].double()
    put = lambda v: torch.zeros(V, dy.shape[1], dtype=torch.float64, device=dy.device).index_put_((i,), v, accumulate=True)
    dW, size = scale * put(g), abs(scale) * put(g.abs())
    n = torch.zeros(V, dtype=torch.float64, device=dy.device).index_put_((i,), torch.ones_like(i).double(), accumulate=True)
    if old is not None:
        dW, size = dW + old.double(), size + old.double().abs()
    t = half_step(dy.dtype) * dW.abs() + (n.unsqueeze(1) + 3) * U32 * size
    return dW, torch.where(n.unsqueeze(1) > 0, t, 0.0)   # (an id that does not occur: exactly 0, or what was there)


def xent(x, W, target, dloss=None):
    """{name: (value, bound)} of loss and lse and, with dloss, of dx and dW.

    Bounds: a logit is a float sum of d products.  The sum of V exponentials is positive
    terms added in at most 16 + V / 64 steps (sixteen of a lane, the runs' sums in turn),
    each with a rounding or, where the largest logit so far grew, three (the exponential
    of the difference, 2 of them, and its product).  An exponential of a difference D is
    off by 2 |D| + 3 roundings.  A probability, a dl or a product below float's normal
    numbers may be 0: off by as much as TINY each.
    """
    u, (T, d), V = half_step(x.dtype), x.shape, W.shape[0]
    ok = (target >= 0) & (target < V)
    at = torch.where(ok, target, 0).long().unsqueeze(1)
    x, W = x.double(), W.double()
    l = x @ W.t()
    tl = (d + 2) * U32 * (x.abs() @ W.abs().t())
    m = l.amax(1, keepdim=True)
    e = torch.exp(l - m)
    s = e.sum(1, keepdim=True)
    lse = m + torch.log(s)
    te = (e * (tl + (2 * (l - m).abs() + 3) * U32)).sum(1, keepdim=True) / s     # of the sum's terms, relative
    tz = te + 3 * (16 + V / 64) * U32 + 4 * U32 * (1 + lse.abs())
    lt = l.gather(1, at)
    out = {"lse": (lse.squeeze(1), tz.squeeze(1)),
           "loss": (torch.where(ok, (lse - lt).squeeze(1), 0.0),
                    torch.where(ok, (tz + tl.gather(1, at) + U32 * (lse - lt).abs()).squeeze(1), 0.0))}
    if dloss is None:
        return out
    g = torch.where(ok, dloss.double(), 0.0).unsqueeze(1)
    p = torch.exp(l - lse)
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    dl = g * (p - one)
    t = g.abs() * (p * (tl + tz + (2 * (l - lse).abs() + 4) * U32) + 2 * U32 * (p - one).abs())
    t = t + u * (dl.abs() + t) + (1 + g.abs().amax()) * TINY   # (bf16: dl is kept relative to the largest g)
    xz = torch.where(ok.unsqueeze(1), x, 0.0)
    for name, a, b, n in (("dx", (dl, t), W, V), ("dW", (dl.t(), t.t()), xz, T)):
        v = a[0] @ b
        tv = a[1] @ b.abs() + (n + 2) * U32 * ((a[0].abs() + a[1]) @ b.abs()) + n * TINY
        out[name] = (v, tv + u * (v.abs() + tv))
    return out


def off(got, want):
    """The largest difference over its bound (0 / 0 counts as 0); NaN counts as off."""
    v, t = want
    d = (got.double() - v).abs()
    if d.numel() == 0:
        return 0.0
    r = torch.where(d == 0, 0.0, d / t)
    return float(torch.where(r == r, r, math.inf).max())
