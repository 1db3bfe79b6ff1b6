"""Operator cases: a training step without a capacity, from token ids to the loss.

  embed  the lookup of token ids in a scaled table ("serve"), and its gradient at the
         table ("step")
  rows   tokens sorted by expert and back, weighted ("serve": dispatch and combine;
         "step": with the gradients of both)
  ffn    the experts' products over sorted rows ("serve": forward; "step": with the
         gradients at the rows and the weights)
  xent   softmax cross entropy over a vocabulary from the last activations and the
         output matrix ("serve": the loss of each token; "step": with the gradients)

A case is a dict of plain values.  ``own`` False computes the operators in their
plain form from elementary torch operations; True calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

#: Weight scale of every matrix (the GPT-2 initialisation).
W_STD = 0.02
#: Token ids follow a power law, rank r with weight 1 / (r + ZIPF).
ZIPF = 2.7


# ------------------------------------------------------------------------ cases
def _embed(name, T, V, d, **kw):
    c = dict(name=name, kind="embed", T=T, V=V, d=d, dtype="bf16", scale=1.0, padded=False, mode="step")
    c.update(kw)
    return c


def _rows(name, T, d, E, k, **kw):
    c = dict(name=name, kind="rows", T=T, d=d, E=E, k=k, dtype="bf16", padded=False, mode="step")
    c.update(kw)
    return c


def _ffn(name, T, d, f, E, k, **kw):
    c = dict(name=name, kind="ffn", T=T, d=d, f=f, E=E, k=k, dtype="bf16", act="gelu_tanh", mode="step")
    c.update(kw)
    return c


def _xent(name, T, V, d, **kw):
    c = dict(name=name, kind="xent", T=T, V=V, d=d, dtype="bf16", padded=False, mode="step")
    c.update(kw)
    return c


def listed():
    return [
        # One token of a decode step: a row of the table, launch latency only.
        _embed("embed_T1_d1024", 1, 50257, 1024, mode="serve"),
        # A small float32 training step over a small vocabulary, scaled by sqrt(d), the batch padded to its end.
        _embed("embed_step_f32_T1111_d640", 1111, 10007, 640, dtype="f32", scale=25.298221, padded=True),
        # One GPU's batch of a training step: the whole table's gradient is written, a few ids hold most tokens.
        _embed("embed_step_T16384_d2048", 16384, 50257, 2048),
        # A decode batch of a few dozen tokens, to its experts and back.
        _rows("rows_T48_d1024_E16", 48, 1024, 16, 2, mode="serve"),
        # Many narrow experts and choices in float32, a padded batch.
        _rows("rows_step_f32_T2000_d512_E160", 2000, 512, 160, 6, dtype="f32", padded=True),
        # One GPU's share of a training step.
        _rows("rows_step_T16384_d2048_E8", 16384, 2048, 8, 2),
        # A decode batch through every expert's weights.
        _ffn("ffn_T48_d1024_E16", 48, 1024, 4096, 16, 2, mode="serve"),
        # One GPU's share of a training step, no token dropped.
        _ffn("ffn_step_T16384_d2048_E8", 16384, 2048, 8192, 8, 2),
        # The loss of one token (scoring a continuation): the output matrix is read once.
        _xent("xent_T1_d1024", 1, 50257, 1024, mode="serve"),
        # A small float32 model's loss and gradients, odd sizes.
        _xent("xent_step_f32_T500_d512", 500, 10007, 512, dtype="f32"),
        # A short batch, padded, over a large vocabulary.
        _xent("xent_step_T2048_d1024", 2048, 50257, 1024, padded=True),
        # One GPU's batch of a training step.
        _xent("xent_step_T16384_d2048", 16384, 50257, 2048),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "rows", "ffn", "xent"])
    while True:
        f32 = rng.random() < 0.3
        dtype, mode, padded = "f32" if f32 else "bf16", rng.choice(["serve", "step", "step"]), rng.random() < 0.4
        if kind == "embed":
            c = _embed("", _log_int(rng, 1, 65536), _log_int(rng, 100, 150000), 8 * _log_int(rng, 8, 320), dtype=dtype,
                       scale=rng.choice([1.0, 1.0, 11.5]), padded=padded, mode=mode)
            fits = (c["T"] + c["V"]) * c["d"] <= 80000 * 2048
        elif kind == "rows":
            E = rng.choice([4, 8, 8, 16, 24, 64, 160, 256, 500])
            c = _rows("", _log_int(rng, 1, 32768), 64 * _log_int(rng, 1, 40), E,
                      min(E, rng.choice([1, 2, 2, 3, 4, 6, 8, 16])), dtype=dtype, padded=padded, mode=mode)
            fits = c["T"] * c["k"] * c["d"] <= 32768 * 2 * 2048
        elif kind == "ffn":
            E = rng.choice([2, 4, 8, 8, 16, 24, 64, 96])
            c = _ffn("", _log_int(rng, 1, 2048 if f32 else 16384), 64 * _log_int(rng, 2, 10 if f32 else 32),
                     64 * _log_int(rng, 2, 32 if f32 else 128), E, min(E, rng.choice([1, 2, 2, 3, 4, 6])), dtype=dtype,
                     act=rng.choice(["gelu_tanh", "gelu_tanh", "gelu_erf", "relu"]), mode=mode)
            fits = (E * c["d"] * c["f"] <= 1 << 27 and
                    c["T"] * c["k"] * c["d"] * c["f"] <= (2e10 if f32 else 16384 * 2 * 2048 * 8192))
        else:
            c = _xent("", _log_int(rng, 1, 2048 if f32 else 16384), _log_int(rng, 100, 20000 if f32 else 131072),
                      64 * _log_int(rng, 1, 10 if f32 else 32), dtype=dtype, padded=padded, mode=mode)
            fits = c["T"] * c["V"] * c["d"] <= (2e10 if f32 else 16384 * 50257 * 2048) and c["T"] * c["V"] <= 16384 * 50257
        if fits:
            del c["name"]
            return c


# ----------------------------------------------------------------------- shapes
def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _live(c):
    """Tokens of a batch that are no padding."""
    return c["T"] - c["T"] // 8 if c["padded"] else c["T"]


def _zipf(V):
    p = 1 / (np.arange(V) + ZIPF)
    return p / p.sum()


def _begins(c, n):
    """First rows of the experts' runs of n[e] rows (bf16: whole blocks of sixteen), and the rows of the buffers."""
    al = 16 if c["dtype"] == "bf16" else 1
    begin = np.concatenate(([0], np.cumsum(-(-n // al) * al)))[:-1]
    most = c["T"] * c["k"] + (al - 1) * min(c["E"], c["T"] * c["k"])
    return begin, -(-most // al) * al


def _counts(c, seed):
    """Rows of each expert: uneven, one expert without a row, one with a single one (as far as there are rows)."""
    g, E = np.random.default_rng(seed), c["E"]
    p = g.uniform(0.5, 1.5, E)
    if E > 2:
        p[1], p[0] = 0.0, 0.0
    n = np.minimum(g.multinomial(c["T"] * c["k"], p / p.sum()), c["T"])
    if E > 2 and n.sum() < c["T"] * c["k"]:
        n[0] = 1
    return n


def work(case):
    c = case
    b, d, step = (2 if c["dtype"] == "bf16" else 4), c["d"], c["mode"] == "step"
    if c["kind"] == "embed":
        n = _live(c)
        rows = float((1 - (1 - _zipf(c["V"])) ** n).sum())   # different ids, on average
        return {"bytes": int(rows * d * b + c["T"] * (d * b + 4) + ((n + c["V"]) * d * b if step else 0)),
                "flops": c["T"] * d * (2 if step else 1)}
    if c["kind"] == "rows":
        n, T = _live(c) * c["k"], c["T"]
        out = (2 * n + 2 * T) * d * b + 4 * (3 * T * c["k"] + 2 * n)
        return {"bytes": out + ((3 * n + 2 * T) * d * b + 8 * T * c["k"] if step else 0), "flops": n * d * (6 if step else 2)}
    if c["kind"] == "ffn":
        n, w = c["T"] * c["k"], 2 * c["E"] * d * c["f"]
        return {"bytes": (w + 2 * n * d) * b * (2 if step else 1), "flops": (12 if step else 4) * n * d * c["f"]}
    T, V = c["T"], c["V"]
    return {"bytes": (T + V) * d * b * (2 if step else 1) + T * (16 if step else 12), "flops": (8 if step else 2) * T * V * d}


# ----------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _ids(c, g):
    """Token ids; a padded batch ends in -1."""
    edges = torch.from_numpy(np.cumsum(_zipf(c["V"]))).cuda()
    u = torch.rand(c["T"], generator=g, device="cuda", dtype=torch.float64)
    ids = torch.searchsorted(edges, u).clamp(max=c["V"] - 1).to(torch.int32)
    ids[_live(c):] = -1
    return ids


def _blocked(m):
    """[.., R, X] as a product reads it in bfloat16: blocks of 16 rows by 32 columns, one after the other."""
    *lead, R, X = m.shape
    return m.view(*lead, R // 16, 16, X // 32, 32).transpose(-3, -2).reshape(*lead, R, X)


def _unblocked(m):
    *lead, R, X = m.shape
    return m.view(*lead, R // 16, X // 32, 16, 32).transpose(-3, -2).reshape(*lead, R, X)


def _embed_inputs(c, seed):
    g, dt = _gen(seed), _dt(c)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    t = {"ids": _ids(c, g), "W": (rn(c["V"], c["d"]) * W_STD).to(dt)}
    if c["mode"] == "step":
        t["dy"] = (rn(c["T"], c["d"]) * 1e-3).to(dt)
    return t


def _rows_inputs(c, seed):
    g, dt, T, d, E, k = _gen(seed), _dt(c), c["T"], c["d"], c["E"], c["k"]
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    t = {"x": rn(T, d).to(dt)}
    score, idx = torch.sort(rn(T, E) + 0.5 * rn(E), dim=1, descending=True)   # some experts are chosen more often
    t["idx"], t["w"] = idx[:, :k].to(torch.int32).contiguous(), torch.softmax(score[:, :k], dim=1).contiguous()
    t["idx"][_live(c):] = -1
    t["w"][_live(c):] = 0
    R = _begins(c, np.zeros(E, np.int64))[1]
    t["O"] = (rn(R, d) * 0.4).to(dt)
    if c["mode"] == "step":
        t["dy"], t["dXe"] = rn(T, d).to(dt), rn(R, d).to(dt)
    return t


def _ffn_inputs(c, seed):
    g, dt, d, f, E = _gen(seed), _dt(c), c["d"], c["f"], c["E"]
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    n = _counts(c, seed)
    begin, R = _begins(c, n)
    t = {"most": int(n.max()), "begin": torch.from_numpy(begin.astype(np.int32)).cuda(),
         "end": torch.from_numpy((begin + n).astype(np.int32)).cuda()}
    t["rows"] = rn(R, d).to(dt)
    t["W1"], t["W2"] = (rn(E, f, d) * W_STD).to(dt), (rn(E, d, f) * W_STD).to(dt)
    if c["mode"] == "step":
        t["dO"] = rn(R, d).to(dt)
    return t


def _xent_inputs(c, seed):
    g, dt = _gen(seed), _dt(c)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    t = {"target": _ids(c, g), "x": rn(c["T"], c["d"]).to(dt), "W": (rn(c["V"], c["d"]) * W_STD).to(dt)}
    if c["mode"] == "step":   # the mean over the tokens that count
        t["dloss"] = torch.full((c["T"],), 1 / _live(c), device="cuda")
    return t


def _inputs(c, seed):
    return {"embed": _embed_inputs, "rows": _rows_inputs, "ffn": _ffn_inputs, "xent": _xent_inputs}[c["kind"]](c, seed)


def prepare(case, seed):
    c, dt = case, _dt(case)
    t = _inputs(c, seed)
    new = lambda *s, dtype=dt: torch.zeros(*s, dtype=dtype, device="cuda")   # noqa: E731
    T, d, step, f32, i32 = c["T"], c["d"], c["mode"] == "step", torch.float32, torch.int32
    out = {}
    if c["kind"] == "embed":
        out["y"] = new(T, d)
        if step:
            out["dW"] = new(c["V"], d)
    elif c["kind"] == "rows":   # rows that hold no choice stay as they are
        R = t["O"].shape[0]
        out = {"row_begin": new(c["E"], dtype=i32), "row_end": new(c["E"], dtype=i32), "slot": new(T, c["k"], dtype=i32),
               "src": new(R, dtype=i32), "rows": new(R, d), "y": new(T, d)}
        if step:
            out |= {"dO": new(R, d), "dw": new(T, c["k"], dtype=f32), "dx": new(T, d)}
    elif c["kind"] == "ffn":
        R = t["rows"].shape[0]
        out = {"expert_out": new(R, d)}
        t["H"], t["A"] = new(R, c["f"]), new(R, c["f"])
        if step:
            out |= {"dXe": new(R, d), "dW1": new(c["E"], c["f"], d), "dW2": new(c["E"], d, c["f"])}
            t["dH"] = new(R, c["f"])
        if c["dtype"] == "bf16":   # the layout that a program keeps for the products
            t["W1p"], t["W2p"] = _blocked(t["W1"]), _blocked(t["W2"])
            t["rows"] = _blocked(t["rows"])
            if step:
                t["dO"] = _blocked(t["dO"])
        else:
            t["W1p"], t["W2p"] = t["W1"], t["W2"]
    else:
        out = {"loss": new(T, dtype=f32), "lse": new(T, dtype=f32)}
        if step:
            out |= {"dx": new(T, d), "dW": new(c["V"], d)}
    return {"case": c, "t": t, "out": out}


# ------------------------------------------------------------------------- runs
def run(state):
    return {"embed": _run_embed, "rows": _run_rows, "ffn": _run_ffn, "xent": _run_xent}[state["case"]["kind"]](state)


def _lib():
    from paper_2404_19429_amd import lancet_moe
    return lancet_moe


def _room(n):
    return torch.empty(max(16, n), dtype=torch.uint8, device="cuda")


def _run_embed(s):
    c, t, out = s["case"], s["t"], s["out"]
    if own:
        L = _lib()
        if "cfg" not in s:
            s["cfg"] = L.make_embed_cfg(c["T"], c["V"], c["d"], c["dtype"], c["scale"])
            s["ws"] = _room(L.moe_embed_bwd_workspace_bytes(s["cfg"]))
        L.moe_embed(s["cfg"], t["ids"], t["W"], out["y"])
        if c["mode"] == "step":
            L.moe_embed_bwd(s["cfg"], t["ids"], t["dy"], out["dW"], s["ws"])
        return out
    ok = (t["ids"] >= 0).unsqueeze(1)
    ids = t["ids"].clamp(min=0).long()
    res = {"y": torch.where(ok, c["scale"] * t["W"][ids].float(), 0.0).to(t["W"].dtype)}
    if c["mode"] == "step":
        dW = torch.zeros(c["V"], c["d"], device="cuda").index_add_(0, ids, torch.where(ok, t["dy"].float(), 0.0))
        res["dW"] = (c["scale"] * dW).to(t["W"].dtype)
    return res


def _run_rows(s):
    c, t, out = s["case"], s["t"], s["out"]
    if own:
        L = _lib()
        if "cfg" not in s:
            s["cfg"] = L.make_sorted_cfg(c["T"], c["d"], 64, c["E"], c["k"], c["dtype"])
            s["ws"] = _room(L.moe_sorted_workspace_bytes(s["cfg"], L.MOE_CALL_DISPATCH))
        L.moe_sorted_dispatch(s["cfg"], t["x"], t["idx"], out["row_begin"], out["row_end"], out["slot"], out["src"],
                              out["rows"], s["ws"])
        L.moe_sorted_combine(s["cfg"], t["O"], out["slot"], t["w"], out["y"])
        if c["mode"] == "step":
            L.moe_sorted_combine_bwd(s["cfg"], t["O"], out["slot"], out["src"], t["w"], t["dy"], out["dO"], out["dw"])
            L.moe_sorted_dispatch_bwd(s["cfg"], out["slot"], t["dXe"], out["dx"])
        return out
    return _plain_rows(c, t)


def _plain_rows(c, t):
    T, d, E, k = c["T"], c["d"], c["E"], c["k"]
    al, R, dt = 16 if c["dtype"] == "bf16" else 1, t["O"].shape[0], t["x"].dtype
    e = torch.where(t["idx"] >= 0, t["idx"], E).reshape(-1).long()
    key, order = torch.sort(e, stable=True)
    n = torch.zeros(E + 1, device="cuda", dtype=torch.int64).index_add_(0, e, torch.ones_like(e))
    room = (n + al - 1) // al * al
    begin = room.cumsum(0) - room
    row = begin[key] + torch.arange(T * k, device="cuda") - (n.cumsum(0) - n)[key]   # of the choices in their order
    slot = torch.full((T * k + 1,), -1, device="cuda", dtype=torch.int64)
    slot[order] = torch.where(key < E, row, -1)
    slot = slot[:T * k].view(T, k)
    held = slot >= 0
    at = torch.where(held, slot, R).view(-1)                        # row R: where dropped choices go
    src = torch.full((R + 1,), -1, device="cuda", dtype=torch.int64)
    src[at] = torch.arange(T * k, device="cuda")
    tok = torch.arange(T, device="cuda").repeat_interleave(k)
    lay = _blocked if c["dtype"] == "bf16" else (lambda m: m)
    rows = torch.zeros(R + 1, d, device="cuda").index_copy_(0, at, t["x"].float()[tok])[:R]
    o = t["O"].float()[slot.clamp(min=0)]                           # [T][k][d]
    w = torch.where(held, t["w"], 0.0).unsqueeze(2)
    res = {"row_begin": begin[:E].int(), "row_end": (begin + n)[:E].int(), "slot": slot.int(), "src": src[:R].int(),
           "rows": lay(rows).to(dt), "y": (w * o).sum(1).to(dt)}
    if c["mode"] == "step":
        dy = t["dy"].float().unsqueeze(1)
        dO = torch.zeros(R + 1, d, device="cuda").index_copy_(0, at, (w * dy).view(T * k, d))[:R]
        res["dO"] = lay(dO).to(dt)
        res["dw"] = torch.where(held, (o * dy).sum(2), 0.0)
        res["dx"] = torch.where(held.unsqueeze(2), t["dXe"].float()[slot.clamp(min=0)], 0.0).sum(1).to(dt)
    return res


def _run_ffn(s):
    c, t, out = s["case"], s["t"], s["out"]
    if own:
        L = _lib()
        if "cfg" not in s:
            s["cfg"] = L.make_sorted_cfg(c["T"], c["d"], c["f"], c["E"], c["k"], c["dtype"], c["act"])
            s["ws"] = _room(max(L.moe_sorted_workspace_bytes(s["cfg"], q)
                                for q in (L.MOE_CALL_FFN_FWD, L.MOE_CALL_BWD_DX, L.MOE_CALL_BWD_DW)))
        L.moe_sorted_ffn_fwd(s["cfg"], t["rows"], t["begin"], t["end"], t["W1p"], t["W2p"], t["H"], t["A"],
                             out["expert_out"], s["ws"])
        if c["mode"] == "step":
            L.moe_sorted_bwd_dx(s["cfg"], t["begin"], t["end"], t["H"], t["W1p"], t["W2p"], t["dO"], t["dH"],
                                out["dXe"], s["ws"])
            L.moe_sorted_bwd_dw(s["cfg"], t["begin"], t["end"], t["rows"], t["A"], t["dO"], t["dH"], out["dW1"],
                                out["dW2"], s["ws"])
        return out
    return _plain_ffn(c, t)


def _act(h, act):
    if act == "relu":
        return torch.where(h > 0, h, 0.0)
    if act == "gelu_erf":
        return 0.5 * h * (1 + torch.erf(h * math.sqrt(0.5)))
    return 0.5 * h * (1 + torch.tanh(math.sqrt(2 / math.pi) * (h + 0.044715 * h * h * h)))


def _dact(h, act):
    if act == "relu":
        return torch.where(h > 0, 1.0, 0.0)
    if act == "gelu_erf":
        return 0.5 * (1 + torch.erf(h * math.sqrt(0.5))) + h * torch.exp(-0.5 * h * h) / math.sqrt(2 * math.pi)
    a = math.sqrt(2 / math.pi)
    u = torch.tanh(a * (h + 0.044715 * h * h * h))
    return 0.5 * (1 + u) + 0.5 * h * (1 - u * u) * a * (1 + 3 * 0.044715 * h * h)


def _plain_ffn(c, t):
    """Every expert on its rows, padded to the longest run with zeros."""
    lay = _unblocked if c["dtype"] == "bf16" else (lambda m: m)
    rows, dt = lay(t["rows"]), t["rows"].dtype
    R, d = rows.shape
    i = t["begin"].long().unsqueeze(1) + torch.arange(t["most"], device="cuda")
    held = (i < t["end"].unsqueeze(1)).unsqueeze(2)
    at = torch.where(held.squeeze(2), i, R)
    take = lambda m: torch.where(held, m[at.clamp(max=R - 1)].float(), 0.0)   # noqa: E731
    back = lambda v: torch.zeros(R + 1, v.shape[2], device="cuda").index_copy_(0, at.view(-1), v.view(-1, v.shape[2]))[:R].to(dt)   # noqa: E731
    turn = lambda m: m.transpose(1, 2).contiguous()   # noqa: E731
    W1, W2, x = t["W1"].float(), t["W2"].float(), take(rows)
    h = torch.bmm(x, turn(W1))
    a = _act(h, c["act"])
    res = {"expert_out": back(torch.bmm(a, turn(W2)))}
    if c["mode"] == "step":
        dO = take(lay(t["dO"]))
        dh = torch.bmm(dO, W2) * _dact(h, c["act"])
        res["dXe"] = back(torch.bmm(dh, W1))
        res["dW1"], res["dW2"] = torch.bmm(turn(dh), x).to(dt), torch.bmm(turn(dO), a).to(dt)
    return res


def _run_xent(s):
    c, t, out = s["case"], s["t"], s["out"]
    if own:
        L = _lib()
        if "cfg" not in s:
            s["cfg"] = L.make_xent_cfg(c["T"], c["V"], c["d"], c["dtype"])
            s["ws"] = _room(max(L.moe_xent_workspace_bytes(s["cfg"], q) for q in range(1 + (c["mode"] == "step"))))
        L.moe_xent(s["cfg"], t["x"], t["W"], t["target"], out["loss"], out["lse"], s["ws"])
        if c["mode"] == "step":
            L.moe_xent_bwd(s["cfg"], t["x"], t["W"], t["target"], out["lse"], t["dloss"], out["dx"], out["dW"], s["ws"])
        return out
    x, W, dt = t["x"].float(), t["W"].float(), t["x"].dtype
    ok, at = t["target"] >= 0, t["target"].clamp(min=0).long().unsqueeze(1)
    l = x @ W.t().contiguous()
    m = l.amax(1, keepdim=True)
    lse = m + torch.log(torch.exp(l - m).sum(1, keepdim=True))
    res = {"loss": torch.where(ok, (lse - l.gather(1, at)).squeeze(1), 0.0), "lse": lse.squeeze(1)}
    if c["mode"] == "step":
        g = torch.where(ok, t["dloss"], 0.0).unsqueeze(1)
        p = torch.exp(l - lse) * g
        p.scatter_add_(1, at, -g)
        res["dx"], res["dW"] = (p @ W).to(dt), (p.t().contiguous() @ x).to(dt)
    return res


# ------------------------------------------------------------------------ exact
def exact(case, seed):
    return {"embed": _exact_embed, "rows": _exact_rows, "ffn": _exact_ffn, "xent": _exact_xent}[case["kind"]](case, _inputs(case, seed))


def _exact_embed(c, t):
    ids = t["ids"].cpu().numpy()
    live = np.flatnonzero(ids >= 0)
    there = torch.from_numpy(ids[live].astype(np.int64)).cuda()
    y = torch.zeros(c["T"], c["d"], dtype=torch.float64, device="cuda")
    y[torch.from_numpy(live).cuda()] = c["scale"] * t["W"].double()[there]
    out = {"y": y}
    if c["mode"] == "step":
        dW = torch.zeros(c["V"], c["d"], dtype=torch.float64, device="cuda")
        dW.index_put_((there,), c["scale"] * t["dy"].double()[torch.from_numpy(live).cuda()], accumulate=True)
        out["dW"] = dW
    return out


def _exact_rows(c, t):
    """The rows by a count on the host, expert by expert."""
    T, d, E, k = c["T"], c["d"], c["E"], c["k"]
    idx = t["idx"].cpu().numpy().reshape(-1)
    n = np.bincount(idx[idx >= 0], minlength=E)
    begin, R = _begins(c, n)
    slot, src = np.full(T * k, -1, np.int64), np.full(R, -1, np.int64)
    for e in range(E):
        at = np.flatnonzero(idx == e)
        slot[at] = begin[e] + np.arange(at.size)
        src[begin[e]:begin[e] + at.size] = at
    held = torch.from_numpy(np.flatnonzero(src >= 0)).cuda()
    choice = torch.from_numpy(src).cuda()[held]
    tok, w = choice // k, t["w"].double().reshape(-1)[choice].unsqueeze(1)
    lay = _blocked if c["dtype"] == "bf16" else (lambda m: m)

    def in_rows(v):
        m = torch.zeros(R, d, dtype=torch.float64, device="cuda")
        m[held] = v
        return m

    def in_tokens(v):
        return torch.zeros(T, d, dtype=torch.float64, device="cuda").index_put_((tok,), v, accumulate=True)

    o = t["O"].double()[held]
    i32 = lambda v: torch.from_numpy(v.astype(np.int32))   # noqa: E731
    out = {"row_begin": i32(begin), "row_end": i32(begin + n), "slot": i32(slot.reshape(T, k)), "src": i32(src),
           "rows": lay(in_rows(t["x"].double()[tok])), "y": in_tokens(w * o)}
    if c["mode"] == "step":
        dy = t["dy"].double()[tok]
        dw = torch.zeros(T * k, dtype=torch.float64, device="cuda")
        dw[choice] = (dy * o).sum(1)
        out |= {"dO": lay(in_rows(w * dy)), "dw": dw.view(T, k), "dx": in_tokens(t["dXe"].double()[held])}
    return out


def _exact_ffn(c, t):
    """Expert by expert; the activation's gradient by differentiation in 64 bits."""
    begin, end, f64 = t["begin"].tolist(), t["end"].tolist(), torch.float64
    out = {"expert_out": torch.zeros_like(t["rows"], dtype=f64)}
    step = c["mode"] == "step"
    if step:
        out |= {"dXe": torch.zeros_like(t["rows"], dtype=f64), "dW1": torch.zeros_like(t["W1"], dtype=f64),
                "dW2": torch.zeros_like(t["W2"], dtype=f64)}
    fn = {"relu": torch.relu, "gelu_erf": torch.nn.functional.gelu,
          "gelu_tanh": lambda h: torch.nn.functional.gelu(h, approximate="tanh")}[c["act"]]
    for e in range(c["E"]):
        at = slice(begin[e], end[e])
        if begin[e] == end[e]:
            continue
        x, W1, W2 = t["rows"][at].double(), t["W1"][e].double(), t["W2"][e].double()
        h = (x @ W1.t()).requires_grad_(step)
        with torch.enable_grad():
            a = fn(h)
        out["expert_out"][at] = a.detach() @ W2.t()
        if step:
            dO = t["dO"][at].double()
            dh, = torch.autograd.grad(a, h, dO @ W2)
            out["dXe"][at], out["dW1"][e], out["dW2"][e] = dh @ W1, dh.t() @ x, dO.t() @ a.detach()
    return out


def _exact_xent(c, t):
    """A thousand tokens at a time."""
    T, f64, step = c["T"], torch.float64, c["mode"] == "step"
    W = t["W"].double()
    out = {"loss": torch.zeros(T, dtype=f64, device="cuda"), "lse": torch.zeros(T, dtype=f64, device="cuda")}
    if step:
        out |= {"dx": torch.zeros(T, c["d"], dtype=f64, device="cuda"), "dW": torch.zeros_like(W)}
    for a in range(0, T, 1024):
        x, tgt = t["x"][a:a + 1024].double(), t["target"][a:a + 1024].long()
        l = x @ W.t()
        lse = torch.logsumexp(l, 1)
        rows = torch.nonzero(tgt >= 0).squeeze(1)
        out["lse"][a:a + 1024] = lse
        out["loss"][a + rows] = lse[rows] - l[rows, tgt[rows]]
        if step:
            dl = torch.softmax(l, 1)
            dl[rows, tgt[rows]] -= 1
            dl = dl * torch.where(tgt >= 0, t["dloss"][a:a + 1024].double(), 0.0).unsqueeze(1)
            out["dx"][a:a + 1024] = dl @ W
            out["dW"] += dl.t() @ x
    return out
