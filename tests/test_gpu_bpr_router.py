"""Batch-prioritized dispatch of choices that a router made: the order is by the router's own
scores, and experts that its contract masks change no token's importance."""
import numpy as np
import pytest
import torch

from oracle import moe_oracle as MO
from oracle import operators_oracle as O
from tests.test_gpu_router_layer import build

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")


def importance(logits, idx, score):
    """The sum of a token's chosen scores in rank order, rounded once to float."""
    s, _ = O.route_scores(logits, score)
    ok = idx >= 0
    imp = np.zeros(s.shape[0])
    for r in range(idx.shape[1]):
        imp = imp + np.where(ok[:, r], s[np.arange(len(s)), np.maximum(idx[:, r], 0)], 0.0)
    return imp.astype(np.float32)


def assign(idx, E, C, imp):
    """slot, fill, order; a choice of -1 takes no row."""
    slot, fill, order = MO.assign_slots_bpr(np.where(idx < 0, E, idx), E + 1, C, imp)
    return np.where(idx < 0, -1, slot), fill[:E], order


def dispatch(logits, idx, C, route, d=64):
    T, E = logits.shape
    k = idx.shape[1]
    cfg = L.make_cfg(T, d, d, E, k, C)
    i32 = dict(dtype=torch.int32, device="cuda")
    x = torch.randn(T, d, generator=torch.Generator("cuda").manual_seed(T), device="cuda").bfloat16()
    fill, slot, order = torch.full((E,), -7, **i32), torch.full((T, k), -7, **i32), torch.full((T,), -7, **i32)
    send = torch.full((L.expert_numel(cfg, d),), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((L.moe_workspace_bytes(cfg, L.MOE_CALL_DISPATCH_BPR),), 255, dtype=torch.uint8, device="cuda")
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()   # noqa: E731
    L.moe_dispatch_bpr_route(cfg, L.make_route_cfg(T, E, k, **route), x, t(logits), t(idx.astype(np.int32)), fill, slot,
                             send, order, ws)
    torch.cuda.synchronize()
    return fill.cpu().numpy(), slot.cpu().numpy(), order.cpu().numpy()


def logits_of(T, E, kind, seed):
    rng = np.random.default_rng(seed)
    l = (1.5 * rng.standard_normal((T, E))).astype(np.float32)
    if kind == "masked":
        l[rng.random((T, E)) < 0.3] = -np.inf
        l[rng.random((T, E)) < 0.1] = np.nan
        l[::7] = np.nan                                        # padding: no choice at all
        l[1::11] = -np.inf
    elif kind == "high":                                       # sigmoids next to 1: sums next to k
        l = np.abs(l) + 3
    elif kind == "inf":
        l[rng.random((T, E)) < 0.1] = np.inf
    elif kind == "low":
        l[::3] = np.finfo(np.float32).min
    return l


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("kind", ["normal", "masked", "high", "inf", "low"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (90, 8, 3), (700, 64, 8), (3000, 16, 2), (9001, 32, 4)])
def test_order_is_by_the_routers_scores(T, E, k, kind, score):
    l = logits_of(T, E, kind, T + E)
    bias = (0.2 * np.random.default_rng(E).standard_normal(E)).astype(np.float32)
    idx = O.route(l, bias, k, score)[0]
    C = max(1, T * k // (2 * E))                               # half of the choices at most are kept
    fill, slot, order = dispatch(l, idx, C, dict(score=score))
    rs, rf, ro = assign(idx, E, C, importance(l, idx, score))
    assert np.array_equal(order, ro) and np.array_equal(slot, rs) and np.array_equal(fill, rf)


def test_equal_scores_keep_the_tokens_order():
    T, E, k = 5000, 8, 2
    rng = np.random.default_rng(3)
    base = rng.standard_normal(E).astype(np.float32)
    l = np.stack([rng.permutation(base) for _ in range(T)])
    for score in ("softmax", "sigmoid"):
        idx = O.route(l, None, k, score)[0]
        assert np.array_equal(dispatch(l, idx, T, dict(score=score))[2], np.arange(T))


@pytest.mark.parametrize("route", [dict(score="sigmoid", scale=2.5), dict(score="softmax", renorm=0), dict(score="softmax")])
def test_layer_drops_what_the_router_scores_least(route):
    cfg, b, t, r = build("bf16", 400, 128, 128, 8, 2, 31, cf=(1, 2), **route)
    r.bias.mul_(5)
    L.layer_forward(b, t["x"], t["Wg"], None, t["W1"], t["W2"], routing="bpr", router=r)
    torch.cuda.synchronize()
    logits, idx = b.logits.cpu().numpy(), b.idx.cpu().numpy()
    slot, fill, order = assign(idx, cfg.E, cfg.C, importance(logits, idx, route["score"]))
    assert (slot < 0).any()
    assert np.array_equal(b.slot.cpu().numpy(), slot) and np.array_equal(b.fill.cpu().numpy(), fill)
    assert np.array_equal(b.order.cpu().numpy(), order)


@pytest.mark.parametrize("T", [500, 9000])
@pytest.mark.parametrize("what", ["nan", "twice"])
def test_gate_rows_that_no_gate_makes(what, T):
    """moe_dispatch_bpr, in one sorted tile and in several: NaN logits have no share of their token's softmax, and
    an expert named twice counts twice (importances of up to k)."""
    E, k, d = 8, 4, 64
    l = np.random.default_rng(T).standard_normal((T, E)).astype(np.float32)
    idx = O.route(l, None, k)[0]
    if what == "nan":
        l[5::50, 3] = np.nan
        l[7::50] = np.nan
    else:
        l[::9] *= 40
        idx[::3] = idx[::3, :1]
    C = T // 2
    cfg = L.make_cfg(T, d, d, E, k, C)
    i32 = dict(dtype=torch.int32, device="cuda")
    fill, slot, order = torch.empty(E, **i32), torch.full((T, k), -7, **i32), torch.empty(T, **i32)
    send = torch.empty(L.expert_numel(cfg, d), dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(L.moe_workspace_bytes(cfg, L.MOE_CALL_DISPATCH_BPR), dtype=torch.uint8, device="cuda")
    L.moe_dispatch_bpr(cfg, torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"), torch.from_numpy(l).cuda(),
                       torch.from_numpy(idx).cuda(), fill, slot, send, order, ws)
    torch.cuda.synchronize()
    rs, rf, ro = assign(idx, E, C, importance(l, idx, "softmax"))
    assert np.array_equal(order.cpu().numpy(), ro) and np.array_equal(slot.cpu().numpy(), rs)
    assert np.array_equal(fill.cpu().numpy(), rf)


def test_layer_step_in_a_graph():
    """Gate, router and batch-prioritized dispatch captured and replayed on new inputs."""
    cfg, b, t, r = build("bf16", 300, 128, 128, 8, 2, 41, cf=(1, 2), score="sigmoid")

    def step():
        r.load.zero_()
        L.layer_forward(b, t["x"], t["Wg"], None, t["W1"], t["W2"], routing="bpr", router=r)
    step()                                                     # loads the kernels
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    names = ("idx", "w", "slot", "fill", "order", "y")
    for i in range(4):
        t["x"].copy_(torch.randn(300, 128, generator=torch.Generator().manual_seed(i)).bfloat16())
        b.ws_bpr.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        got = {n: getattr(b, n).clone() for n in names}
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], getattr(b, n)) for n in names), i
