"""The router, the checkpoint and the layer's products as a training step uses them, the
router and the 4-bit experts as serving uses them, and both captured into a HIP graph."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as O
from tests.gpu_harness import TOL, assert_close, ebuf, nan_fill

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")


def dact(h, name):
    if name == "relu":
        return (h > 0).astype(np.float64)
    c = np.sqrt(2 / np.pi)
    th = np.tanh(c * (h + 0.044715 * h ** 3))
    return 0.5 * (1 + th) + 0.5 * h * (1 - th * th) * c * (1 + 3 * 0.044715 * h * h)


def build(dtype, T, d, f, E, k, seed, act="gelu_tanh", cf=(5, 4), **route):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(seed)
    rn = lambda *s, std=1.0: torch.from_numpy((std * rng.standard_normal(s)).astype(np.float32)).to(dt).cuda()   # noqa: E731
    C = L.moe_capacity(T, E, k, *cf)
    cfg = L.make_cfg(T, d, f, E, k, C, 1, dtype, act)
    b = L.alloc_layer(cfg)
    nan_fill(b)
    t = dict(x=rn(T, d), Wg=rn(E, d, std=0.1), W1=rn(E, f, d, std=0.05), W2=rn(E, d, f, std=0.05), dy=rn(T, d))
    r = L.Router(L.make_route_cfg(T, E, k, **route),
                 torch.from_numpy((0.1 * rng.standard_normal(E)).astype(np.float32)).cuda(),
                 torch.zeros(E, dtype=torch.int32, device="cuda"))
    return cfg, b, t, r


def reference(cfg, b, t, route):
    """The backward in float64 from the activations the layer holds now."""
    T, d, E, k = cfg.T, cfg.d_model, cfg.E, cfg.k
    h = {n: v.double().cpu().numpy() for n, v in t.items()}
    idx, slot, w = b.idx.cpu().numpy(), b.slot.cpu().numpy(), b.w.double().cpu().numpy()
    X, H, A, Oe = (ebuf(b, n).astype(np.float64) for n in ("send_buf", "H", "A", "O"))
    act = {v: n for n, v in L.ACTS.items()}[cfg.act]
    dw = np.zeros((T, k))
    dx = np.zeros((T, d))
    dW1, dW2 = np.zeros_like(h["W1"]), np.zeros_like(h["W2"])
    for t_ in range(T):
        for r in range(k):
            e, s = idx[t_, r], slot[t_, r]
            if s < 0:
                continue
            dw[t_, r] = h["dy"][t_] @ Oe[e, s]
            do = w[t_, r] * h["dy"][t_]
            dh = (do @ h["W2"][e]) * dact(H[e, s], act)
            dx[t_] += dh @ h["W1"][e]
            dW2[e] += np.outer(do, A[e, s])
            dW1[e] += np.outer(dh, X[e, s])
    dl = O.route_bwd(b.logits.double().cpu().numpy(), idx, dw, *route)[0]
    return dict(dw=dw, dlogits=dl, dx=dx + dl @ h["Wg"], dW1=dW1, dW2=dW2, dWg=dl.T @ h["x"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("route", [dict(score="sigmoid", groups=4, top_groups=2, scale=2.5), dict(score="softmax", renorm=0),
                                   dict(score="softmax"), dict(score="sigmoid", renorm=0)])
def test_training_step_with_router_and_checkpoint(route, dtype):
    cfg, b, t, r = build(dtype, 150, 128, 192, 8, 2, 11, cf=(1, 1), **route)
    L.layer_forward(b, t["x"], t["Wg"], None, t["W1"], t["W2"], router=r)
    idx, w, load = O.route(b.logits.cpu().numpy(), r.bias.cpu().numpy(), 2, **route)
    assert np.array_equal(b.idx.cpu().numpy(), idx) and np.array_equal(r.load.cpu().numpy(), load)
    slot = b.slot.cpu().numpy()
    assert (slot < 0).any()                                       # some choices past the capacity
    before = {n: ebuf(b, n).copy() for n in ("send_buf", "H", "A", "O")}
    ck = L.alloc_ckpt(cfg)
    L.layer_save(b, ck)
    for n in ("send_buf", "H", "A", "O"):                          # another layer used them meanwhile
        getattr(b, n).fill_(float("nan"))
    L.layer_restore(b, ck)
    fill = b.fill.cpu().numpy()
    for n in before:
        for e in range(cfg.E):
            v, g = before[n][e, :fill[e]], ebuf(b, n)[e, :fill[e]]
            if n != "A" and v.size:   # half a step of 1/127 of the group's largest, then the type's rounding
                top = np.abs(v).max(1, keepdims=True)
                assert (np.abs(g - v) <= top / 254 * (1 + 1e-6) + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * top).all(), n
    L.layer_backward(b, t["x"], t["Wg"], t["dy"], router=r)
    torch.cuda.synchronize()
    ref = reference(cfg, b, t, (route["score"], route.get("renorm", 1), route.get("scale", 1.0)))
    for n, v in ref.items():
        assert_close(n, getattr(b, n).double().cpu().numpy(), v, TOL[dtype])


@pytest.mark.parametrize("routing", ["token", "bpr"])
@pytest.mark.parametrize("route", [dict(score="sigmoid"), dict(score="softmax", renorm=0), dict(score="softmax")])
def test_choices_left_open_take_no_part(route, routing):
    """Two live experts (the others' bias is -inf) for three choices: the third is -1 throughout the layer."""
    cfg, b, t, r = build("bf16", 90, 128, 128, 8, 3, 17, cf=(3, 1), **route)
    r.bias.fill_(float("-inf"))
    r.bias[[2, 7]] = 0.0
    L.layer_forward(b, t["x"], t["Wg"], None, t["W1"], t["W2"], routing=routing, router=r)
    torch.cuda.synchronize()
    idx, slot = b.idx.cpu().numpy(), b.slot.cpu().numpy()
    assert (np.sort(idx, 1) == [-1, 2, 7]).all() and (idx[:, 2] == -1).all()
    assert (slot[:, 2] < 0).all() and (slot[:, :2] >= 0).all() and (b.w[:, 2] == 0).all()
    O_, w = ebuf(b, "O").astype(np.float64), b.w.double().cpu().numpy()
    y = sum(w[:, r_, None] * O_[idx[:, r_], slot[:, r_]] for r_ in (0, 1))
    assert_close("y", b.y.double().cpu().numpy(), y, TOL["bf16"])
    L.layer_backward(b, t["x"], t["Wg"], t["dy"], router=r)
    torch.cuda.synchronize()
    ref = reference(cfg, b, t, (route["score"], route.get("renorm", 1), 1.0))
    assert (b.dw[:, 2] == 0).all()
    for n, v in ref.items():
        assert_close(n, getattr(b, n).double().cpu().numpy(), v, TOL["bf16"])


def test_softmax_router_is_the_gate():
    """Without bias and groups the router is moe_gate_topk, and its backward moe_bwd_dx's."""
    for renorm in (0, 1):
        cfg, b, t, r = build("bf16", 200, 128, 128, 8, 2, 5, renorm=renorm)
        cfg.renorm = b.cfg.renorm = renorm
        r.bias = None
        L.layer_forward(b, t["x"], t["Wg"], None, t["W1"], t["W2"])
        L.layer_backward(b, t["x"], t["Wg"], t["dy"])
        want = {n: getattr(b, n).clone() for n in ("idx", "w", "slot", "y", "dx", "dlogits", "dW1", "dWg")}
        L.layer_forward(b, t["x"], t["Wg"], None, t["W1"], t["W2"], router=r)
        L.layer_backward(b, t["x"], t["Wg"], t["dy"], router=r)
        assert torch.equal(b.idx, want["idx"]) and torch.equal(b.slot, want["slot"])
        assert (b.w - want["w"]).abs().max() <= 64 * O.U32
        for n in ("y", "dx", "dlogits", "dW1", "dWg"):
            assert_close(n, getattr(b, n).double().cpu().numpy(), want[n].double().cpu().numpy(), TOL["bf16"])


def serve_state(T, d, f, E, k, seed):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).bfloat16().cuda()
    Wg = torch.from_numpy((0.1 * rng.standard_normal((E, d))).astype(np.float32)).bfloat16().cuda()
    W = [torch.from_numpy(0.05 * rng.standard_normal(s).astype(np.float32)).bfloat16().cuda() for s in ((E, f, d), (E, d, f))]
    q = [L.alloc_w4(E, f, d), L.alloc_w4(E, d, f)]
    for a, b in zip(W, q):
        L.moe_w4_quantize(a, *b)
    gate = L.make_cfg(T, d, 64, E, k, T, 1)
    rc = L.make_route_cfg(T, E, k, "sigmoid", groups=4, top_groups=2, scale=2.5)
    wc = L.make_w4_cfg(T, d, f, E, k)
    e = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device="cuda")   # noqa: E731
    s = dict(x=x, lg=e(T, E), idx=e(T, k, dt=torch.int32), w=e(T, k), y=torch.empty_like(x),
             bias=torch.from_numpy((0.1 * rng.standard_normal(E)).astype(np.float32)).cuda(),
             load=torch.zeros(E, dtype=torch.int32, device="cuda"),
             ws=e(L.moe_experts_w4_workspace_bytes(wc), dt=torch.uint8))

    def step():
        L.moe_gate_topk(gate, s["x"], Wg, None, s["lg"], s["idx"], s["w"])
        s["load"].zero_()
        L.moe_route(rc, s["lg"], s["bias"], s["idx"], s["w"], s["load"])
        L.moe_experts_w4(wc, s["x"], s["idx"], s["w"], *q[0], *q[1], s["y"], s["ws"])
    return s, step, q


@pytest.mark.parametrize("T", [1, 24, 70])
def test_serving_step(T):
    s, step, q = serve_state(T, 128, 160, 16, 2, T)
    step()
    torch.cuda.synchronize()
    idx, w, load = O.route(s["lg"].cpu().numpy(), s["bias"].cpu().numpy(), 2, "sigmoid", groups=4, top_groups=2, scale=2.5)
    assert np.array_equal(s["idx"].cpu().numpy(), idx) and np.array_equal(s["load"].cpu().numpy(), load)
    dec = [O.w4_decode(*(v.cpu().numpy() for v in p)) for p in q]
    ref, err = O.experts(s["x"].double().cpu().numpy(), idx, s["w"].double().cpu().numpy(), *dec, "gelu_tanh")
    got = s["y"].double().cpu().numpy()
    assert (np.abs(got - ref) <= err + 2.0 ** -8 * (np.abs(ref) + err)).all()


@pytest.mark.parametrize("T", [3, 70])
def test_serving_step_in_a_graph(T):
    s, step, _ = serve_state(T, 128, 160, 16, 2, T)
    step()                                           # loads the kernels
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        s["x"].copy_(torch.randn(T, 128, generator=torch.Generator().manual_seed(i)).bfloat16())
        s["ws"].fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        got = {n: s[n].clone() for n in ("idx", "w", "load", "y")}
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], s[n]) for n in got), i


def test_training_step_in_a_graph():
    cfg, b, t, r = build("bf16", 130, 128, 192, 8, 2, 3, score="sigmoid", groups=4, top_groups=2)
    ck = L.alloc_ckpt(cfg)

    def step():
        r.load.zero_()
        L.layer_forward(b, t["x"], t["Wg"], None, t["W1"], t["W2"], router=r)
        L.layer_save(b, ck)
        L.layer_restore(b, ck)
        L.layer_backward(b, t["x"], t["Wg"], t["dy"], router=r)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    names = ("idx", "w", "y", "dw", "dlogits", "dx", "dW1", "dW2", "dWg")
    for i in range(4):
        t["x"].copy_(torch.randn(130, 128, generator=torch.Generator().manual_seed(i)).bfloat16())
        ck.fill_(0x7F)
        g.replay()
        torch.cuda.synchronize()
        got = {n: getattr(b, n).clone() for n in names}
        load = r.load.clone()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], getattr(b, n)) for n in names) and torch.equal(load, r.load), i


def test_two_layers_share_buffers_through_checkpoints():
    """Forward of both layers in one set of expert buffers, backward from the checkpoints."""
    cfg, b, t, r = build("bf16", 150, 128, 192, 8, 2, 21, score="sigmoid")
    _, b2, t2, r2 = build("bf16", 150, 128, 192, 8, 2, 22, score="softmax")
    for n in ("send_buf", "H", "A", "O", "dO", "dH", "dXe"):
        setattr(b2, n, getattr(b, n))
    cks = [L.alloc_ckpt(cfg), L.alloc_ckpt(cfg)]
    for bb, tt, rr, ck in ((b, t, r, cks[0]), (b2, t2, r2, cks[1])):
        L.layer_forward(bb, tt["x"], tt["Wg"], None, tt["W1"], tt["W2"], router=rr)
        L.layer_save(bb, ck)
    for bb, tt, rr, ck, route in ((b2, t2, r2, cks[1], ("softmax", 1, 1.0)), (b, t, r, cks[0], ("sigmoid", 1, 1.0))):
        L.layer_restore(bb, ck)
        L.layer_backward(bb, tt["x"], tt["Wg"], tt["dy"], router=rr)
        torch.cuda.synchronize()
        for n, v in reference(cfg, bb, tt, route).items():
            assert_close(n, getattr(bb, n).double().cpu().numpy(), v, TOL["bf16"])
