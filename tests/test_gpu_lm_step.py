"""The step of token lookup, blocks and loss: each part against its 64-bit form on the step's
own activations, the blocks against their own calls, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")
from oracle import training_oracle as O  # noqa: E402


def _make(B=2, S=96, heads=2, f=384, E=4, k=2, V=1003, n_blocks=2, tied=True, seed=0):
    torch.manual_seed(seed)
    T = B * S
    C = L.moe_capacity(T, E, k, 5, 4)
    cfg = L.make_block_cfg(B, S, heads, f, E, k, C)
    shp = L.block_shapes(cfg, 1)
    weights = []
    for _ in range(n_blocks):
        w = {n: (torch.randn(shp[n][0], device="cuda") * 0.05).bfloat16() for n in L.BLOCK_WEIGHTS}
        for n in ("ln1_g", "ln2_g"):
            w[n] += 1
        weights.append(w)
    acts = [L.alloc_block(cfg, 1) for _ in range(n_blocks)]
    b = L.alloc_lm(cfg, V, n_blocks, scale=16.0, tied=tied)
    d = 128 * heads
    Wout = (torch.randn(V, d, device="cuda") * 0.05).bfloat16()
    Win = Wout if tied else (torch.randn(V, d, device="cuda") * 0.05).bfloat16()
    ids = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    target = torch.roll(ids, -1)
    ids[-5:], target[-6:] = -1, -1                       # a padded batch
    dloss = torch.full((T,), 1 / (T - 6), device="cuda")
    return cfg, b, weights, acts, Win, Wout, ids, target, dloss


@pytest.mark.parametrize("tied", [True, False])
def test_step(tied):
    cfg, b, weights, acts, Win, Wout, ids, target, dloss = _make(tied=tied)
    s = [torch.cuda.current_stream()] * 3
    L.lm_forward(b, cfg, ids, target, Win, Wout, weights, acts, 1, s)
    L.lm_backward(b, cfg, ids, target, Wout, weights, acts, acts, dloss, 1, s)
    torch.cuda.synchronize()
    assert O.off(b.h[0], O.embed(ids, Win, 16.0)) <= 1
    want = O.xent(b.h[-1], Wout, target, dloss)
    assert O.off(b.loss, want["loss"]) <= 1
    # the blocks once more, by their own calls
    dy = torch.empty_like(b.h[0])
    dW = torch.empty_like(Wout)
    L.moe_xent_bwd(b.xent, b.h[-1], Wout, target, b.lse, dloss, dy, dW, b.ws)
    assert O.off(dy, want["dx"]) <= 1 and O.off(dW, want["dW"]) <= 1
    for i in reversed(range(len(weights))):
        again = L.alloc_block(cfg, 1)
        out, dx = torch.empty_like(b.h[0]), torch.empty_like(b.h[0])
        L.moe_block_chunked(cfg, weights[i], again, b.h[i], out, dy, dx, again, L.MOE_BLOCK_FWD | L.MOE_BLOCK_BWD, 1, s,
                            again["ws"])
        assert torch.equal(out, b.h[i + 1]), i
        for n in L.BLOCK_GRADS:
            assert torch.equal(again[n], acts[i][n]), (i, n)
        dy = dx
    if tied:
        assert O.off(b.dWout, O.embed_bwd(ids, dy, Wout.shape[0], 16.0, dW)) <= 1
    else:
        assert torch.equal(b.dWout, dW)
        assert O.off(b.dWin, O.embed_bwd(ids, dy, Win.shape[0], 16.0)) <= 1


def test_graph_replays_the_step():
    cfg, b, weights, acts, Win, Wout, ids, target, dloss = _make(seed=3)

    def step():
        s = [torch.cuda.current_stream()] * 3
        L.lm_forward(b, cfg, ids, target, Win, Wout, weights, acts, 1, s)
        L.lm_backward(b, cfg, ids, target, Wout, weights, acts, acts, dloss, 1, s)
    step()
    torch.cuda.synchronize()
    want = {"loss": b.loss.clone(), "dWout": b.dWout.clone(), "dW1": acts[0]["dW1"].clone()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    keep = ids.clone()
    for _ in range(3):
        ids.copy_(torch.randint_like(ids, 0, 1003))
        step()
        ids.copy_(keep)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.loss, want["loss"]) and torch.equal(b.dWout, want["dWout"])
        assert torch.equal(acts[0]["dW1"], want["dW1"])
