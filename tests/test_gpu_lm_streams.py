"""The step of token lookup, blocks and loss in partitions over three streams: the bits of one partition on one
stream, eagerly and from a captured graph."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")

B, S, HEADS, FF, E, K, V, BLOCKS = 4, 200, 2, 512, 8, 2, 5003, 3


class Step:
    def __init__(self, n_chunks, tied, seed=2):
        torch.manual_seed(seed)
        T = B * S
        self.n = n_chunks
        self.cfg = L.make_block_cfg(B, S, HEADS, FF, E, K, L.moe_capacity(T, E, K, 5, 4))
        shp = L.block_shapes(self.cfg, n_chunks)
        self.weights = []
        for _ in range(BLOCKS):
            w = {n: (torch.randn(shp[n][0], device="cuda") * 0.05).bfloat16() for n in L.BLOCK_WEIGHTS}
            for n in ("ln1_g", "ln2_g"):
                w[n] += 1
            self.weights.append(w)
        d = 128 * HEADS
        self.Wout = (torch.randn(V, d, device="cuda") * 0.05).bfloat16()
        self.Win = self.Wout if tied else (torch.randn(V, d, device="cuda") * 0.05).bfloat16()
        self.ids = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
        self.target = torch.roll(self.ids, -1)
        self.ids[-5:], self.target[-6:] = -1, -1
        self.dloss = torch.full((T,), 1 / (T - 6), device="cuda")
        self.acts = [L.alloc_block(self.cfg, n_chunks) for _ in range(BLOCKS)]
        self.b = L.alloc_lm(self.cfg, V, BLOCKS, scale=16.0, tied=tied)

    def run(self, streams):
        L.lm_forward(self.b, self.cfg, self.ids, self.target, self.Win, self.Wout, self.weights, self.acts, self.n, streams)
        L.lm_backward(self.b, self.cfg, self.ids, self.target, self.Wout, self.weights, self.acts, self.acts, self.dloss,
                      self.n, streams)

    def results(self):
        out = {"loss": self.b.loss, "lse": self.b.lse, "dWout": self.b.dWout}
        if self.b.dWin is not None:
            out["dWin"] = self.b.dWin
        for i, a in enumerate(self.acts):
            out |= {f"{n}[{i}]": a[n] for n in L.BLOCK_GRADS}
        return out

    def clear(self):
        for v in list(self.results().values()) + self.b.h + [self.b.dh, self.b.dx]:
            v.fill_(3.0)
        torch.cuda.synchronize()


def _one_stream(tied):
    s = Step(1, tied)
    s.run([torch.cuda.current_stream()] * 3)
    torch.cuda.synchronize()
    return {n: v.clone() for n, v in s.results().items()}


@pytest.mark.parametrize("n_chunks", [1, 2, 4])
@pytest.mark.parametrize("tied", [True, False])
@pytest.mark.parametrize("how", ["objects", "handles"])
def test_three_streams(how, tied, n_chunks):
    want, s = _one_stream(tied), Step(n_chunks, tied)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for i in range(3):
        s.clear()
        s.run(streams if how == "objects" else [q.cuda_stream for q in streams])
        torch.cuda.synchronize()
        for n, v in s.results().items():
            assert torch.equal(v, want[n]), (i, n)


@pytest.mark.parametrize("n_chunks", [1, 2])
def test_captured(n_chunks):
    want, s = _one_stream(True), Step(n_chunks, True)
    side = [torch.cuda.Stream() for _ in range(2)]
    s.run([torch.cuda.current_stream()] + side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run([torch.cuda.current_stream()] + side)
    keep = s.ids.clone()
    for i in range(3):
        s.ids.copy_(torch.randint_like(s.ids, 0, V))
        s.run([torch.cuda.current_stream()] + side)          # eager work on other tokens between the replays
        s.ids.copy_(keep)
        s.clear()
        graph.replay()
        torch.cuda.synchronize()
        for n, v in s.results().items():
            assert torch.equal(v, want[n]), (i, n)
