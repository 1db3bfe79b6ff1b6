"""Float cross entropy whose dx is a sum over pieces of the vocabulary and, in each, over slices of it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")
from oracle import training_oracle as O  # noqa: E402


@pytest.mark.parametrize("T,V,d", [(20000, 10007, 64), (9000, 40009, 72)])   # two and three pieces, in three slices each
def test_slices_of_pieces(T, V, d):
    torch.manual_seed(T)
    x, W = torch.randn(T, d, device="cuda"), torch.randn(V, d, device="cuda") * 0.1
    target = torch.randint(-1, V, (T,), device="cuda", dtype=torch.int32)
    dloss = torch.rand(T, device="cuda") - 0.3
    cfg = L.make_xent_cfg(T, V, d, "f32")
    ws = torch.full((max(L.moe_xent_workspace_bytes(cfg, b) for b in (0, 1)),), 0xff, dtype=torch.uint8, device="cuda")
    loss, lse, dx, dW = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.full_like(x, 7.0), torch.full_like(W, 7.0)
    L.moe_xent(cfg, x, W, target, loss, lse, ws)
    L.moe_xent_bwd(cfg, x, W, target, lse, dloss, dx, dW, ws)
    want = O.xent(x, W, target, dloss)
    for n, got in (("loss", loss), ("lse", lse), ("dx", dx), ("dW", dW)):
        assert O.off(got, want[n]) <= 1, n
    again = torch.full_like(dx, 5.0)
    ws.fill_(0xff)
    L.moe_xent_bwd(cfg, x, W, target, lse, dloss, again, None, ws)
    assert torch.equal(again, dx)
