"""Sorted rows, token lookup and cross entropy past 32-bit byte offsets."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")
from oracle import training_oracle as O  # noqa: E402


def test_lookup_in_a_table_of_over_four_gib():
    V, d, T = 300000, 8192, 2000
    W = torch.randn(V, 8, device="cuda").bfloat16().repeat(1, d // 8)
    assert W.numel() * 2 > 1 << 32
    ids = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    ids[:4] = torch.tensor([V - 1, 0, V - 1, V], dtype=torch.int32)
    cfg = L.make_embed_cfg(T, V, d, "bf16", 0.5)
    y = torch.empty(T, d, device="cuda", dtype=torch.bfloat16)
    L.moe_embed(cfg, ids, W, y)
    assert O.off(y, O.embed(ids, W, 0.5)) <= 1
    ws = torch.empty(L.moe_embed_bwd_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    L.moe_embed_bwd(cfg, ids, y, W, ws)          # over the table: every row is written
    live = ids < V
    want = O.embed_bwd(torch.unique(ids[live], return_inverse=True)[1].int(), y[live], int(torch.unique(ids[live]).numel()), 0.5)
    rows = torch.unique(ids[live]).long()
    assert O.off(W[rows], want) <= 1
    W[rows] = 0
    assert not W.any()


def test_rows_of_over_four_gib():
    """More rows than 32-bit offsets reach (the products refuse them; sorting, gathering and summing do not)."""
    T, d, E, k = 150000, 4096, 8, 4
    cfg = L.make_sorted_cfg(T, d, 64, E, k)
    R = L.moe_sorted_rows(cfg)
    assert R * d * 2 > 1 << 32
    x = torch.randn(T, 16, device="cuda").bfloat16().repeat(1, d // 16)
    idx = torch.argsort(torch.rand(T, E, device="cuda"), dim=1)[:, :k].int().contiguous()
    i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")   # noqa: E731
    rb, re, sl, sr = i32(E), i32(E), i32(T, k), i32(R)
    rows = torch.zeros(R, d, device="cuda", dtype=torch.bfloat16)
    ws = torch.empty(L.moe_sorted_workspace_bytes(cfg, L.MOE_CALL_DISPATCH), dtype=torch.uint8, device="cuda")
    L.moe_sorted_dispatch(cfg, x, idx, rb, re, sl, sr, rows, ws)
    held = sr >= 0
    assert int(held.sum()) == T * k
    last = torch.nonzero(held).squeeze(1)[-1000:]
    # element (r, c) of the blocks, of the last rows
    c = torch.arange(d, device="cuda")
    at = ((last // 16).unsqueeze(1) * (d // 32) + c // 32) * 512 + (last % 16).unsqueeze(1) * 32 + c % 32
    assert torch.equal(rows.view(-1)[at], x[sr[last].long() // k])
    w = torch.rand(T, k, device="cuda")
    y = torch.empty_like(x)
    L.moe_sorted_combine(cfg, rows, sl, w, y)    # (the same buffer taken as row-major)
    some = torch.arange(T - 500, T, device="cuda")
    assert O.off(y[some], O.back(rows, sl[some], w[some])) <= 1
    dO, dw = torch.zeros_like(rows), torch.empty(T, k, device="cuda")
    L.moe_sorted_combine_bwd(cfg, rows, sl, sr, w, x, dO, dw)
    i = sr[last].long()
    assert O.off(dO.view(-1)[at], (x.double()[i // k] * w.double().reshape(-1)[i].unsqueeze(1),
                                   (O.UBF + O.U32) * (x.double()[i // k] * w.double().reshape(-1)[i].unsqueeze(1)).abs())) <= 1
    p = x.double()[i // k] * rows.double()[last] if rows.numel() < 1 << 31 else torch.stack(
        [x[q // k].double() * rows[r].double() for q, r in zip(i.tolist(), last.tolist())])
    assert O.off(dw.reshape(-1)[i], (p.sum(1), (d + 8) * O.U32 * p.abs().sum(1))) <= 1


@pytest.mark.parametrize("T", [3, 300])
def test_vocabulary_of_over_four_gib(T):
    """The output matrix in pieces that 32-bit offsets reach, forward and backward."""
    V, d = 70000, 32768
    torch.manual_seed(T)
    W = (torch.randn(V, 64, device="cuda") * 0.01).bfloat16().repeat(1, d // 64)
    assert W.numel() * 2 > 1 << 32
    x = (torch.randn(T, d, device="cuda") * 0.1).bfloat16()
    target = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    target[:2] = torch.tensor([V - 1, 0], dtype=torch.int32)
    dloss = torch.rand(T, device="cuda")
    cfg = L.make_xent_cfg(T, V, d)
    ws = torch.empty(max(L.moe_xent_workspace_bytes(cfg, b) for b in (0, 1)), dtype=torch.uint8, device="cuda")
    loss, lse, dx, dW = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(x), torch.empty_like(W)
    L.moe_xent(cfg, x, W, target, loss, lse, ws)
    L.moe_xent_bwd(cfg, x, W, target, lse, dloss, dx, dW, ws)
    want = O.xent(x, W, target, dloss)
    for n, got in (("loss", loss), ("lse", lse), ("dx", dx), ("dW", dW)):
        assert O.off(got, want[n]) <= 1, n
