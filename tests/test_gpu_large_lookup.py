"""Token lookup and its gradient where one thread for each piece of work would be more than a launch counts
(2^32 threads)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")


@pytest.mark.parametrize("dtype,T", [(torch.bfloat16, (1 << 24) + 3), (torch.float32, (1 << 23) + 3)])
def test_lookup_of_over_64_gib(dtype, T):
    V, d = 1000, 2048
    assert T * d * dtype.itemsize // 16 > 1 << 32
    W = torch.randn(V, d, device="cuda").to(dtype)
    ids = torch.randint(-1, V + 1, (T,), device="cuda", dtype=torch.int32)
    y = torch.full((T, d), 7.0, device="cuda", dtype=dtype)
    L.moe_embed(L.make_embed_cfg(T, V, d, "bf16" if dtype == torch.bfloat16 else "f32"), ids, W, y)
    table = torch.cat([W, torch.zeros(1, d, device="cuda", dtype=dtype)])
    at = torch.where(ids < 0, V, ids).long()
    for a in range(0, T, 1 << 20):
        assert torch.equal(y[a:a + (1 << 20)], table[at[a:a + (1 << 20)]]), a
    del y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("accum", [0, 1])
def test_gradient_of_over_2_to_28_tokens(accum):
    """Every id's tokens cross many runs, also past the last run of the first launch.  Whole numbers: exact sums."""
    T, V, d = (1 << 28) + 5, 1000, 8
    ids = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    col = torch.arange(1, d + 1, device="cuda")
    dy = torch.empty(T, d, device="cuda")
    for a in range(0, T, 1 << 24):
        dy[a:a + (1 << 24)] = ((ids[a:a + (1 << 24)] % 5 + 1).unsqueeze(1) * col).float()
    cfg = L.make_embed_cfg(T, V, d, "f32", 1.0, accum)
    ws = torch.empty(L.moe_embed_bwd_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    dW = torch.full((V, d), 2.0, device="cuda")
    L.moe_embed_bwd(cfg, ids, dy, dW, ws)
    n = torch.bincount(ids, minlength=V)
    want = (n * (torch.arange(V, device="cuda") % 5 + 1)).unsqueeze(1) * col + 2 * accum
    assert int(want.max()) < 1 << 24
    assert torch.equal(dW.long(), want)
    del dy, ws
    torch.cuda.empty_cache()
