"""The loss's workspaces against what the header says of them, over few and many tokens of either type."""
import pytest

L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")

SIZES = [(1, 50257, 64), (63, 50257, 64), (64, 50257, 1024), (1024, 100003, 512), (1025, 100003, 512), (8191, 50257, 2048),
         (8192, 50257, 2048), (65536, 32000, 1024), (131072, 50257, 1024), (262144, 65536, 256), (1 << 21, 65536, 200),
         (1 << 22, 4096, 40), (1 << 20, 65600, 64), (300, 70000, 32768), (5, 1 << 20, 64), (100, 3, 1 << 15)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", SIZES)
def test_workspaces(T, V, d, dtype):
    d = d // 64 * 64 or 64 if dtype == "bf16" else d
    e, rows = (2, -(-T // 16) * 16) if dtype == "bf16" else (4, -(-T // 16) * 16)
    cfg = L.make_xent_cfg(T, V, d, dtype)
    fwd, bwd = (L.moe_xent_workspace_bytes(cfg, b) for b in (False, True))
    assert fwd > 0 and bwd > 0
    # the runs, and in each piece of the vocabulary what whole tiles leave past its end
    a_logit = (2 if T <= 1024 else 1) / (8 if dtype == "bf16" else 4)
    blocked = dtype == "bf16" and T >= 8192
    pieces = 2 * (1 + 2 * V * d // ((1 << 27) if blocked else (1 << 31)) + T * V // (1 << 35))
    copies = 2 * rows * d + (max(1 << 27, 512 * d) if blocked else 0) if dtype == "bf16" else 0
    assert fwd <= a_logit * T * V + (8 + 256 * pieces) * T + 4 * T + copies + 4 * 256
    dl = max(512 << 20, min(2048 * rows * e, 1 << 31 if dtype == "bf16" else 1 << 32), 64 * rows * e)
    w = min(V + 16, dl // (rows * e) + 16) * d * 2 if blocked else 0      # a piece of W
    x = rows * d * (e + (4 if dtype == "bf16" else 0))                     # x, and the float sums of dx
    assert bwd <= dl + 64 * rows * e + x + w + (64 << 20) + 6 * 256        # (partial tiles or slices: 64 MiB)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_tokens_need_none(dtype):
    cfg = L.make_xent_cfg(0, 1000, 64, dtype)
    assert [L.moe_xent_workspace_bytes(cfg, b) for b in (False, True)] == [0, 0]
