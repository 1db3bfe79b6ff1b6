"""What the step of lookup, blocks and loss refuses before anything runs."""
import pytest
import torch

L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")


def _cfg(B=2, S=16, heads=1):
    return L.make_block_cfg(B, S, heads, 64, 2, 1, 64)


@pytest.mark.parametrize("cfg,V,scale", [(_cfg(B=1 << 12, S=1 << 12, heads=8), 100, 1.0),     # 2^34 elements of x
                                         (_cfg(), 0, 1.0), (_cfg(), 100, float("inf")), (_cfg(), (1 << 30) + 1, 1.0)])
def test_sizes_that_the_calls_do_not_take(monkeypatch, cfg, V, scale):
    monkeypatch.setattr(torch, "empty", lambda *a, **k: pytest.fail("allocated"))
    with pytest.raises(L.MoeError):
        L.alloc_lm(cfg, V, scale=scale, device="cpu")


def test_no_tokens_are_allowed():
    assert L.alloc_lm(_cfg(B=0), 100, device="cpu").ws.numel() == 16


@pytest.mark.parametrize("weights,acts", [(1, 2), (2, 1), (1, 1), (3, 3)])
def test_other_numbers_of_blocks(monkeypatch, weights, acts):
    b = L.alloc_lm(_cfg(), 100, n_blocks=2, device="cpu")
    for n in ("moe_embed", "moe_xent", "moe_xent_bwd", "moe_block_chunked", "moe_embed_bwd"):
        monkeypatch.setattr(L, n, lambda *a, **k: pytest.fail("called"))
    w, a = [{}] * weights, [{"ws": None}] * acts
    with pytest.raises(ValueError):
        L.lm_forward(b, _cfg(), None, None, None, None, w, a, 1, [None] * 3)
    with pytest.raises(ValueError):
        L.lm_backward(b, _cfg(), None, None, None, w, w, a, None, 1, [None] * 3)
