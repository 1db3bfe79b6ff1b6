"""Sizes whose launches would have 2^32 threads or more, of which the device runs the remainder only: refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu
L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")


def _layer(T):
    cfg = L.make_cfg(T, 8, 8, 1, 1, 16, dtype="f32")
    b = L.alloc_layer(cfg)
    x, Wg, W1, W2 = torch.ones(T, 8, device="cuda"), *(torch.ones(1, 8, *s, device="cuda") for s in ((), (8,), (8,)))
    L.layer_forward(b, x, Wg, None, W1, W2)
    return b, x, Wg


def test_a_layer_of_over_2_to_26_tokens():
    """A wave a token in the combine's backward and in the importance keys."""
    T = (1 << 26) + 4096
    b, x, Wg = _layer(T)
    b.dx.fill_(7.0)
    with pytest.raises(L.MoeError) as e:
        L.layer_backward(b, x, Wg, x)
    assert e.value.status == L.MOE_ELAUNCH and "2^32" in str(e.value)
    order = torch.full((T,), -7, dtype=torch.int32, device="cuda")
    ws = torch.empty(L.moe_workspace_bytes(b.cfg, L.MOE_CALL_DISPATCH_BPR), dtype=torch.uint8, device="cuda")
    with pytest.raises(L.MoeError) as e:
        L.moe_dispatch_bpr(b.cfg, x, b.logits, b.idx, b.fill, b.slot, b.send_buf, order, ws)
    assert e.value.status == L.MOE_ELAUNCH
    torch.cuda.synchronize()
    assert bool((b.dx == 7).all()) and bool((order == -7).all())      # nothing of the call has run
    small, x, Wg = _layer(100)                                        # and the next call runs as ever
    L.layer_backward(small, x, Wg, x)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(small.dx).all())
