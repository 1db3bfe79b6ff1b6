"""What the router's calls and the layer with a router refuse, without a GPU."""
import ctypes

import pytest

from tests.test_operators_cpu import L, P, bwd_dx_route, lib, no_device, rcfg


@no_device
@pytest.mark.parametrize("out,at", [("dw", 15), ("dlogits", 16)])
def test_bwd_dx_route_outputs_alias_no_array(out, at):
    c = L.make_cfg(64, 128, 256, 16, 2, 20)
    names = ["Wg", "logits", "idx", "w", "slot", "rb", "re", "H", "O", "W1p", "W2p", "dy", "dO", "dH", "dXe", "dw",
             "dlogits", "dx"]
    for i, n in enumerate(names):
        if i != at:
            assert bwd_dx_route(c, rcfg(), **{out: P(i)}) == L.MOE_EINVAL and "alias" in L.moe_last_error(), n
    assert bwd_dx_route(c, rcfg(), rb=None) == L.MOE_EDEVICE     # valid; no GPU here
    z = L.make_cfg(0, 128, 256, 16, 2, 20)
    assert bwd_dx_route(z, rcfg(T=0), dw=None, dlogits=None) == L.MOE_EDEVICE


@no_device
def test_route_bwd_output_aliases_no_input():
    c = rcfg(E=2)                                                # dlogits and the choices are of one size
    for i in range(4):
        assert lib.moe_route_bwd(ctypes.byref(c), P(0), P(1), P(2), P(3), P(i), None) == L.MOE_EINVAL
        assert "alias" in L.moe_last_error()


def bpr_route(c, r, n=None, **over):
    names = ["x", "logits", "idx", "fill", "slot", "send", "order", "ws"]
    p = [over.get(m, P(i)) for i, m in enumerate(names)]
    need = L.moe_workspace_bytes(c, L.MOE_CALL_DISPATCH_BPR) if n is None else n
    return lib.moe_dispatch_bpr_route(ctypes.byref(c), None if r is None else ctypes.byref(r), *p, need, None)


@no_device
def test_dispatch_bpr_route_refused():
    c = L.make_cfg(64, 128, 256, 16, 2, 20)
    assert bpr_route(c, rcfg()) == L.MOE_EDEVICE and bpr_route(c, rcfg(), order=None) == L.MOE_EDEVICE   # valid
    assert bpr_route(c, None) == L.MOE_EINVAL
    for kw in (dict(T=65), dict(E=32), dict(k=3)):
        assert bpr_route(c, rcfg(**kw)) == L.MOE_EINVAL and "differ" in L.moe_last_error()
    assert bpr_route(c, rcfg(score=2)) == L.MOE_EINVAL and bpr_route(L.make_cfg(64, 12, 256, 16, 2, 20), rcfg()) == L.MOE_ESHAPE
    assert bpr_route(c, rcfg(), n=64) == L.MOE_EWORKSPACE and bpr_route(c, rcfg(), ws=None) == L.MOE_EWORKSPACE
    assert bpr_route(c, rcfg(), logits=None) == L.MOE_EINVAL and bpr_route(c, rcfg(), order=8) == L.MOE_EALIGN
    z = L.make_cfg(0, 128, 256, 16, 2, 20)
    assert bpr_route(z, rcfg(T=0), x=None, logits=None, idx=None, slot=None) == L.MOE_EDEVICE


def test_layer_forward_refuses_a_router_of_another_layer():
    """Before anything is launched: tokens past a shorter router's would keep the gate's own choices."""
    import types
    b = types.SimpleNamespace(cfg=L.make_cfg(64, 128, 256, 16, 2, 20))
    for kw in (dict(T=63), dict(T=65), dict(E=32), dict(k=1)):
        with pytest.raises(ValueError, match="router"):
            L.layer_forward(b, None, None, None, None, None, router=L.Router(rcfg(**kw)))


def test_layer_buffers_of_a_layer_without_a_router():
    """The gradient at w is a router's: a layer without one is built without it."""
    import dataclasses
    names = [f.name for f in dataclasses.fields(L.LayerBuffers)]
    b = L.LayerBuffers(**{n: None for n in names if n != "dw"})
    assert b.dw is None
