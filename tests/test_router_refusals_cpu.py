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
