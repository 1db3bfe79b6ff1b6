"""Router, 4-bit experts and 8-bit checkpoint without a GPU: the oracle's pins (hand-worked
values, differences) and every refusal of the C ABI and of the binding."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as O

L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")
lib = L._lib
GOOD = 4096   # a fake, 16-byte aligned address: validation never dereferences it


def P(i):
    return GOOD * (i + 1)


# ------------------------------------------------------------------- oracle pins
def test_route_hand_worked():
    # sigmoid scores .5, .731.., .881.., .269..; the bias moves expert 3 past all, not its weight
    l = np.array([[0.0, 1.0, 2.0, -1.0]])
    idx, w, load = O.route(l, None, 2, "sigmoid", renorm=1)
    s = 1 / (1 + np.exp(-l[0]))
    assert idx.tolist() == [[2, 1]] and np.allclose(w, [[s[2] / (s[1] + s[2]), s[1] / (s[1] + s[2])]])
    idx, w, load = O.route(l, [0, 0, 0, 1.0], 2, "sigmoid", renorm=0, scale=2.0)
    assert idx.tolist() == [[3, 2]] and np.allclose(w, [[2 * s[3], 2 * s[2]]]) and load.tolist() == [0, 0, 1, 1]
    # groups {0, 1} and {2, 3}: 0.5 + 0.731 beats 0.881 + 0.269
    assert O.route(l, None, 2, "sigmoid", groups=2, top_groups=1)[0].tolist() == [[1, 0]]
    # ties go to the lowest index, masked experts are not chosen, an empty row chooses none
    l = np.array([[1.0, 1.0, 1.0], [-np.inf, np.nan, 3.0], [-np.inf] * 3])
    idx, w, load = O.route(l, None, 2)
    assert idx.tolist() == [[0, 1], [2, -1], [-1, -1]] and w.tolist() == [[0.5, 0.5], [1.0, 0.0], [0.0, 0.0]]
    # equal groups: the lowest; +inf logits share the softmax
    assert O.route(np.zeros((1, 4)), None, 2, groups=2, top_groups=1)[0].tolist() == [[0, 1]]
    assert O.route(np.array([[np.inf, 0.0, np.inf]]), None, 3, renorm=0)[1].tolist() == [[0.5, 0.5, 0.0]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [0, 1])
def test_route_gradient_against_differences(score, renorm):
    rng = np.random.default_rng(3)
    l = rng.standard_normal((5, 7))
    l[4, 2] = -np.inf
    idx = O.route(l, None, 3, score, renorm)[0]
    idx[1, 2] = -1
    dw = rng.standard_normal((5, 3))
    dl, mag = O.route_bwd(l, idx, dw, score, renorm, 2.5)
    f = lambda v: (dw * O.route_weights(v, idx, score, renorm, 2.5)).sum()   # noqa: E731
    h = 1e-5
    for t in range(5):
        for e in range(7):
            a, b = l.copy(), l.copy()
            a[t, e] += h
            b[t, e] -= h
            # central differences: h^2 / 6 of third derivatives (below 2.5 * 16) and 1e-16 / h of rounding
            assert abs((f(a) - f(b)) / (2 * h) - dl[t, e]) < 1e-9, (t, e)
    assert (np.abs(dl) <= mag + 1e-300).all()


def test_w4_codes_hand_worked():
    x = np.zeros((1, 32))
    x[0, :12] = [7.0, -6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.01, 0.26, -0.0]
    c, s = O.w4_quantize(x)
    q = np.stack((c & 15, c >> 4), -1).reshape(-1)
    assert s.tolist() == [[127]] and q[:12].tolist() == [7, 15, 0, 2, 2, 4, 4, 6, 6, 15, 1, 8]
    assert O.w4_quantize(x * 1.001)[1].tolist() == [[128]] and O.w4_quantize(x / 2)[1].tolist() == [[126]]
    d = O.w4_decode(c, s)
    assert d[0, :4].tolist() == [6.0, -6.0, 0.0, 1.0]
    x[0, 5] = np.inf
    assert np.isnan(O.w4_decode(*O.w4_quantize(x))).all()


def test_w4_error_is_half_a_spacing():
    x = np.random.default_rng(0).standard_normal((20, 64)) * np.exp2(np.arange(20) - 10.0)[:, None]
    c, s = O.w4_quantize(x)
    u = np.repeat(2.0 ** (s.astype(float) - 127), 32, -1)
    a = np.abs(x) / u
    gap = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert (np.abs(O.w4_decode(c, s) - x) <= gap / 2 * u * (1 + 1e-12)).all() and a.max() <= 7


def test_ckpt_oracle_hand_worked():
    x = np.zeros((2, 72), np.float32)
    x[0, :4] = [127.0, -63.5, 62.5, 0.49]
    x[0, 64:67] = [1e-31, 0.0, -1e-31]
    x[1, 3], x[1, 70] = np.nan, 5.0
    y = O.ckpt_round_trip(x)
    assert y[0, :4].tolist() == [127.0, -64.0, 62.0, 0.0] and (y[0, 64:] == 0).all()
    assert np.isnan(y[1, :64]).all() and y[1, 70] == 5.0 and (y[1, 64:70] == 0).all()


def test_bf16_codes_rounding_rule_holds_for_every_pair():
    """The kernel's rule for bfloat16 (a float product, rounded to 19 bits, then to an integer) against
    exact integers: every pair of significands, exponents 0 .. 9 apart."""
    A = np.arange(128, 256)
    for s in range(10):
        X = np.arange(128, 256)
        if s == 0:
            x, a = np.meshgrid(X, A, indexing="ij")
            x, a = x[x <= a], a[x <= a]
        else:
            x, a = (v.reshape(-1) for v in np.meshgrid(X, A, indexing="ij"))
        for scale in (1.0, 2.0 ** -40, 2.0 ** 60):
            amax = (a * scale).astype(np.float32)
            v = (x * 2.0 ** -s * scale).astype(np.float32)
            q = v * (np.float32(127) / amax)
            q = ((q.view(np.uint32) + np.uint32(8)) & ~np.uint32(15)).view(np.float32)
            got = np.rint(q).astype(np.int64)
            num, den = 2 * 127 * x, a * 2 ** s            # twice the quotient
            lo = num // (2 * den)
            rest = num - 2 * den * lo                      # against den: below, at or above the half
            want = lo + ((rest > den) | ((rest == den) & (lo % 2 == 1)))
            assert np.array_equal(got, want), s


# ------------------------------------------------------------------ struct layout
def test_struct_layouts():
    assert ctypes.sizeof(L.moe_route_cfg) == 40 and L.moe_route_cfg.scale.offset == 32
    assert ctypes.sizeof(L.moe_w4_cfg) == 32 and L.moe_w4_cfg.act.offset == 28


# ----------------------------------------------------------------------- refusals
# These calls pass addresses that are none: on a machine with a device a valid one would run.
no_device = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="passes addresses that are not memory")


def rcfg(**kw):
    base = dict(T=64, E=16, k=2)
    base.update(kw)
    return L.make_route_cfg(**base)


def route(c, logits=P(0), bias=None, idx=P(1), w=P(2), load=None):
    return lib.moe_route(ctypes.byref(c) if c is not None else None, logits, bias, idx, w, load, None)


@no_device
@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), L.MOE_EINVAL), (dict(T=2 ** 31 + 1), L.MOE_ESHAPE), (dict(E=0), L.MOE_ESHAPE),
    (dict(E=513), L.MOE_ESHAPE), (dict(k=0), L.MOE_EINVAL), (dict(k=17), L.MOE_EINVAL), (dict(E=4, k=5), L.MOE_EINVAL),
    (dict(score=2), L.MOE_EINVAL), (dict(score=-1), L.MOE_EINVAL), (dict(renorm=2), L.MOE_EINVAL),
    (dict(groups=0), L.MOE_EINVAL), (dict(groups=3), L.MOE_EINVAL), (dict(groups=4, top_groups=5), L.MOE_EINVAL),
    (dict(groups=4, top_groups=0), L.MOE_EINVAL), (dict(groups=16, top_groups=1), L.MOE_EINVAL),
    (dict(scale=0.0), L.MOE_EINVAL), (dict(scale=-1.0), L.MOE_EINVAL), (dict(scale=math.inf), L.MOE_EINVAL),
    (dict(scale=math.nan), L.MOE_EINVAL)])
def test_route_cfg_refused(kw, status):
    c = rcfg(**kw)
    assert route(c) == status and L.moe_last_error()
    assert lib.moe_route_bwd(ctypes.byref(c), P(0), P(1), P(2), P(3), P(4), None) == status


@no_device
def test_route_pointers():
    c = rcfg()
    assert route(None) == L.MOE_EINVAL
    assert route(c) == L.MOE_EDEVICE and route(c, bias=P(5), load=P(6)) == L.MOE_EDEVICE   # valid; no GPU here
    assert route(c, logits=None) == L.MOE_EINVAL and "logits is NULL" in L.moe_last_error()
    assert route(c, idx=P(1) + 4) == L.MOE_EALIGN and route(c, load=8) == L.MOE_EALIGN
    for kw in (dict(w=P(0)), dict(idx=P(0)), dict(idx=P(2)), dict(bias=P(5), w=P(5)), dict(load=P(1)), dict(bias=P(5), load=P(5))):
        assert route(c, **kw) == L.MOE_EINVAL and "alias" in L.moe_last_error(), kw
    z = rcfg(T=0)
    assert route(z, logits=None, idx=None, w=None) == L.MOE_EDEVICE
    assert lib.moe_route_bwd(ctypes.byref(c), P(0), P(1), P(2), P(3), P(0), None) == L.MOE_EINVAL
    assert "alias" in L.moe_last_error()
    assert lib.moe_route_bwd(ctypes.byref(c), P(0), P(1), P(2), P(3), None, None) == L.MOE_EINVAL
    assert lib.moe_route_bwd(ctypes.byref(z), None, None, None, None, None, None) == L.MOE_EDEVICE


def bwd_dx_route(c, r, ws=None, **over):
    names = ["Wg", "logits", "idx", "w", "slot", "rb", "re", "H", "O", "W1p", "W2p", "dy", "dO", "dH", "dXe", "dw",
             "dlogits", "dx"]
    p = [over.get(n, P(i)) for i, n in enumerate(names)]
    need = L.moe_workspace_bytes(c, L.MOE_CALL_BWD_DX)
    return lib.moe_bwd_dx_route(ctypes.byref(c), ctypes.byref(r), *p, P(30), need if ws is None else ws, None)


@no_device
def test_bwd_dx_route_refused():
    c = L.make_cfg(64, 128, 256, 16, 2, 20)
    assert bwd_dx_route(c, rcfg()) == L.MOE_EDEVICE
    assert bwd_dx_route(c, rcfg(), ws=16) == L.MOE_EWORKSPACE
    for kw in (dict(T=65), dict(E=32), dict(k=3)):
        assert bwd_dx_route(c, rcfg(**kw)) == L.MOE_EINVAL and "differ" in L.moe_last_error()
    assert bwd_dx_route(c, rcfg(scale=0.0)) == L.MOE_EINVAL
    assert bwd_dx_route(c, rcfg(), dw=None) == L.MOE_EINVAL and bwd_dx_route(c, rcfg(), dx=P(0) + 8) == L.MOE_EALIGN
    assert bwd_dx_route(c, rcfg(), dw=P(16)) == L.MOE_EINVAL and "alias" in L.moe_last_error()
    assert bwd_dx_route(L.make_cfg(64, 72, 256, 16, 2, 20), rcfg()) == L.MOE_ESHAPE


def wcfg(**kw):
    base = dict(T=8, d_model=64, d_ff=128, E=16, k=2)
    base.update(kw)
    return L.make_w4_cfg(**base)


def experts(c, ws=None, **over):
    names = ["x", "idx", "w", "W1c", "W1s", "W2c", "W2s", "y"]
    p = [over.get(n, P(i)) for i, n in enumerate(names)]
    need = L.moe_experts_w4_workspace_bytes(c) if ws is None else ws
    return lib.moe_experts_w4(ctypes.byref(c), *p, over.get("ws_ptr", P(20)), need, None)


@no_device
@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), L.MOE_EINVAL), (dict(d_model=48), L.MOE_ESHAPE), (dict(d_model=0), L.MOE_ESHAPE),
    (dict(d_ff=100), L.MOE_ESHAPE), (dict(d_ff=2 ** 20 + 32), L.MOE_ESHAPE), (dict(E=0), L.MOE_ESHAPE),
    (dict(E=513), L.MOE_ESHAPE), (dict(k=0), L.MOE_EINVAL), (dict(k=17), L.MOE_EINVAL), (dict(dtype=3), L.MOE_EDTYPE),
    (dict(act=4), L.MOE_EINVAL), (dict(T=2 ** 20 + 1), L.MOE_ESHAPE), (dict(T=2 ** 62), L.MOE_ESHAPE),
    (dict(T=2 ** 20, d_ff=2 ** 13), L.MOE_ESHAPE)])
def test_experts_cfg_refused(kw, status):
    c = wcfg(**kw)
    assert experts(c, ws=1 << 40) == status and L.moe_last_error()
    assert L.moe_experts_w4_workspace_bytes(c) == 0


@no_device
def test_experts_pointers_and_workspace():
    c = wcfg()
    need = L.moe_experts_w4_workspace_bytes(c)
    assert experts(c) == L.MOE_EDEVICE and experts(c, ws=need - 1) == L.MOE_EWORKSPACE
    assert experts(c, ws_ptr=None) == L.MOE_EWORKSPACE and experts(c, ws_ptr=P(20) + 8) == L.MOE_EALIGN
    for n in ("x", "idx", "w", "W1c", "W1s", "W2c", "W2s", "y"):
        assert experts(c, **{n: None}) == L.MOE_EINVAL and n in L.moe_last_error()
    assert experts(c, W2s=P(6) + 2) == L.MOE_EALIGN
    assert experts(wcfg(T=0), ws=0, x=None, idx=None, w=None, y=None, ws_ptr=None) == L.MOE_EDEVICE


@pytest.mark.parametrize("k,E,dtype", [(1, 1, "bf16"), (2, 16, "bf16"), (8, 160, "f32"), (16, 512, "bf16")])
def test_experts_workspace_of_a_longer_batch_serves_a_shorter_one(k, E, dtype):
    need = [L.moe_experts_w4_workspace_bytes(L.make_w4_cfg(T, 1024, 512, E, k, dtype)) for T in range(0, 2100)]
    assert all(a <= b for a, b in zip(need, need[1:])) and need[1] > 0


@no_device
def test_quantize_refused():
    q = lib.moe_w4_quantize
    assert q(4, 64, 1, P(0), P(1), P(2), None) == L.MOE_EDEVICE
    assert q(0, 64, 1, None, None, None, None) == L.MOE_EDEVICE
    assert q(4, 48, 1, P(0), P(1), P(2), None) == L.MOE_ESHAPE and q(4, 0, 1, P(0), P(1), P(2), None) == L.MOE_ESHAPE
    assert q(-1, 64, 1, P(0), P(1), P(2), None) == L.MOE_EINVAL and q(4, 64, 2, P(0), P(1), P(2), None) == L.MOE_EDTYPE
    assert q(2 ** 40, 64, 1, P(0), P(1), P(2), None) == L.MOE_ESHAPE
    assert q(4, 64, 1, None, P(1), P(2), None) == L.MOE_EINVAL and q(4, 64, 1, P(0), P(1), P(1), None) == L.MOE_EINVAL
    assert q(4, 64, 1, P(0), P(1) + 8, P(2), None) == L.MOE_EALIGN


def ccfg(**kw):
    base = dict(T=64, d_model=128, d_ff=256, E=4, k=2, C=40)
    base.update(kw)
    return L.make_cfg(**base)


@no_device
def test_ckpt_refused():
    c = ccfg()
    need = L.moe_ckpt_bytes(c)
    # 4 experts x 3 row blocks x (2 + 4 + 2) units of 1024 codes and 16 floats
    assert need == 4 * 3 * 8 * (1024 + 64)
    assert L.moe_ckpt_bytes(ccfg(d_model=72)) == 0 and L.moe_ckpt_bytes(ccfg(d_model=72, d_ff=8, dtype="f32")) > 0
    R = ctypes.byref(c)
    save = lambda s=P(0), h=P(1), o=P(2), rb=None, re=P(4), ck=P(5), n=need: lib.moe_ckpt_save(R, s, h, o, rb, re, ck, n, None)  # noqa: E731
    assert save() == L.MOE_EDEVICE and save(s=None, o=None, rb=P(6)) == L.MOE_EDEVICE
    assert save(n=need - 1) == L.MOE_EWORKSPACE and save(re=None) == L.MOE_EINVAL and save(ck=None) == L.MOE_EINVAL
    assert save(ck=P(1)) == L.MOE_EINVAL and save(h=P(1) + 8) == L.MOE_EALIGN and save(rb=P(3) + 4) == L.MOE_EALIGN
    load = lambda s=P(0), h=P(1), a=P(2), o=P(3), rb=None, re=P(4), ck=P(5), n=need: lib.moe_ckpt_load(R, ck, n, rb, re, s, h, a, o, None)  # noqa: E731
    assert load() == L.MOE_EDEVICE and load(s=None, h=None, o=None) == L.MOE_EDEVICE
    assert load(n=0) == L.MOE_EWORKSPACE and load(a=P(1)) == L.MOE_EINVAL and load(o=P(5)) == L.MOE_EINVAL
    assert load(re=None) == L.MOE_EINVAL and load(a=P(2) + 4) == L.MOE_EALIGN
    assert lib.moe_ckpt_load(ctypes.byref(ccfg(C=0)), P(5), need, None, P(4), P(0), P(1), P(2), P(3), None) == L.MOE_EINVAL


def test_binding_refuses_host_short_and_mistyped_tensors():
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        e = lambda n, dt: torch.empty(n, dtype=dt, device="cuda")   # noqa: E731
        lg, idx, w = e(64 * 16, torch.float32), e(128, torch.int32), e(128, torch.float32)
        x, u8 = e(8 * 64, torch.bfloat16), e(10, torch.uint8)
        nc = e((4, 6, 64), torch.bfloat16).transpose(0, 1)
    r = rcfg()
    with pytest.raises(ValueError, match="logits must be torch.float32"):
        L.moe_route(r, idx, None, idx, w, stream=0)
    with pytest.raises(ValueError, match="logits has 128 elements, the call touches 1024"):
        L.moe_route(r, w, None, idx, w, stream=0)
    with pytest.raises(ValueError, match="idx must be a device tensor"):
        L.moe_route(r, lg, None, torch.zeros(128, dtype=torch.int32), w, stream=0)
    with pytest.raises(ValueError, match="load has 10 elements|load must be"):
        L.moe_route(r, lg, None, idx, w, u8, stream=0)
    with pytest.raises(TypeError, match="moe_route_cfg"):
        L.moe_route(wcfg(), lg, None, idx, w, stream=0)
    with pytest.raises(ValueError, match="dw has"):
        L.moe_route_bwd(rcfg(k=4), lg, lg.view(torch.int32), lg, w, lg, stream=0)
    with pytest.raises(ValueError, match="W1c has 10 elements"):
        L.moe_experts_w4(wcfg(), x, idx, w, u8, u8, u8, u8, x, u8, stream=0)
    with pytest.raises(ValueError, match="W must be contiguous"):
        L.moe_w4_quantize(nc, u8, u8, stream=0)
    with pytest.raises(ValueError, match="W must be torch.float32"):
        L.moe_w4_quantize(idx.view(4, 32), u8, u8, stream=0)
    with pytest.raises(ValueError, match="ckpt has 10 elements"):
        L.moe_ckpt_save(ccfg(), None, None, None, None, idx, u8, stream=0)
    with pytest.raises(ValueError, match="ckpt is required"):
        L.moe_ckpt_load(ccfg(), None, None, idx, None, None, None, None, stream=0)
    with pytest.raises(ValueError, match="not a multiple of 32"):
        L.alloc_w4(4, 40)
