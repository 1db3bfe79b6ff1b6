"""Refusals of the sorted rows and the token lookup, and pins of their oracle (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")
from oracle import training_oracle as O  # noqa: E402

GOOD = 4096   # an aligned address that validation never reads


def _ptrs(n):
    """Different aligned addresses (no output aliases another array)."""
    return [GOOD * (i + 1) for i in range(n)]


def _sorted(**kw):
    base = dict(T=100, d_model=128, d_ff=256, E=8, k=2, dtype="bf16", act="relu", wpacked=0)
    base.update(kw)
    return L.make_sorted_cfg(**base)


BAD = [(dict(T=-1), L.MOE_EINVAL), (dict(T=1 << 31), L.MOE_ESHAPE), (dict(E=0), L.MOE_ESHAPE), (dict(E=513), L.MOE_ESHAPE),
       (dict(k=0), L.MOE_EINVAL), (dict(k=17), L.MOE_EINVAL), (dict(d_model=96), L.MOE_ESHAPE), (dict(d_ff=0), L.MOE_ESHAPE),
       (dict(d_model=12, dtype="f32"), L.MOE_ESHAPE), (dict(dtype=3), L.MOE_EDTYPE), (dict(act=9), L.MOE_EINVAL),
       (dict(wpacked=2), L.MOE_EINVAL), (dict(T=1 << 28, d_model=1 << 20), L.MOE_ESHAPE)]


@pytest.mark.parametrize("kw,status", BAD)
def test_sorted_sizes_are_refused(kw, status):
    c = _sorted(**kw)
    assert L._lib.moe_sorted_rows(c) == -1 and L.moe_last_error()
    p = _ptrs(12)
    assert L._lib.moe_sorted_dispatch(c, *p[:8], 1 << 30, None) == status
    assert L._lib.moe_sorted_ffn_fwd(c, *p[:9], 1 << 30, None) == status
    assert L._lib.moe_sorted_combine(c, *p[:4], None) == status
    assert L._lib.moe_sorted_combine_bwd(c, *p[:7], None) == status
    assert L._lib.moe_sorted_bwd_dx(c, *p[:9], 1 << 30, None) == status
    assert L._lib.moe_sorted_dispatch_bwd(c, *p[:5], None) == status
    assert L._lib.moe_sorted_bwd_dw(c, *p[:12], 1 << 30, None) == status


# (call, arguments before the workspace size or the stream, index of each output, has a workspace)
CALLS = [("moe_sorted_dispatch", 8, [2, 3, 4, 5, 6], True), ("moe_sorted_ffn_fwd", 9, [5, 6, 7], True),
         ("moe_sorted_combine", 4, [3], False), ("moe_sorted_combine_bwd", 7, [5, 6], False),
         ("moe_sorted_bwd_dx", 9, [6, 7], True), ("moe_sorted_dispatch_bwd", 5, [4], False),
         ("moe_sorted_bwd_dw", 12, [6, 7, 10], True)]


@pytest.mark.parametrize("name,n,outs,ws", CALLS)
def test_sorted_pointers_are_refused(name, n, outs, ws):
    c, fn = _sorted(T=5000), getattr(L._lib, name)
    tail = [1 << 30, None] if ws else [None]
    arrays = n - 1 if ws else n
    optional = {"moe_sorted_dispatch_bwd": [2, 3], "moe_sorted_bwd_dw": [8, 9, 10]}.get(name, [])
    for i in range(arrays):
        p = _ptrs(n)
        p[i] = None
        assert fn(c, *p, *tail) == L.MOE_EINVAL, i     # missing, or one of a pair missing
        p = _ptrs(n)
        p[i] += 4
        assert fn(c, *p, *tail) == L.MOE_EALIGN, i
    for o in outs:
        for i in range(arrays):
            if i != o:
                p = _ptrs(n)
                p[o] = p[i]
                assert fn(c, *p, *tail) == L.MOE_EINVAL, (o, i)
    if ws:
        p = _ptrs(n)
        p[n - 1] = None
        assert fn(c, *p, *tail) == L.MOE_EWORKSPACE
        assert fn(c, *_ptrs(n), 8, None) == L.MOE_EWORKSPACE
    assert fn(None, *_ptrs(n), *tail) == L.MOE_EINVAL
    if not torch.cuda.is_available():      # all in order but for the device
        assert fn(c, *_ptrs(n), *tail) == L.MOE_EDEVICE
        p = _ptrs(n)
        for i in optional:
            p[i] = None
        assert fn(c, *p, *tail) == L.MOE_EDEVICE


def test_products_past_two_gib_are_refused_and_rows_are_not():
    c = _sorted(T=1 << 17, k=8, d_model=1024, d_ff=1024)     # 2^20 rows of 1024: 2 GiB
    p = _ptrs(12)
    assert L._lib.moe_sorted_ffn_fwd(c, *p[:9], 1 << 30, None) == L.MOE_ESHAPE
    assert L._lib.moe_sorted_bwd_dx(c, *p[:9], 1 << 30, None) == L.MOE_ESHAPE
    assert L._lib.moe_sorted_bwd_dw(c, *p[:12], 1 << 30, None) == L.MOE_ESHAPE
    assert L._lib.moe_sorted_rows(c) == (1 << 20) + 15 * 8 + 8
    assert L._lib.moe_sorted_ffn_fwd(_sorted(d_model=32768, d_ff=32768), *p[:9], 1 << 30, None) == L.MOE_ESHAPE


def test_gate_gradient_takes_up_to_64_experts():
    p = _ptrs(12)
    assert L._lib.moe_sorted_bwd_dw(_sorted(E=65), *p, 1 << 30, None) == L.MOE_ESHAPE


def test_rows_and_workspaces():
    assert L.moe_sorted_rows(_sorted(T=0)) == 0
    assert L.moe_sorted_rows(_sorted(T=1, E=512, k=1)) == 16
    assert L.moe_sorted_rows(_sorted(T=1000, dtype="f32")) == 2000
    assert L.moe_sorted_workspace_bytes(_sorted(T=512), L.MOE_CALL_DISPATCH) == 0
    assert L.moe_sorted_workspace_bytes(_sorted(T=513), L.MOE_CALL_DISPATCH) > 0
    assert L.moe_sorted_workspace_bytes(_sorted(), L.MOE_CALL_DISPATCH_BPR) == 0 and L.moe_last_error()


def _embed(**kw):
    base = dict(T=100, V=1000, d_model=64, dtype="bf16", scale=1.0, accum=0)
    base.update(kw)
    return L.make_embed_cfg(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), L.MOE_EINVAL), (dict(T=1 << 31), L.MOE_ESHAPE), (dict(V=0), L.MOE_ESHAPE), (dict(V=(1 << 30) + 1), L.MOE_ESHAPE),
    (dict(d_model=0), L.MOE_ESHAPE), (dict(d_model=20), L.MOE_ESHAPE), (dict(V=1 << 30, d_model=2048), L.MOE_ESHAPE),
    (dict(dtype=2), L.MOE_EDTYPE), (dict(scale=float("inf")), L.MOE_EINVAL), (dict(scale=float("nan")), L.MOE_EINVAL),
    (dict(accum=2), L.MOE_EINVAL)])
def test_embed_sizes_are_refused(kw, status):
    c, p = _embed(**kw), _ptrs(4)
    assert L._lib.moe_embed(c, *p[:3], None) == status
    assert L._lib.moe_embed_bwd(c, *p, 1 << 40, None) == status
    assert L.moe_embed_bwd_workspace_bytes(c) == 0 and L.moe_last_error()


def test_embed_pointers_are_refused():
    c = _embed()
    for i in range(3):
        p = _ptrs(4)
        p[i] = None
        assert L._lib.moe_embed(c, *p[:3], None) == L.MOE_EINVAL
        assert L._lib.moe_embed_bwd(c, *p, 1 << 30, None) == L.MOE_EINVAL
        p[i] = GOOD * 50 + 8
        assert L._lib.moe_embed(c, *p[:3], None) == L.MOE_EALIGN
        assert L._lib.moe_embed_bwd(c, *p, 1 << 30, None) == L.MOE_EALIGN
    for o, i in ((2, 0), (2, 1), (3, 0), (3, 1), (3, 2)):
        p = _ptrs(4)
        p[o] = p[i]
        assert L._lib.moe_embed_bwd(c, *p, 1 << 30, None) == L.MOE_EINVAL
    assert L._lib.moe_embed_bwd(c, *_ptrs(4), 16, None) == L.MOE_EWORKSPACE
    assert L._lib.moe_embed_bwd(c, *_ptrs(3), None, 0, None) == L.MOE_EWORKSPACE


def test_binding_checks_tensors():
    c = _embed(dtype="f32")
    t = torch.zeros(1000, 64)
    with pytest.raises(ValueError, match="device tensor"):
        L.moe_embed(c, torch.zeros(100, dtype=torch.int32), t, t)
    with pytest.raises(TypeError, match="moe_embed_cfg"):
        L.moe_embed(_sorted(), torch.zeros(100, dtype=torch.int32), t, t)
    with pytest.raises(TypeError, match="moe_sorted_cfg"):
        L.moe_sorted_combine(c, t, t, t, t)
    assert ctypes.sizeof(L.moe_sorted_cfg) == 40 and ctypes.sizeof(L.moe_embed_cfg) == 32


def test_oracle_sort_by_hand():
    idx = np.array([[2, 0], [0, -1], [2, 2], [9, 0]], np.int32)
    b, e, slot, src = O.sort_rows(idx, 3, "f32")
    assert b.tolist() == [0, 3, 3] and e.tolist() == [3, 3, 6]
    assert slot.tolist() == [[3, 0], [1, -1], [4, 5], [-1, 2]]
    assert src.tolist() == [1, 2, 7, 0, 4, 5, -1, -1]
    b, e, slot, src = O.sort_rows(idx, 3, "bf16")
    assert b.tolist() == [0, 16, 16] and e.tolist() == [3, 16, 19] and slot[2].tolist() == [17, 18] and len(src) == 64


@pytest.mark.parametrize("name", ["relu", "gelu_tanh", "gelu_erf", "identity"])
def test_oracle_expert_against_differences(name):
    torch.manual_seed(0)
    x, W1, W2, dO = (torch.randn(*s, dtype=torch.float64) for s in ((5, 4), (6, 4), (4, 6), (5, 4)))
    got = O.expert(x, W1, W2, name, dO)
    f = lambda: float((dO * O.expert(x, W1, W2, name)["O"][0]).sum())   # noqa: E731
    for m, key in ((x, "dX"), (W1, "dW1"), (W2, "dW2")):
        for i in ((0, 0), (3, 2)):
            was, h = float(m[i]), 1e-6
            m[i] = was + h
            up = f()
            m[i] = was - h
            slope = (up - f()) / (2 * h)
            m[i] = was
            assert abs(slope - float(got[key][0][i])) <= 1e-6 * (1 + abs(slope))


def test_oracle_layout_is_the_header_s():
    m = torch.arange(32 * 64).view(32, 64)
    flat = O.blocked(m).reshape(-1)
    for r, c in ((0, 0), (5, 33), (17, 2), (31, 63)):
        assert int(flat[((r // 16) * 2 + c // 32) * 512 + (r % 16) * 32 + c % 32]) == r * 64 + c
    assert torch.equal(O.unblocked(O.blocked(m)), m)


def _xent(**kw):
    base = dict(T=100, V=1000, d_model=128, dtype="bf16")
    base.update(kw)
    return L.make_xent_cfg(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), L.MOE_EINVAL), (dict(T=1 << 30), L.MOE_ESHAPE), (dict(T=1 << 22), L.MOE_ESHAPE), (dict(V=0), L.MOE_ESHAPE),
    (dict(T=1 << 20, V=(1 << 22) + 1), L.MOE_ESHAPE), (dict(V=(1 << 30) + 1), L.MOE_ESHAPE), (dict(V=1 << 30, d_model=2048), L.MOE_ESHAPE), (dict(d_model=96), L.MOE_ESHAPE),
    (dict(d_model=12, dtype="f32"), L.MOE_ESHAPE), (dict(d_model=1 << 21), L.MOE_ESHAPE), (dict(dtype=2), L.MOE_EDTYPE)])
def test_xent_sizes_are_refused(kw, status):
    c, p = _xent(**kw), _ptrs(8)
    assert L._lib.moe_xent(c, *p[:6], 1 << 40, None) == status
    assert L._lib.moe_xent_bwd(c, *p, 1 << 40, None) == status
    for b in (0, 1):
        assert L.moe_xent_workspace_bytes(c, b) == 0 and L.moe_last_error()


def test_xent_pointers_are_refused():
    c = _xent()
    for n, fn, optional in ((6, L._lib.moe_xent, ()), (8, L._lib.moe_xent_bwd, (5, 6))):
        for i in range(n - 1):
            p = _ptrs(n)
            p[i] += 4
            assert fn(c, *p, 1 << 40, None) == L.MOE_EALIGN, i
            p[i] = None
            if i not in optional:
                assert fn(c, *p, 1 << 40, None) == L.MOE_EINVAL, i
        for o in ((3, 4, 5) if n == 6 else (5, 6, 7)):
            for i in range(o):
                p = _ptrs(n)
                p[o] = p[i]
                assert fn(c, *p, 1 << 40, None) == L.MOE_EINVAL, (o, i)
        assert fn(c, *_ptrs(n), 1024, None) == L.MOE_EWORKSPACE
        assert fn(c, *_ptrs(n - 1), None, 0, None) == L.MOE_EWORKSPACE
        assert fn(None, *_ptrs(n), 1 << 40, None) == L.MOE_EINVAL
    p = _ptrs(8)
    p[5] = p[6] = None
    assert L._lib.moe_xent_bwd(c, *p, 1 << 40, None) == L.MOE_EINVAL
    if not torch.cuda.is_available():
        for i in (5, 6):
            p = _ptrs(8)
            p[i] = None
            assert L._lib.moe_xent_bwd(c, *p, 1 << 40, None) == L.MOE_EDEVICE
    with pytest.raises(TypeError, match="moe_xent_cfg"):
        L.moe_xent(_embed(), *[torch.zeros(1)] * 6)


def test_xent_workspaces_stay_small():
    """Beside copies of x and of a piece of W, the forward keeps an eighth of a byte for each
    logit, and the backward never holds the whole vocabulary's gradient of many tokens."""
    c = _xent(T=16384, V=50257, d_model=2048)
    assert L.moe_xent_workspace_bytes(c, 0) <= 16384 * (50257 / 8 + 2 * 128) + 16384 * 2048 * 2 + (128 << 20)
    assert L.moe_xent_workspace_bytes(c, 1) <= (512 << 20) + 16384 * 2048 * (4 + 2 + 2) + (64 << 20) + 65536
    assert L.moe_xent_workspace_bytes(_xent(T=0), 1) == 0


@pytest.mark.parametrize("T,V,d", [(3, 5, 4), (6, 2, 3)])
def test_oracle_xent_against_differences(T, V, d):
    torch.manual_seed(0)
    x, W, dloss = (torch.randn(*s, dtype=torch.float64) for s in ((T, d), (V, d), (T,)))
    target = torch.randint(0, V, (T,))
    target[0] = -1
    got = O.xent(x, W, target, dloss)
    assert torch.allclose(got["lse"][0], torch.logsumexp(x @ W.t(), 1)) and float(got["loss"][0][0]) == 0
    f = lambda: float((dloss * O.xent(x, W, target)["loss"][0]).sum())   # noqa: E731
    for m, key in ((x, "dx"), (W, "dW")):
        for i in ((0, 0), (1, 2)):
            was, h = float(m[i]), 1e-6
            m[i] = was + h
            up = f()
            m[i] = was - h
            slope = (up - f()) / (2 * h)
            m[i] = was
            assert abs(slope - float(got[key][0][i])) <= 1e-6 * (1 + abs(slope))


def test_oracle_embed_by_hand():
    ids = torch.tensor([2, -1, 0, 2, 3], dtype=torch.int32)
    dy = torch.arange(10.0).view(5, 2)
    dW, _ = O.embed_bwd(ids, dy, 3, 2.0)
    assert dW.tolist() == [[8.0, 10.0], [0.0, 0.0], [12.0, 16.0]]
    y, _ = O.embed(ids, torch.tensor([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]]), 0.5)
    assert y.tolist() == [[2.5, 3.0], [0.0, 0.0], [0.5, 1.0], [2.5, 3.0], [0.0, 0.0]]
