"""Python binding of liblancet_moe.so (ctypes).

Argument marshalling only: every function here has the name of the C-ABI
entry point it calls, checks that each tensor is a contiguous device tensor
of the right dtype and at least the size the call will touch (the C ABI takes
bare pointers and cannot check sizes), and passes pointers and the current
HIP stream; the calls of a step do this in native code (csrc/bind.cpp).  All
computation happens in the HIP kernels.  There is no CPU fallback: if the
library or its binding is missing, importing this module raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
#: The in-tree build; LANCET_MOE_LIB may name another build of the same library.
LIB_PATH = os.environ.get("LANCET_MOE_LIB") or os.path.join(_HERE, "liblancet_moe.so")

MOE_OK, MOE_EINVAL, MOE_ESHAPE, MOE_EALIGN, MOE_EDTYPE, MOE_EDEVICE, MOE_ELAUNCH, MOE_EWORKSPACE = 0, -1, -2, -3, -4, -5, -6, -7
MOE_F32, MOE_BF16 = 0, 1
ACTS = {"identity": 0, "relu": 1, "gelu_tanh": 2, "gelu_erf": 3}
SCORES = {"softmax": 0, "sigmoid": 1}
MOE_CALL_DISPATCH, MOE_CALL_BWD_DX, MOE_CALL_BWD_DW, MOE_CALL_FFN_FWD, MOE_CALL_DISPATCH_BPR = 0, 1, 2, 3, 4

#: Every symbol include/lancet_moe.h declares.
EXPORTS = ["moe_capacity", "moe_workspace_bytes", "moe_last_error", "moe_gate_topk", "moe_dispatch",
           "moe_dispatch_noalloc", "moe_dispatch_bpr", "moe_pack_weights", "moe_expert_ffn_fwd", "moe_combine", "moe_bwd_dx", "moe_bwd_dw",
           "moe_block_workspace_bytes", "moe_block_chunked", "moe_block_op_times", "moe_block_dw_schedule",
           "moe_dw_schedule", "moe_pipeline_plan", "moe_pipeline_range_cost", "moe_product_timing",
           "moe_product_times", "moe_route", "moe_route_bwd", "moe_dispatch_bpr_route", "moe_bwd_dx_route", "moe_w4_quantize",
           "moe_experts_w4_workspace_bytes", "moe_experts_w4", "moe_ckpt_bytes", "moe_ckpt_save", "moe_ckpt_load",
           "moe_sorted_rows", "moe_sorted_workspace_bytes", "moe_sorted_dispatch", "moe_sorted_ffn_fwd", "moe_sorted_combine",
           "moe_sorted_combine_bwd", "moe_sorted_bwd_dx", "moe_sorted_dispatch_bwd", "moe_sorted_bwd_dw", "moe_embed",
           "moe_embed_bwd_workspace_bytes", "moe_embed_bwd", "moe_xent_workspace_bytes", "moe_xent", "moe_xent_bwd"]
#: The expert products moe_product_times reports, in its order.
PRODUCTS = ["fwd1", "fwd2", "dA", "dXe", "dW2", "dW1"]
#: Experts and choices that the gate (moe_gate_topk) takes; moe_route and the moe_sorted_* calls take 512 and 16.
GATE_MAX_E, GATE_MAX_K = 64, 8
MOE_BLOCK_FWD, MOE_BLOCK_BWD, MOE_BLOCK_TIMED = 1, 2, 4
#: The block backward's operations (moe_block_op): the chain 0..7, the weight-gradient groups 8..13.
BLOCK_OPS = ["combine_bwd", "expert_dx", "dispatch_bwd", "ln2_bwd", "dattn", "attn_bwd", "da", "ln1_bwd",
             "dw_expert", "dwg", "dln2", "dwo", "dwqkv", "dln1"]
MOE_BOP_DW_EXPERT = 8


class MoeError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"status {status}: {msg}")
        self.status = status


class moe_cfg(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32),
                ("E", ctypes.c_int32), ("k", ctypes.c_int32), ("C", ctypes.c_int32), ("G", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("renorm", ctypes.c_int32),
                ("wpacked", ctypes.c_int32), ("ksplit", ctypes.c_int32)]


class moe_block_cfg(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("S", ctypes.c_int32), ("heads", ctypes.c_int32), ("moe", moe_cfg),
                ("dw_order", ctypes.c_int32 * 6)]


class moe_route_cfg(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("E", ctypes.c_int32), ("k", ctypes.c_int32), ("score", ctypes.c_int32),
                ("renorm", ctypes.c_int32), ("groups", ctypes.c_int32), ("top_groups", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class moe_w4_cfg(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("E", ctypes.c_int32),
                ("k", ctypes.c_int32), ("dtype", ctypes.c_int32), ("act", ctypes.c_int32)]


class moe_sorted_cfg(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("E", ctypes.c_int32),
                ("k", ctypes.c_int32), ("dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("wpacked", ctypes.c_int32)]


class moe_embed_cfg(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("V", ctypes.c_int32), ("d_model", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("accum", ctypes.c_int32)]


class moe_xent_cfg(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("V", ctypes.c_int32), ("d_model", ctypes.c_int32), ("dtype", ctypes.c_int32)]


BLOCK_WEIGHTS = ["ln1_g", "ln1_b", "Wqkv", "Wo", "ln2_g", "ln2_b", "Wg", "W1", "W2"]
BLOCK_GRADS = ["dln1_g", "dln1_b", "dWqkv", "dWo", "dln2_g", "dln2_b", "dWg", "dW1", "dW2"]
BLOCK_ACTS_FWD = ["a", "ln1_mean", "ln1_rstd", "qkv", "attn", "lse", "h", "ln2_mean", "ln2_rstd", "m", "logits",
                  "idx", "w", "slot", "fill", "send_buf", "H", "A", "expert_out", "W1p", "W2p"]
BLOCK_ACTS_BWD = ["dO", "dH", "dXe", "dlogits", "dm", "dh", "dattn", "delta", "dqkv", "da"]


class moe_block_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in BLOCK_WEIGHTS]


class moe_block_grads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in BLOCK_GRADS]


class moe_block_acts(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in BLOCK_ACTS_FWD + BLOCK_ACTS_BWD]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2404_19429_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    CFG, SORTED, EMBED, XENT = (ctypes.POINTER(t) for t in (moe_cfg, moe_sorted_cfg, moe_embed_cfg, moe_xent_cfg))
    sig = {
        "moe_capacity": (I32, [I64, I32, I32, I32, I32]),
        "moe_workspace_bytes": (SZ, [CFG, I32]),
        "moe_last_error": (ctypes.c_char_p, []),
        "moe_gate_topk": (I32, [CFG, P, P, P, P, P, P, P]),
        "moe_dispatch": (I32, [CFG, P, P, P, P, P, P, P, SZ, P]),
        "moe_dispatch_noalloc": (I32, [CFG, P, P, P, P, P, P, P]),
        "moe_dispatch_bpr": (I32, [CFG, P, P, P, P, P, P, P, P, SZ, P]),
        "moe_pack_weights": (I32, [CFG, P, P, P, P, P]),
        "moe_expert_ffn_fwd": (I32, [CFG, P, P, P, P, P, P, P, P, P, SZ, P]),
        "moe_combine": (I32, [CFG, P, P, P, P, P, P]),
        "moe_bwd_dx": (I32, [CFG] + [P] * 18 + [SZ, P]),
        "moe_bwd_dw": (I32, [CFG] + [P] * 12 + [SZ, P]),
        "moe_dw_schedule": (I32, [I32, P, P, I32, P, P, P, P, P]),
        "moe_block_op_times": (I32, [P]),
        "moe_product_timing": (I32, [I32]),
        "moe_product_times": (I32, [P, P]),
        "moe_block_dw_schedule": (I32, [P, ctypes.c_double, P, P, P]),
        "moe_pipeline_plan": (I32, [I32, I32, P, P, P, I32, P, P, P, P, P]),
        "moe_pipeline_range_cost": (I32, [I32, I32, P, P, P, I32, I32, I32, P]),
        "moe_route": (I32, [ctypes.POINTER(moe_route_cfg)] + [P] * 6),
        "moe_route_bwd": (I32, [ctypes.POINTER(moe_route_cfg)] + [P] * 6),
        "moe_dispatch_bpr_route": (I32, [CFG, ctypes.POINTER(moe_route_cfg)] + [P] * 8 + [SZ, P]),
        "moe_bwd_dx_route": (I32, [CFG, ctypes.POINTER(moe_route_cfg)] + [P] * 19 + [SZ, P]),
        "moe_w4_quantize": (I32, [I64, I32, I32, P, P, P, P]),
        "moe_experts_w4_workspace_bytes": (SZ, [ctypes.POINTER(moe_w4_cfg)]),
        "moe_experts_w4": (I32, [ctypes.POINTER(moe_w4_cfg)] + [P] * 9 + [SZ, P]),
        "moe_ckpt_bytes": (SZ, [CFG]),
        "moe_ckpt_save": (I32, [CFG] + [P] * 6 + [SZ, P]),
        "moe_ckpt_load": (I32, [CFG, P, SZ] + [P] * 7),
        "moe_sorted_rows": (I64, [SORTED]),
        "moe_sorted_workspace_bytes": (SZ, [SORTED, I32]),
        "moe_sorted_dispatch": (I32, [SORTED] + [P] * 8 + [SZ, P]),
        "moe_sorted_ffn_fwd": (I32, [SORTED] + [P] * 9 + [SZ, P]),
        "moe_sorted_combine": (I32, [SORTED] + [P] * 5),
        "moe_sorted_combine_bwd": (I32, [SORTED] + [P] * 8),
        "moe_sorted_bwd_dx": (I32, [SORTED] + [P] * 9 + [SZ, P]),
        "moe_sorted_dispatch_bwd": (I32, [SORTED] + [P] * 6),
        "moe_sorted_bwd_dw": (I32, [SORTED] + [P] * 12 + [SZ, P]),
        "moe_embed": (I32, [EMBED] + [P] * 4),
        "moe_embed_bwd_workspace_bytes": (SZ, [EMBED]),
        "moe_embed_bwd": (I32, [EMBED] + [P] * 4 + [SZ, P]),
        "moe_xent_workspace_bytes": (SZ, [XENT, I32]),
        "moe_xent": (I32, [XENT] + [P] * 6 + [SZ, P]),
        "moe_xent_bwd": (I32, [XENT] + [P] * 8 + [SZ, P]),
        "moe_block_workspace_bytes": (SZ, [ctypes.POINTER(moe_block_cfg), I32]),
        "moe_block_chunked": (I32, [ctypes.POINTER(moe_block_cfg), ctypes.POINTER(moe_block_weights),
                                    ctypes.POINTER(moe_block_grads), P, P, P, P, ctypes.POINTER(moe_block_acts),
                                    I32, I32, ctypes.POINTER(P), P, SZ]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


_lib = _load()


def _load_bind():
    try:
        from paper_2404_19429_amd import _bind
    except ImportError as e:
        raise ImportError("the native binding is not built; run `python -m paper_2404_19429_amd.build`") from e
    _bind.init({n: ctypes.cast(getattr(_lib, n), ctypes.c_void_p).value for n in EXPORTS}, lambda s: _stream(s),
               moe_cfg, moe_block_cfg, moe_route_cfg, moe_w4_cfg, moe_sorted_cfg, moe_embed_cfg, moe_xent_cfg)
    return _bind


_bind = _load_bind()


# ----------------------------------------------------------------------- helpers
def make_cfg(T, d_model, d_ff, E, k, C, G=1, dtype="bf16", act="gelu_tanh", renorm=1, wpacked=0,
             ksplit=1) -> moe_cfg:
    dt = {"bf16": MOE_BF16, "f32": MOE_F32}[dtype] if isinstance(dtype, str) else int(dtype)
    return moe_cfg(int(T), int(d_model), int(d_ff), int(E), int(k), int(C), int(G), dt,
                   ACTS[act] if isinstance(act, str) else int(act), int(renorm), int(wpacked), int(ksplit))


def torch_dtype(cfg: moe_cfg):
    return torch.bfloat16 if cfg.dtype == MOE_BF16 else torch.float32


def rows_alloc(cfg: moe_cfg) -> int:
    """Rows per expert of an [E][C][X] buffer: C rounded up to 16 for bf16 (blocked layout), C for float."""
    return (cfg.C + 15) // 16 * 16 if cfg.dtype == MOE_BF16 else cfg.C


def expert_numel(cfg: moe_cfg, X: int) -> int:
    """Elements of an [E][C][X] expert buffer (see the layout note in include/lancet_moe.h)."""
    return cfg.E * rows_alloc(cfg) * X


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _torch_stream(stream) -> torch.cuda.Stream:
    """The torch stream of whatever an entry point takes as its stream (None: the current one)."""
    if isinstance(stream, torch.cuda.Stream):
        return stream
    if stream is None:
        return torch.cuda.current_stream()
    handle = int(stream)
    return torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()


def _wait_for(stream, earlier):
    """What is called on `stream` from here on runs after what is on `earlier` so far."""
    ev = torch.cuda.Event()
    ev.record(_torch_stream(earlier))
    _torch_stream(stream).wait_event(ev)


def _check(st: int):
    if st != MOE_OK:
        raise MoeError(st, _lib.moe_last_error().decode())


# ------------------------------------------------------------------- entry points
def moe_capacity(T: int, E: int, k: int, cf_num: int, cf_den: int) -> int:
    return int(_lib.moe_capacity(T, E, k, cf_num, cf_den))


def moe_workspace_bytes(cfg: moe_cfg, call: int) -> int:
    return int(_lib.moe_workspace_bytes(ctypes.byref(cfg), call))


def moe_last_error() -> str:
    return _lib.moe_last_error().decode()


def moe_gate_topk(cfg, x, Wg, bias, logits, idx, w, stream=None):
    _check(_bind.gate_topk(cfg, x, Wg, bias, logits, idx, w, stream))


def moe_dispatch(cfg, x, idx, carry, fill, slot, send_buf, ws, stream=None):
    _check(_bind.dispatch(cfg, x, idx, carry, fill, slot, send_buf, ws, stream))


def moe_dispatch_noalloc(cfg, x, idx, carry, fill, slot, send_buf, stream=None):
    _check(_bind.dispatch_noalloc(cfg, x, idx, carry, fill, slot, send_buf, stream))


def moe_dispatch_bpr(cfg, x, logits, idx, fill, slot, send_buf, order, ws, stream=None):
    _check(_bind.dispatch_bpr(cfg, x, logits, idx, fill, slot, send_buf, order, ws, stream))


def moe_dw_schedule(kinds, times, edges):
    """Weight-gradient schedule pass on the host (see include/lancet_moe.h).
    kinds: 0 other / 1 all-to-all / 2 weight gradient; times: per instruction;
    edges: (src, dst) pairs.  Returns (assign [n] int32, order [n] int32, overlap)."""
    import numpy as np
    kinds = np.ascontiguousarray(kinds, np.int32)
    times = np.ascontiguousarray(times, np.float64)
    e = np.ascontiguousarray(np.asarray(edges, np.int32).reshape(-1, 2))
    src, dst = np.ascontiguousarray(e[:, 0]), np.ascontiguousarray(e[:, 1])
    n = int(kinds.size)
    assign = np.empty(n, np.int32)
    order = np.empty(n, np.int32)
    ov = ctypes.c_double(0.0)
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p) if a.size else None
    _check(_lib.moe_dw_schedule(n, p(kinds), p(times), int(src.size), p(src), p(dst), p(assign), p(order),
                                ctypes.byref(ov)))
    return assign, order, ov.value


def _pipeline_args(kinds, times, join):
    import numpy as np
    kinds = np.ascontiguousarray(kinds, np.int32)
    times = np.ascontiguousarray(times, np.float64).reshape(kinds.size, -1)
    join = np.ascontiguousarray(join, np.float64)
    assert times.shape[1] == join.size, "times needs one column per k = 1..K"
    p = lambda a: a.ctypes.data_as(ctypes.c_void_p) if a.size else None
    return kinds, times, join, p


def moe_pipeline_plan(kinds, times, join, G=0):
    """Partition-range plan on the host (see include/lancet_moe.h).  times [N][K],
    join [K].  Returns (T(N), [(begin, end, k), ...] 1-based inclusive)."""
    import numpy as np
    kinds, times, join, p = _pipeline_args(kinds, times, join)
    N, K = int(kinds.size), int(join.size)
    b, e, k = (np.zeros(max(N, 1), np.int32) for _ in range(3))
    n_seg, total = ctypes.c_int32(0), ctypes.c_double(0.0)
    _check(_lib.moe_pipeline_plan(N, K, p(kinds), p(times), p(join), int(G), p(b), p(e), p(k), ctypes.byref(n_seg),
                                  ctypes.byref(total)))
    return total.value, [(int(b[q]), int(e[q]), int(k[q])) for q in range(n_seg.value)]


def moe_pipeline_range_cost(kinds, times, join, i, n, k):
    kinds, times, join, p = _pipeline_args(kinds, times, join)
    c = ctypes.c_double(0.0)
    _check(_lib.moe_pipeline_range_cost(int(kinds.size), int(join.size), p(kinds), p(times), p(join), int(i), int(n),
                                        int(k), ctypes.byref(c)))
    return c.value


def moe_pack_weights(cfg, W1, W2, W1p, W2p, stream=None):
    _check(_bind.pack_weights(cfg, W1, W2, W1p, W2p, stream))


def moe_expert_ffn_fwd(cfg, send_buf, row_begin, row_end, W1p, W2p, H, A, expert_out, ws=None, stream=None):
    _check(_bind.expert_ffn_fwd(cfg, send_buf, row_begin, row_end, W1p, W2p, H, A, expert_out, ws, stream))


def moe_combine(cfg, expert_out, idx, slot, w, y, stream=None):
    _check(_bind.combine(cfg, expert_out, idx, slot, w, y, stream))


def moe_bwd_dx(cfg, Wg, logits, idx, w, slot, row_begin, row_end, H, expert_out, W1p, W2p, dy, dO, dH, dXe,
               dlogits, dx, ws=None, stream=None):
    _check(_bind.bwd_dx(cfg, Wg, logits, idx, w, slot, row_begin, row_end, H, expert_out, W1p, W2p, dy, dO, dH, dXe,
                        dlogits, dx, ws, stream))


def moe_bwd_dw(cfg, x, dlogits, row_begin, row_end, send_buf, A, dO, dH, dW1, dW2, dWg, ws, stream=None):
    _check(_bind.bwd_dw(cfg, x, dlogits, row_begin, row_end, send_buf, A, dO, dH, dW1, dW2, dWg, ws, stream))


# ------------------------------------------------------------------------ router
def make_route_cfg(T, E, k, score="softmax", renorm=1, groups=1, top_groups=1, scale=1.0) -> moe_route_cfg:
    return moe_route_cfg(int(T), int(E), int(k), SCORES[score] if isinstance(score, str) else int(score), int(renorm),
                         int(groups), int(top_groups), float(scale))


def moe_route(cfg, logits, bias, idx, w, load=None, stream=None):
    """load: the choices of each expert are added to it."""
    _check(_bind.route(cfg, logits, bias, idx, w, load, stream))


def moe_route_bwd(cfg, logits, idx, w, dw, dlogits, stream=None):
    _check(_bind.route_bwd(cfg, logits, idx, w, dw, dlogits, stream))


def moe_dispatch_bpr_route(cfg, route, x, logits, idx, fill, slot, send_buf, order, ws, stream=None):
    _check(_bind.dispatch_bpr_route(cfg, route, x, logits, idx, fill, slot, send_buf, order, ws, stream))


def moe_bwd_dx_route(cfg, route, Wg, logits, idx, w, slot, row_begin, row_end, H, expert_out, W1p, W2p, dy, dO, dH, dXe,
                     dw, dlogits, dx, ws=None, stream=None):
    _check(_bind.bwd_dx_route(cfg, route, Wg, logits, idx, w, slot, row_begin, row_end, H, expert_out, W1p, W2p, dy, dO,
                              dH, dXe, dw, dlogits, dx, ws, stream))


# --------------------------------------------------------- experts on 4-bit weights
def make_w4_cfg(T, d_model, d_ff, E, k, dtype="bf16", act="gelu_tanh") -> moe_w4_cfg:
    dt = {"bf16": MOE_BF16, "f32": MOE_F32}[dtype] if isinstance(dtype, str) else int(dtype)
    return moe_w4_cfg(int(T), int(d_model), int(d_ff), int(E), int(k), dt, ACTS[act] if isinstance(act, str) else int(act))


def moe_w4_quantize(W, codes, scales, stream=None):
    """W [..., K] (bf16 or f32) -> codes [..., K/2] and scales [..., K/32] (uint8)."""
    if not isinstance(W, torch.Tensor) or W.dim() < 1:
        raise ValueError("W must be a device tensor of at least one dimension")
    K = W.shape[-1]
    _check(_bind.w4_quantize(W.numel() // K if K else 0, K, MOE_BF16 if W.dtype == torch.bfloat16 else MOE_F32, W, codes,
                             scales, stream))


def alloc_w4(*shape, device="cuda"):
    """Empty codes and scales of a weight of `shape` [..., K]."""
    K = shape[-1]
    if K % 32:
        raise ValueError(f"{K} inputs are not a multiple of 32")
    return (torch.empty(*shape[:-1], K // 2, dtype=torch.uint8, device=device),
            torch.empty(*shape[:-1], K // 32, dtype=torch.uint8, device=device))


def moe_experts_w4_workspace_bytes(cfg: moe_w4_cfg) -> int:
    return int(_lib.moe_experts_w4_workspace_bytes(ctypes.byref(cfg)))


def moe_experts_w4(cfg, x, idx, w, W1c, W1s, W2c, W2s, y, ws, stream=None):
    _check(_bind.experts_w4(cfg, x, idx, w, W1c, W1s, W2c, W2s, y, ws, stream))


# ------------------------------------------------------- 8-bit activation checkpoint
def moe_ckpt_bytes(cfg: moe_cfg) -> int:
    return int(_lib.moe_ckpt_bytes(ctypes.byref(cfg)))


def moe_ckpt_save(cfg, send_buf, H, expert_out, row_begin, row_end, ckpt, stream=None):
    _check(_bind.ckpt_save(cfg, send_buf, H, expert_out, row_begin, row_end, ckpt, stream))


def moe_ckpt_load(cfg, ckpt, row_begin, row_end, send_buf, H, A, expert_out, stream=None):
    _check(_bind.ckpt_load(cfg, ckpt, row_begin, row_end, send_buf, H, A, expert_out, stream))


# ------------------------------------------------ rows sorted by expert, no capacity
def _dtype(dtype) -> int:
    return {"bf16": MOE_BF16, "f32": MOE_F32}[dtype] if isinstance(dtype, str) else int(dtype)


def make_sorted_cfg(T, d_model, d_ff, E, k, dtype="bf16", act="gelu_tanh", wpacked=0) -> moe_sorted_cfg:
    return moe_sorted_cfg(int(T), int(d_model), int(d_ff), int(E), int(k), _dtype(dtype),
                          ACTS[act] if isinstance(act, str) else int(act), int(wpacked))


def moe_sorted_rows(cfg: moe_sorted_cfg) -> int:
    return int(_lib.moe_sorted_rows(ctypes.byref(cfg)))


def moe_sorted_workspace_bytes(cfg: moe_sorted_cfg, call: int) -> int:
    return int(_lib.moe_sorted_workspace_bytes(ctypes.byref(cfg), call))


def moe_sorted_dispatch(cfg, x, idx, row_begin, row_end, slot, src, rows, ws, stream=None):
    _check(_bind.sorted_dispatch(cfg, x, idx, row_begin, row_end, slot, src, rows, ws, stream))


def moe_sorted_ffn_fwd(cfg, rows, row_begin, row_end, W1p, W2p, H, A, expert_out, ws=None, stream=None):
    _check(_bind.sorted_ffn_fwd(cfg, rows, row_begin, row_end, W1p, W2p, H, A, expert_out, ws, stream))


def moe_sorted_combine(cfg, expert_out, slot, w, y, stream=None):
    _check(_bind.sorted_combine(cfg, expert_out, slot, w, y, stream))


def moe_sorted_combine_bwd(cfg, expert_out, slot, src, w, dy, dO, dw, stream=None):
    _check(_bind.sorted_combine_bwd(cfg, expert_out, slot, src, w, dy, dO, dw, stream))


def moe_sorted_bwd_dx(cfg, row_begin, row_end, H, W1p, W2p, dO, dH, dXe, ws=None, stream=None):
    _check(_bind.sorted_bwd_dx(cfg, row_begin, row_end, H, W1p, W2p, dO, dH, dXe, ws, stream))


def moe_sorted_dispatch_bwd(cfg, slot, dXe, dx, Wg=None, dlogits=None, stream=None):
    _check(_bind.sorted_dispatch_bwd(cfg, slot, dXe, Wg, dlogits, dx, stream))


def moe_sorted_bwd_dw(cfg, row_begin, row_end, rows, A, dO, dH, dW1, dW2, ws=None, x=None, dlogits=None, dWg=None,
                      stream=None):
    """x, dlogits and dWg together: the gate's weight gradient too (ws is for that)."""
    _check(_bind.sorted_bwd_dw(cfg, row_begin, row_end, rows, A, dO, dH, dW1, dW2, x, dlogits, dWg, ws, stream))


# ------------------------------------------------------------------ token lookup
def make_embed_cfg(T, V, d_model, dtype="bf16", scale=1.0, accum=0) -> moe_embed_cfg:
    return moe_embed_cfg(int(T), int(V), int(d_model), _dtype(dtype), float(scale), int(accum))


def moe_embed(cfg, ids, W, y, stream=None):
    _check(_bind.embed(cfg, ids, W, y, stream))


def moe_embed_bwd_workspace_bytes(cfg: moe_embed_cfg) -> int:
    return int(_lib.moe_embed_bwd_workspace_bytes(ctypes.byref(cfg)))


def moe_embed_bwd(cfg, ids, dy, dW, ws, stream=None):
    _check(_bind.embed_bwd(cfg, ids, dy, dW, ws, stream))


# -------------------------------------------------- cross entropy over a vocabulary
def make_xent_cfg(T, V, d_model, dtype="bf16") -> moe_xent_cfg:
    return moe_xent_cfg(int(T), int(V), int(d_model), _dtype(dtype))


def moe_xent_workspace_bytes(cfg: moe_xent_cfg, backward=False) -> int:
    return int(_lib.moe_xent_workspace_bytes(ctypes.byref(cfg), 1 if backward else 0))


def moe_xent(cfg, x, W, target, loss, lse, ws, stream=None):
    _check(_bind.xent(cfg, x, W, target, loss, lse, ws, stream))


def moe_xent_bwd(cfg, x, W, target, lse, dloss, dx, dW, ws, stream=None):
    """dx or dW None: not wanted."""
    _check(_bind.xent_bwd(cfg, x, W, target, lse, dloss, dx, dW, ws, stream))


# ------------------------------------------------------------- layer step driver
@dataclass
class LayerBuffers:
    """Device tensors of one MoE layer step (allocated once, reused every step)."""
    cfg: moe_cfg
    logits: torch.Tensor
    idx: torch.Tensor
    w: torch.Tensor
    carry: torch.Tensor
    fill: torch.Tensor
    slot: torch.Tensor
    send_buf: torch.Tensor
    H: torch.Tensor
    A: torch.Tensor
    O: torch.Tensor
    y: torch.Tensor
    dO: torch.Tensor
    dH: torch.Tensor
    dXe: torch.Tensor
    dlogits: torch.Tensor
    dx: torch.Tensor
    dW1: torch.Tensor
    dW2: torch.Tensor
    dWg: torch.Tensor
    W1p: torch.Tensor
    W2p: torch.Tensor
    ws_dispatch: torch.Tensor
    ws_ffn: torch.Tensor
    ws_dx: torch.Tensor
    ws_dw: torch.Tensor
    order: torch.Tensor       # batch-prioritized routing: the visiting order
    ws_bpr: torch.Tensor
    dw: Optional[torch.Tensor] = None   # layers with a router: the gradient at w


def alloc_layer(cfg: moe_cfg, device="cuda") -> LayerBuffers:
    dt = torch_dtype(cfg)
    T, d, f, E, k, C = cfg.T, cfg.d_model, cfg.d_ff, cfg.E, cfg.k, cfg.C
    e = lambda *s, dtype=dt: torch.empty(*s, dtype=dtype, device=device)
    nd, nf = expert_numel(cfg, d), expert_numel(cfg, f)
    return LayerBuffers(
        cfg=cfg, logits=e(T, E, dtype=torch.float32), idx=e(T, k, dtype=torch.int32), w=e(T, k, dtype=torch.float32),
        carry=torch.zeros(E, dtype=torch.int32, device=device), fill=e(E, dtype=torch.int32),
        slot=e(T, k, dtype=torch.int32), send_buf=e(nd), H=e(nf), A=e(nf), O=e(nd), y=e(T, d),
        dO=e(nd), dH=e(nf), dXe=e(nd), dlogits=e(T, E, dtype=torch.float32), dx=e(T, d),
        dW1=e(E, f, d), dW2=e(E, d, f), dWg=e(E, d, dtype=torch.float32), W1p=e(E * f * d), W2p=e(E * d * f),
        ws_dispatch=e(max(16, moe_workspace_bytes(cfg, MOE_CALL_DISPATCH)), dtype=torch.uint8),
        ws_ffn=e(max(16, moe_workspace_bytes(cfg, MOE_CALL_FFN_FWD)), dtype=torch.uint8),
        ws_dx=e(max(16, moe_workspace_bytes(cfg, MOE_CALL_BWD_DX)), dtype=torch.uint8),
        ws_dw=e(max(16, moe_workspace_bytes(cfg, MOE_CALL_BWD_DW)), dtype=torch.uint8),
        order=e(max(1, T), dtype=torch.int32),
        ws_bpr=e(max(16, moe_workspace_bytes(cfg, MOE_CALL_DISPATCH_BPR)), dtype=torch.uint8),
        dw=e(T, k, dtype=torch.float32),
    )


@dataclass
class Router:
    """How a layer's choices and weights come from the gate's logits (moe_route), in the place of the gate's own."""
    cfg: moe_route_cfg
    bias: Optional[torch.Tensor] = None    # [E] float, in the choice only
    load: Optional[torch.Tensor] = None    # [E] int32, the choices of each expert are added to it


def layer_forward(b: LayerBuffers, x, Wg, bias, W1, W2, stream=None, routing="token", router: Optional[Router] = None):
    """weight packing -> gate [-> router] -> dispatch -> experts -> combine, all on one stream.
    routing "bpr": batch-prioritized capacity order, by the router's scores if there is one (no carry-in;
    b.carry must be zero)."""
    c = b.cfg
    if router is not None and (router.cfg.T, router.cfg.E, router.cfg.k) != (c.T, c.E, c.k):
        raise ValueError("the router's T, E and k are not the layer's")
    moe_pack_weights(c, W1, W2, b.W1p, b.W2p, stream)
    moe_gate_topk(c, x, Wg, bias, b.logits, b.idx, b.w, stream)
    if router is not None:
        moe_route(router.cfg, b.logits, router.bias, b.idx, b.w, router.load, stream)
    if routing == "bpr" and router is not None:
        moe_dispatch_bpr_route(c, router.cfg, x, b.logits, b.idx, b.fill, b.slot, b.send_buf, b.order, b.ws_bpr, stream)
    elif routing == "bpr":
        moe_dispatch_bpr(c, x, b.logits, b.idx, b.fill, b.slot, b.send_buf, b.order, b.ws_bpr, stream)
    else:
        moe_dispatch(c, x, b.idx, b.carry, b.fill, b.slot, b.send_buf, b.ws_dispatch, stream)
    moe_expert_ffn_fwd(c, b.send_buf, b.carry, b.fill, b.W1p, b.W2p, b.H, b.A, b.O, b.ws_ffn, stream)
    moe_combine(c, b.O, b.idx, b.slot, b.w, b.y, stream)


def alloc_ckpt(cfg: moe_cfg, device="cuda") -> torch.Tensor:
    """An empty checkpoint of one layer's saved activations."""
    return torch.empty(max(16, moe_ckpt_bytes(cfg)), dtype=torch.uint8, device=device)


def layer_save(b: LayerBuffers, ckpt, stream=None):
    """After layer_forward: what its backward reads of the expert buffers, in 8 bits (another layer may then
    use them; the token-sized results, the weights and carry and fill stay the layer's own)."""
    moe_ckpt_save(b.cfg, b.send_buf, b.H, b.O, b.carry, b.fill, ckpt, stream)


def layer_restore(b: LayerBuffers, ckpt, stream=None):
    """Before layer_backward: the expert buffers as layer_save kept them, A from H."""
    moe_ckpt_load(b.cfg, ckpt, b.carry, b.fill, b.send_buf, b.H, b.A, b.O, stream)


def layer_backward(b: LayerBuffers, x, Wg, dy, stream=None, dw_stream=None, router: Optional[Router] = None):
    """dX chain on `stream` (with the weights packed by layer_forward); the dW
    products on `dw_stream` (default: same stream), ordered after the dX chain by an event."""
    c = b.cfg
    if router is not None:
        moe_bwd_dx_route(c, router.cfg, Wg, b.logits, b.idx, b.w, b.slot, b.carry, b.fill, b.H, b.O, b.W1p, b.W2p, dy,
                         b.dO, b.dH, b.dXe, b.dw, b.dlogits, b.dx, b.ws_dx, stream)
    else:
        moe_bwd_dx(c, Wg, b.logits, b.idx, b.w, b.slot, b.carry, b.fill, b.H, b.O, b.W1p, b.W2p, dy, b.dO, b.dH, b.dXe,
                   b.dlogits, b.dx, b.ws_dx, stream)
    if dw_stream is not None:
        _wait_for(dw_stream, stream)
    moe_bwd_dw(c, x, b.dlogits, b.carry, b.fill, b.send_buf, b.A, b.dO, b.dH, b.dW1, b.dW2, b.dWg, b.ws_dw,
               dw_stream if dw_stream is not None else stream)


# ------------------------------------------------- layer step without a capacity
@dataclass
class SortedBuffers:
    """Device tensors of one MoE layer step over sorted rows (allocated once, reused every step)."""
    cfg: moe_sorted_cfg
    gate: moe_cfg             # the gate's sizes (its C plays no part)
    logits: torch.Tensor
    idx: torch.Tensor
    w: torch.Tensor
    row_begin: torch.Tensor
    row_end: torch.Tensor
    slot: torch.Tensor
    src: torch.Tensor
    rows: torch.Tensor
    H: torch.Tensor
    A: torch.Tensor
    O: torch.Tensor
    y: torch.Tensor
    dO: torch.Tensor
    dH: torch.Tensor
    dXe: torch.Tensor
    dw: torch.Tensor
    dlogits: torch.Tensor
    dx: torch.Tensor
    dW1: torch.Tensor
    dW2: torch.Tensor
    dWg: torch.Tensor
    W1p: torch.Tensor
    W2p: torch.Tensor
    ws: torch.Tensor          # of the calls on the layer's stream
    ws_dw: torch.Tensor       # of the weight gradients


def alloc_sorted(cfg: moe_sorted_cfg, renorm=1, device="cuda") -> SortedBuffers:
    """E <= GATE_MAX_E and k <= min(E, GATE_MAX_K), as the gate takes them (MoeError otherwise).  More experts or
    choices: the moe_sorted_* calls themselves, with choices from elsewhere (moe_route)."""
    T, d, f, E, k, R = cfg.T, cfg.d_model, cfg.d_ff, cfg.E, cfg.k, moe_sorted_rows(cfg)
    if R < 0:
        raise MoeError(MOE_ESHAPE, moe_last_error())
    if E > GATE_MAX_E:
        raise MoeError(MOE_ESHAPE, f"alloc_sorted: the step's gate takes up to {GATE_MAX_E} experts, E={E}")
    if k > min(E, GATE_MAX_K):
        raise MoeError(MOE_EINVAL, f"alloc_sorted: the step's gate takes k up to min(E, {GATE_MAX_K}), k={k}")
    gate = make_cfg(T, d, f, E, k, 1, 1, cfg.dtype, cfg.act, renorm, cfg.wpacked)
    dt, f32, i32 = torch_dtype(gate), torch.float32, torch.int32
    e = lambda *s, dtype=dt: torch.empty(*s, dtype=dtype, device=device)
    ws = lambda *calls: e(max(16, *(moe_sorted_workspace_bytes(cfg, c) for c in calls)), dtype=torch.uint8)
    return SortedBuffers(
        cfg=cfg, gate=gate, logits=e(T, E, dtype=f32), idx=e(T, k, dtype=i32), w=e(T, k, dtype=f32),
        row_begin=e(E, dtype=i32), row_end=e(E, dtype=i32), slot=e(T, k, dtype=i32), src=e(R, dtype=i32),
        rows=e(R, d), H=e(R, f), A=e(R, f), O=e(R, d), y=e(T, d), dO=e(R, d), dH=e(R, f), dXe=e(R, d),
        dw=e(T, k, dtype=f32), dlogits=e(T, E, dtype=f32), dx=e(T, d), dW1=e(E, f, d), dW2=e(E, d, f),
        dWg=e(E, d, dtype=f32), W1p=e(E, f, d), W2p=e(E, d, f),
        ws=ws(MOE_CALL_DISPATCH, MOE_CALL_FFN_FWD, MOE_CALL_BWD_DX), ws_dw=ws(MOE_CALL_BWD_DW))


def sorted_layer_forward(b: SortedBuffers, x, Wg, bias, W1, W2, stream=None, router: Optional[Router] = None):
    """layer_forward without a capacity: weight packing -> gate [-> router] -> rows by expert -> experts -> combine.
    No token is dropped, and no buffer is padded to the busiest expert."""
    c = b.cfg
    if router is not None and (router.cfg.T, router.cfg.E, router.cfg.k) != (c.T, c.E, c.k):
        raise ValueError("the router's T, E and k are not the layer's")
    moe_pack_weights(b.gate, W1, W2, b.W1p, b.W2p, stream)
    moe_gate_topk(b.gate, x, Wg, bias, b.logits, b.idx, b.w, stream)
    if router is not None:
        moe_route(router.cfg, b.logits, router.bias, b.idx, b.w, router.load, stream)
    moe_sorted_dispatch(c, x, b.idx, b.row_begin, b.row_end, b.slot, b.src, b.rows, b.ws, stream)
    moe_sorted_ffn_fwd(c, b.rows, b.row_begin, b.row_end, b.W1p, b.W2p, b.H, b.A, b.O, b.ws, stream)
    moe_sorted_combine(c, b.O, b.slot, b.w, b.y, stream)


def sorted_layer_backward(b: SortedBuffers, x, Wg, dy, stream=None, dw_stream=None, router: Optional[Router] = None):
    """The dX chain on `stream` (with the weights packed by sorted_layer_forward); the weight gradients on
    `dw_stream` (default: the same), ordered after it by an event."""
    c = b.cfg
    route = router.cfg if router is not None else make_route_cfg(c.T, c.E, c.k, "softmax", b.gate.renorm)
    moe_sorted_combine_bwd(c, b.O, b.slot, b.src, b.w, dy, b.dO, b.dw, stream)
    moe_route_bwd(route, b.logits, b.idx, b.w, b.dw, b.dlogits, stream)
    moe_sorted_bwd_dx(c, b.row_begin, b.row_end, b.H, b.W1p, b.W2p, b.dO, b.dH, b.dXe, b.ws, stream)
    moe_sorted_dispatch_bwd(c, b.slot, b.dXe, b.dx, Wg, b.dlogits, stream)
    if dw_stream is not None:
        _wait_for(dw_stream, stream)
    moe_sorted_bwd_dw(c, b.row_begin, b.row_end, b.rows, b.A, b.dO, b.dH, b.dW1, b.dW2, b.ws_dw, x, b.dlogits, b.dWg,
                      dw_stream if dw_stream is not None else stream)


# ------------------------------------------------------------------------ block
def make_block_cfg(B, S, heads, d_ff, E, k, C, G=1, act="gelu_tanh", renorm=1, dw_order=None,
                   wpacked=0) -> moe_block_cfg:
    """dw_order: the weight-gradient groups (8..13) in launch order; None = the default order.
    wpacked: 1 = the block's W1, W2 are the packed copies and dW1, dW2 come packed."""
    d = 128 * heads
    order = (ctypes.c_int32 * 6)(*([-1] * 6 if dw_order is None else [int(v) for v in dw_order]))
    return moe_block_cfg(int(B), int(S), int(heads),
                         make_cfg(B * S, d, d_ff, E, k, C, G, "bf16", act, renorm, wpacked=wpacked), order)


def moe_product_timing(on):
    """Start (True) or stop (False) recording per-product events on this thread; either clears the record."""
    _check(_lib.moe_product_timing(1 if on else 0))


def moe_product_times():
    """(ms, counts) per expert product (PRODUCTS order) since the last clear; clears the record."""
    import numpy as np
    ms = np.zeros(len(PRODUCTS), np.float64)
    counts = np.zeros(len(PRODUCTS), np.int32)
    _check(_lib.moe_product_times(ms.ctypes.data, counts.ctypes.data))
    return ms, counts


def moe_block_op_times():
    """Durations (ms) of the backward operations of this thread's last timed block call (BLOCK_OPS order)."""
    import numpy as np
    ms = np.zeros(len(BLOCK_OPS), np.float64)
    _check(_lib.moe_block_op_times(ms.ctypes.data))
    return ms


def moe_block_dw_schedule(op_ms, a2a_ms):
    """The block backward's weight-gradient schedule: (dw_order [6], assign [16], overlap)."""
    import numpy as np
    t = np.ascontiguousarray(op_ms, np.float64)
    assert t.size == len(BLOCK_OPS)
    order = np.empty(6, np.int32)
    assign = np.empty(16, np.int32)
    ov = ctypes.c_double(0.0)
    _check(_lib.moe_block_dw_schedule(t.ctypes.data, float(a2a_ms), order.ctypes.data, assign.ctypes.data,
                                      ctypes.byref(ov)))
    return order, assign, ov.value


def block_shapes(cfg: moe_block_cfg, n_chunks: int):
    """{name: (numel, dtype)} of every weight, gradient and activation of the block."""
    m = cfg.moe
    T, d, f, E, k = m.T, m.d_model, m.d_ff, m.E, m.k
    nd, nf = expert_numel(m, d), expert_numel(m, f)
    Sp = (cfg.S + 63) // 64 * 64
    st = cfg.B * cfg.heads * Sp
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    return {
        "ln1_g": (d, bf), "ln1_b": (d, bf), "Wqkv": (3 * d * d, bf), "Wo": (d * d, bf), "ln2_g": (d, bf),
        "ln2_b": (d, bf), "Wg": (E * d, bf), "W1": (E * f * d, bf), "W2": (E * d * f, bf),
        "dln1_g": (d, f32), "dln1_b": (d, f32), "dWqkv": (3 * d * d, bf), "dWo": (d * d, bf), "dln2_g": (d, f32),
        "dln2_b": (d, f32), "dWg": (E * d, f32), "dW1": (E * f * d, bf), "dW2": (E * d * f, bf),
        "a": (T * d, bf), "ln1_mean": (T, f32), "ln1_rstd": (T, f32), "qkv": (T * 3 * d, bf), "attn": (T * d, bf),
        "lse": (st, f32), "h": (T * d, bf), "ln2_mean": (T, f32), "ln2_rstd": (T, f32), "m": (T * d, bf),
        "logits": (T * E, f32), "idx": (T * k, i32), "w": (T * k, f32), "slot": (T * k, i32),
        "fill": (n_chunks * E, i32), "send_buf": (nd, bf), "H": (nf, bf), "A": (nf, bf),
        "expert_out": (nd, bf), "W1p": (E * f * d, bf), "W2p": (E * d * f, bf), "dO": (nd, bf), "dH": (nf, bf),
        "dXe": (nd, bf),
        "dlogits": (T * E, f32), "dm": (T * d, bf), "dh": (T * d, bf), "dattn": (T * d, bf), "delta": (st, f32),
        "dqkv": (T * 3 * d, bf), "da": (T * d, bf),
    }


def moe_block_workspace_bytes(cfg: moe_block_cfg, n_chunks: int) -> int:
    return int(_lib.moe_block_workspace_bytes(ctypes.byref(cfg), n_chunks))


def moe_block_chunked(cfg: moe_block_cfg, weights: dict, grads: Optional[dict], x, out, dy, dx, acts: dict,
                      passes: int, n_chunks: int, streams, ws):
    """streams: three torch.cuda.Stream (or raw handles) -- compute, data movement, weight gradients."""
    _check(_bind.block_chunked(cfg, weights, grads, x, out, dy, dx, acts, passes, n_chunks, streams, ws))


def alloc_block(cfg: moe_block_cfg, n_chunks: int, device="cuda", names=None) -> dict:
    """Empty device tensors for the block's gradients and activations (and its
    workspace under "ws"); weights are the caller's."""
    shp = block_shapes(cfg, n_chunks)
    out = {}
    for n in BLOCK_GRADS + BLOCK_ACTS_FWD + BLOCK_ACTS_BWD:
        if names is None or n in names:
            numel, dt = shp[n]
            out[n] = torch.empty(numel, dtype=dt, device=device)
    out["ws"] = torch.empty(max(16, moe_block_workspace_bytes(cfg, n_chunks)), dtype=torch.uint8, device=device)
    return out


# ----------------------------------------------------- lookup and loss around the block
@dataclass
class LmBuffers:
    """What a step of token lookup, blocks and loss keeps beside the blocks' own buffers."""
    embed: moe_embed_cfg
    embed_add: moe_embed_cfg   # the lookup's gradient added to the loss's, for a tied table
    xent: moe_xent_cfg
    h: list                    # [T][d] the blocks' inputs, and the last one's output
    loss: torch.Tensor
    lse: torch.Tensor
    dh: torch.Tensor           # gradients at the activations, in turn
    dx: torch.Tensor
    dWout: torch.Tensor        # [V][d]
    dWin: Optional[torch.Tensor]   # [V][d]; None: tied to the output matrix
    ws: torch.Tensor


def alloc_lm(cfg: moe_block_cfg, V: int, n_blocks: int = 1, scale: float = 1.0, tied: bool = True,
             device="cuda") -> LmBuffers:
    m = cfg.moe
    T, d, bf = m.T, m.d_model, torch.bfloat16
    embed, xent = make_embed_cfg(T, V, d, "bf16", scale), make_xent_cfg(T, V, d, "bf16")
    e = lambda *s, dtype=bf: torch.empty(*s, dtype=dtype, device=device)
    sizes = [moe_embed_bwd_workspace_bytes(embed), moe_xent_workspace_bytes(xent), moe_xent_workspace_bytes(xent, True)]
    if T > 0 and 0 in sizes:   # (tokens need some of each; the message is of the last one refused)
        raise MoeError(MOE_ESHAPE, moe_last_error())
    need = max(sizes)
    return LmBuffers(embed=embed, embed_add=make_embed_cfg(T, V, d, "bf16", scale, accum=1), xent=xent,
                     h=[e(T, d) for _ in range(n_blocks + 1)], loss=e(T, dtype=torch.float32),
                     lse=e(T, dtype=torch.float32), dh=e(T, d), dx=e(T, d), dWout=e(V, d),
                     dWin=None if tied else e(V, d), ws=e(max(16, need), dtype=torch.uint8))


def _lm_blocks(b: LmBuffers, *per_block):
    if any(len(q) != len(b.h) - 1 for q in per_block):
        raise ValueError(f"{len(b.h) - 1} blocks were allocated, got {[len(q) for q in per_block]}")


def lm_forward(b: LmBuffers, cfg: moe_block_cfg, ids, target, Win, Wout, weights: list, acts: list, n_chunks: int, streams):
    """Token lookup -> blocks (with a capacity) -> cross entropy of every token (b.loss), which takes the last block's
    output as it is: a norm in front of the output matrix is the caller's, with moe_xent called behind it.  weights, acts: of each block (block_shapes,
    alloc_block); ids, target [T] int32.  streams as for moe_block_chunked; the rest runs on the first."""
    _lm_blocks(b, weights, acts)
    moe_embed(b.embed, ids, Win, b.h[0], streams[0])
    for i, (w, a) in enumerate(zip(weights, acts)):
        moe_block_chunked(cfg, w, None, b.h[i], b.h[i + 1], None, None, a, MOE_BLOCK_FWD, n_chunks, streams, a["ws"])
    moe_xent(b.xent, b.h[-1], Wout, target, b.loss, b.lse, b.ws, streams[0])


def lm_backward(b: LmBuffers, cfg: moe_block_cfg, ids, target, Wout, weights: list, grads: list, acts: list, dloss,
                n_chunks: int, streams):
    """After lm_forward: dloss [T] float (1 / n for the mean of n tokens) -> b.dWout, every block's grads, and the
    table's gradient in b.dWin, or added to b.dWout where the two are tied."""
    _lm_blocks(b, weights, grads, acts)
    moe_xent_bwd(b.xent, b.h[-1], Wout, target, b.lse, dloss, b.dh, b.dWout, b.ws, streams[0])
    dy, dx = b.dh, b.dx
    for i in reversed(range(len(weights))):
        moe_block_chunked(cfg, weights[i], grads[i], b.h[i], b.h[i + 1], dy, dx, acts[i], MOE_BLOCK_BWD, n_chunks, streams,
                          acts[i]["ws"])
        dy, dx = dx, dy
    if b.dWin is None:
        moe_embed_bwd(b.embed_add, ids, dy, b.dWout, b.ws, streams[0])
    else:
        moe_embed_bwd(b.embed, ids, dy, b.dWin, b.ws, streams[0])
