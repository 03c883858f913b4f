"""ctypes binding of libdqt.so: the C ABI of include/dqt.h, one Python function
per entry point with the same name.  Argument marshalling only: torch tensors
are passed as device pointers on torch's current stream, every step of the
path runs in the library's HIP kernels, and a missing or unloadable library
raises immediately (there is no fallback).
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdqt.so")

# dqt_status
DQT_OK, DQT_ERR_NULL, DQT_ERR_SHAPE, DQT_ERR_ALIGN, DQT_ERR_DTYPE = 0, 1, 2, 3, 4
DQT_ERR_RANGE, DQT_ERR_WORKSPACE, DQT_ERR_UNSUPPORTED, DQT_ERR_HIP = 5, 6, 7, 8
# dqt_dtype
DQT_F32, DQT_BF16, DQT_I8, DQT_FP8E4M3, DQT_TERNARY2, DQT_INT4, DQT_INT3 = 0, 1, 2, 3, 4, 5, 6

EXPORTS = (
    "dqt_act_quant", "dqt_act_quant_batch", "dqt_linear_fwd_workspace", "dqt_linear_fwd", "dqt_linear_bwd_workspace",
    "dqt_linear_bwd", "dqt_linear_fwd_batch_workspace", "dqt_linear_fwd_batch",
    "dqt_linear_bwd_batch_workspace", "dqt_linear_bwd_batch", "dqt_linear_bwd_sr_batch",
    "dqt_linear_fwd_batch_noalloc", "dqt_sr_table_bytes", "dqt_sr_table_build",
    "dqt_sr_update_table", "dqt_rmsnorm_act_quant", "dqt_rmsnorm_backward", "dqt_absmax_requant_workspace",
    "dqt_absmax_requant_batch",
    "dqt_sr_update_batch", "dqt_adamw_sr_update", "dqt_adamw_sr_update_batch",
    "dqt_update_variant_workspace", "dqt_update_variant_batch",
    "dqt_sr_update", "dqt_debug_rng", "dqt_absmean_init", "dqt_pack_ternary",
    "dqt_unpack_ternary", "dqt_pack_int4", "dqt_unpack_int4", "dqt_pack_int3", "dqt_unpack_int3", "dqt_launch_timer_start", "dqt_launch_timer_stop", "dqt_read_stream",
    "dqt_swiglu_act_quant", "dqt_swiglu_backward", "dqt_logprob_workspace", "dqt_logprob_fwd",
    "dqt_logprob_bwd", "dqt_attn_fwd_workspace", "dqt_attn_fwd", "dqt_attn_bwd_workspace",
    "dqt_attn_bwd", "dqt_status_string", "dqt_version",
)


class DqtWeight(ctypes.Structure):
    _fields_ = [
        ("d_out", ctypes.c_int32), ("d_in", ctypes.c_int32), ("wfmt", ctypes.c_int32),
        ("qmin", ctypes.c_int32), ("qmax", ctypes.c_int32), ("alpha", ctypes.c_float),
        ("tensor_id", ctypes.c_uint32), ("reserved", ctypes.c_uint32),
    ]


MAX_BATCH = 8


class DqtLinearIO(ctypes.Structure):
    _fields_ = [
        ("w", ctypes.POINTER(DqtWeight)), ("Wq", ctypes.c_void_p), ("Xq", ctypes.c_void_p),
        ("xdq", ctypes.c_void_p), ("Y", ctypes.c_void_p), ("dY", ctypes.c_void_p),
        ("dX", ctypes.c_void_p), ("dW", ctypes.c_void_p),
    ]


class DqtActIO(ctypes.Structure):
    _fields_ = [("X", ctypes.c_void_p), ("Xq", ctypes.c_void_p), ("xdq", ctypes.c_void_p),
                ("K", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class DqtCkptIO(ctypes.Structure):
    _fields_ = [("Gq", ctypes.c_void_p), ("Uq", ctypes.c_void_p), ("gs", ctypes.c_void_p),
                ("us", ctypes.c_void_p)]


class DqtAttn(ctypes.Structure):
    _fields_ = [("q_start", ctypes.c_void_p), ("k_start", ctypes.c_void_p),
                ("q_tokens", ctypes.c_int64), ("k_tokens", ctypes.c_int64),
                ("n_seq", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("d", ctypes.c_int32), ("scale", ctypes.c_float), ("causal", ctypes.c_int32),
                ("reserved", ctypes.c_int64)]


class DqtRows(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


def weight(d_out: int, d_in: int, wfmt: int, qmin: int, qmax: int, alpha: float,
           tensor_id: int = 0) -> DqtWeight:
    return DqtWeight(d_out, d_in, wfmt, qmin, qmax, float(alpha), tensor_id, 0)


class DqtError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn}: {status_string(status)}")


_lib = None

_vp, _i32, _i64, _u32, _u64, _f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                     ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float)
_wp = ctypes.POINTER(DqtWeight)

_SIGS = {
    "dqt_act_quant": (_i32, [_vp, _i32, _i64, _i32, _i32, _vp, _vp, _vp]),
    "dqt_act_quant_batch": (_i32, [_i32, _vp, _i32, _i64, _i32, _vp]),
    "dqt_rmsnorm_act_quant": (_i32, [_vp, _i32, _vp, _f32, _i64, _i32, _i32, _vp, _vp, _vp, _vp]),
    "dqt_rmsnorm_backward": (_i32, [_i32, _vp, _vp, _i32, _vp, _vp, _i64, _i32, _vp, _vp, _i32, _vp]),
    "dqt_swiglu_act_quant": (_i32, [_vp, _vp, _i32, _i64, _i32, _i32, _vp, _vp, _vp, _vp]),
    "dqt_swiglu_backward": (_i32, [_vp, _i32, _vp, _vp, _vp, _i64, _i32, _vp, _vp, _vp]),
    "dqt_logprob_workspace": (ctypes.c_size_t, [_i64, _i32, _i32]),
    "dqt_logprob_fwd": (_i32, [_vp, _i32, _i64, _i32, _i64, _vp, _vp, _vp, _vp, _vp, _i32, _vp, _vp,
                               _vp, ctypes.c_size_t, _vp]),
    "dqt_logprob_bwd": (_i32, [_vp, _i32, _i64, _i32, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp]),
    "dqt_attn_fwd_workspace": (ctypes.c_size_t, [_vp]),
    "dqt_attn_fwd": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    "dqt_attn_bwd_workspace": (ctypes.c_size_t, [_vp]),
    "dqt_attn_bwd": (_i32, [_vp] * 11 + [ctypes.c_size_t, _vp]),
    "dqt_linear_fwd_workspace": (ctypes.c_size_t, [_wp]),
    "dqt_linear_fwd": (_i32, [_wp, _vp, _vp, _i32, _i64, _i32, _vp, _vp, _vp, _i32, _vp,
                              ctypes.c_size_t, _vp]),
    "dqt_linear_bwd_workspace": (ctypes.c_size_t, [_wp, _i64]),
    "dqt_linear_bwd": (_i32, [_wp, _vp, _vp, _i32, _vp, _vp, _i32, _i64, _i32, _vp, _i32, _vp,
                              _vp, ctypes.c_size_t, _vp]),
    "dqt_sr_update": (_i32, [_wp, _vp, _vp, _f32, _u64, _u32, _vp, _vp]),
    "dqt_linear_fwd_batch_workspace": (ctypes.c_size_t, [_i32, _vp]),
    "dqt_linear_fwd_batch": (_i32, [_i32, _vp, _i64, _i32, _i32, _vp, ctypes.c_size_t, _vp]),
    "dqt_linear_fwd_batch_noalloc": (_i32, [_i32, _vp, _i64, _i32, _i32, _vp]),
    "dqt_linear_bwd_batch_workspace": (ctypes.c_size_t, [_i32, _vp, _i64]),
    "dqt_linear_bwd_batch": (_i32, [_i32, _vp, _i64, _i32, _i32, _i32, _i32, _vp,
                                    ctypes.c_size_t, _vp]),
    "dqt_linear_bwd_sr_batch": (_i32, [_i32, _vp, _i64, _i32, _i32, _i32, _i32, _f32, _u64, _u32,
                                       _vp, _vp, ctypes.c_size_t, _vp]),
    "dqt_sr_update_batch": (_i32, [_i32, _vp, _f32, _u64, _u32, _vp, _vp]),
    "dqt_sr_table_bytes": (ctypes.c_size_t, [_i32]),
    "dqt_sr_table_build": (_i32, [_i32, _vp, _vp, ctypes.c_size_t]),
    "dqt_sr_update_table": (_i32, [_i32, _vp, _vp, _f32, _u64, _u32, _vp, _vp, _vp]),
    "dqt_update_variant_workspace": (ctypes.c_size_t, [_i32]),
    "dqt_absmax_requant_workspace": (ctypes.c_size_t, [_i32]),
    "dqt_absmax_requant_batch": (_i32, [_i32, _vp, _f32, _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    "dqt_update_variant_batch": (_i32, [_i32, _vp, _f32, _u64, _u32, _i32, _f32, _vp, _vp,
                                        ctypes.c_size_t, _vp]),
    "dqt_adamw_sr_update": (_i32, [_wp, _vp, _vp, _vp, _vp, _vp, _u64, _u32, _vp, _vp]),
    "dqt_adamw_sr_update_batch": (_i32, [_i32, _vp, _vp, _vp, _vp, _u64, _u32, _vp, _vp]),
    "dqt_debug_rng": (_i32, [_u64, _u32, _u32, _u64, _i64, _vp, _vp]),
    "dqt_absmean_init": (_i32, [_vp, _i64, _i32, _i32, _vp, _vp]),
    "dqt_pack_ternary": (_i32, [_vp, _i64, _i64, _vp]),
    "dqt_unpack_ternary": (_i32, [_vp, _i64, _i64, _vp]),
    "dqt_pack_int4": (_i32, [_vp, _i64, _i64, _vp]),
    "dqt_unpack_int4": (_i32, [_vp, _i64, _i64, _vp]),
    "dqt_pack_int3": (_i32, [_vp, _i64, _i64, _vp]),
    "dqt_unpack_int3": (_i32, [_vp, _i64, _i64, _vp]),
    "dqt_launch_timer_start": (_i32, [_i32]),
    "dqt_launch_timer_stop": (_i32, [_vp, _i32, _vp]),
    "dqt_read_stream": (_i32, [_vp, ctypes.c_size_t, _vp, _vp]),
    "dqt_status_string": (ctypes.c_char_p, [_i32]),
    "dqt_version": (_i32, []),
}


def load(path: str = LIB_PATH):
    """Load libdqt.so (once).  Raises if it is missing: there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with "
                           "`python -m paper_2412_04787_amd.build_lib`")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(fn: str, st: int):
    if st != DQT_OK:
        raise DqtError(fn, st)


def status_string(st: int) -> str:
    return load().dqt_status_string(st).decode()


def version() -> int:
    return load().dqt_version()


# ----------------------------------------------------------------- tensors

_TORCH = None           # (imported late)


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _addr(t):
    return None if t is None else t.data_ptr()


def _same(*ts):
    """The shape [M, K] that contiguous tensors of one dtype share."""
    shape, dtype = ts[0].shape, ts[0].dtype
    ok = ts[0].is_contiguous()
    for t in ts[1:]:
        ok = ok and t.dtype is dtype and t.shape == shape and t.is_contiguous()
    if not ok:
        raise ValueError("expected contiguous tensors of one shape and dtype")
    return shape


def _here(t, *others):
    """The current device, on whose stream the kernels run: refuses tensors of
    another one and in host memory."""
    dev = t.get_device()                   # (-1 in host memory)
    if dev < 0 or dev != _torch()._C._cuda_getDevice():
        raise ValueError("tensor in host memory" if dev < 0 else f"tensor on device {dev}, which is not the current one")
    for o in others:
        if o.get_device() != dev:
            raise ValueError(f"tensor on {o.device}, others on device {dev}")
    return dev


def _bufs(dev, *bufs):
    """Refuses a buffer (tensor or None, n, dtype) that is not one of at least n
    consecutive bytes, values of dtype, on device dev."""
    for t, n, dtype in bufs:
        if t is not None and (t.get_device() != dev or t.dtype is not dtype or t.nbytes < n or not t.is_contiguous()):
            raise ValueError(f"expected {n} consecutive bytes, {dtype}, on device {dev}, got {tuple(t.shape)} of "
                             f"{t.dtype} with strides {t.stride()} on {t.device}")


def _ws_bytes(dev, t):
    """The bytes of a workspace on device dev."""
    if t is None:
        return 0
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"expected a contiguous workspace on device {dev}, got strides {t.stride()} on {t.device}")
    return t.nbytes


def _unit_stride(t):
    if t.dim() != 2 or (t.stride(1) != 1 and t.numel() > 0 and t.shape[1] > 1):
        raise ValueError("expected a [rows, columns] tensor with unit column stride")


def _stream(stream=None):
    """The stream's handle (an integer); without one, that of torch's current stream on the
    current device.  (Asked for directly: building the Stream object of
    torch.cuda.current_stream() was a third of a small call's host time.)"""
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    if not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    c = torch._C
    return c._cuda_getCurrentRawStream(c._cuda_getDevice())


_DTYPE_CODES = {}       # (filled on first use: torch is imported late)


def dtype_code(t) -> int:
    if not _DTYPE_CODES:
        torch = _torch()
        _DTYPE_CODES.update({torch.float32: DQT_F32, torch.bfloat16: DQT_BF16, torch.int8: DQT_I8,
                             torch.float8_e4m3fn: DQT_FP8E4M3, torch.uint8: DQT_FP8E4M3})
    return _DTYPE_CODES[t.dtype]


def dqt_act_quant(X, act_q: int, Xq, xdq, stream=None):
    M, K = X.shape
    _check("dqt_act_quant", load().dqt_act_quant(_ptr(X), dtype_code(X), M, K, act_q, _ptr(Xq),
                                                 _ptr(xdq), _stream(stream)))


def dqt_rmsnorm_act_quant(X, gamma, eps: float, act_q: int, Xq, xdq, rinv=None, stream=None):
    M, K = X.shape
    _check("dqt_rmsnorm_act_quant",
           load().dqt_rmsnorm_act_quant(_ptr(X), dtype_code(X), _ptr(gamma), eps, M, K, act_q,
                                        _ptr(Xq), _ptr(xdq), _ptr(rinv), _stream(stream)))


def dqt_rmsnorm_backward(dYs, X, gamma, rinv, dX, gpart, stream=None):
    """dYs: list of 1..4 [M, K] bf16 tensors; gpart: [blocks, K] fp32."""
    M, K = X.shape
    ptrs = (ctypes.c_void_p * len(dYs))(*[t.data_ptr() for t in dYs])
    _check("dqt_rmsnorm_backward",
           load().dqt_rmsnorm_backward(len(dYs), ptrs, _ptr(X), dtype_code(X), _ptr(gamma),
                                       _ptr(rinv), M, K, _ptr(dX), _ptr(gpart), gpart.shape[0],
                                       _stream(stream)))


CKPT_GROUP = 128


class SwigluCkpt:
    """8-bit checkpoint of gate and up [M, K]: codes Gq, Uq (int8) and scales
    gs, us (fp32, one for CKPT_GROUP consecutive elements of a row)."""

    def __init__(self, Gq, Uq, gs, us):
        torch = _torch()
        M, K = _same(Gq, Uq)
        if Gq.dtype is not torch.int8 or gs.dtype is not torch.float32:
            raise ValueError("expected int8 codes and fp32 scales")
        if _same(gs, us) != (M, (K + CKPT_GROUP - 1) // CKPT_GROUP):
            raise ValueError(f"expected one scale for {CKPT_GROUP} elements of a row, got {tuple(gs.shape)}")
        self.Gq, self.Uq, self.gs, self.us = Gq, Uq, gs, us
        self.io = DqtCkptIO(_addr(Gq), _addr(Uq), _addr(gs), _addr(us))


def swiglu_ckpt(M: int, K: int, device="cuda:0") -> SwigluCkpt:
    """Buffers for the checkpoint of a gate and an up of shape [M, K]."""
    torch = _torch()
    groups = (K + CKPT_GROUP - 1) // CKPT_GROUP
    q = [torch.empty((M, K), dtype=torch.int8, device=device) for _ in range(2)]
    s = [torch.empty((M, groups), dtype=torch.float32, device=device) for _ in range(2)]
    return SwigluCkpt(*q, *s)


def _check_ckpt(ckpt: SwigluCkpt, M, K, x):
    """Refuses a checkpoint of another size, or of another device than x."""
    if ckpt.Gq.shape != (M, K):
        raise ValueError(f"checkpoint of {tuple(ckpt.Gq.shape)}, expected {(M, K)}")
    _here(x, ckpt.Gq, ckpt.Uq, ckpt.gs, ckpt.us)


def dqt_swiglu_act_quant(G, U, act_q: int, Xq, xdq, ckpt: SwigluCkpt | None = None, stream=None):
    """G, U: contiguous [M, K] of one dtype; Xq: M K bytes, xdq: M fp32 values
    (larger buffers are used from their start)."""
    M, K = _same(G, U)
    dev = _here(G, U)
    if Xq is not None and Xq.element_size() != 1:
        raise ValueError(f"expected 8-bit codes, got {Xq.dtype}")
    _bufs(dev, (Xq, M * K, None if Xq is None else Xq.dtype), (xdq, 4 * M, _torch().float32))
    if ckpt is not None:
        _check_ckpt(ckpt, M, K, G)
    _check("dqt_swiglu_act_quant",
           load().dqt_swiglu_act_quant(_addr(G), _addr(U), dtype_code(G), M, K, act_q, _addr(Xq), _addr(xdq),
                                       None if ckpt is None else ctypes.byref(ckpt.io), _stream(stream)))


def dqt_swiglu_backward(dH, G, U, dG, dU, stream=None):
    """dH, G, U, dG, dU: contiguous [M, K] of one dtype."""
    M, K = _same(dH, G, U, dG, dU)
    _here(dH, G, U, dG, dU)
    _check("dqt_swiglu_backward",
           load().dqt_swiglu_backward(_addr(dH), dtype_code(dH), _addr(G), _addr(U), None, M, K, _addr(dG),
                                      _addr(dU), _stream(stream)))


def dqt_swiglu_backward_ckpt(dH, ckpt: SwigluCkpt, dG, dU, stream=None):
    """dqt_swiglu_backward with gate and up from their 8-bit checkpoint."""
    M, K = _same(dH, dG, dU)
    _here(dH, dG, dU)
    _check_ckpt(ckpt, M, K, dH)
    _check("dqt_swiglu_backward",
           load().dqt_swiglu_backward(_addr(dH), dtype_code(dH), None, None, ctypes.byref(ckpt.io), M, K,
                                      _addr(dG), _addr(dU), _stream(stream)))


MAX_TOP = 32


def dqt_logprob_workspace(M: int, V: int, top_k: int = 0) -> int:
    return int(load().dqt_logprob_workspace(M, V, top_k))


def _as_many(targets, M):
    if targets is not None and targets.numel() != M:
        raise ValueError(f"expected {M} targets, got {targets.numel()}")


def dqt_logprob_fwd(X, targets, logp, lse=None, entropy=None, stat=None, top_ids=None, top_logp=None,
                    ws=None, stream=None):
    """X: [M, V] logits, rows of any stride; targets: int64 [M]; logp, lse,
    entropy: fp32 [M], stat (for the backward): fp32 [M, 2], or None; top_ids
    (int64) and top_logp (fp32): [M, k], or None.  All but X contiguous; larger
    outputs are used from their start."""
    _unit_stride(X)
    M, V = X.shape
    dev, torch = _here(X), _torch()
    f32, i64, top_k = torch.float32, torch.int64, 0
    if top_ids is not None:
        if top_ids.dim() != 2:
            raise ValueError("expected top_ids of shape [M, k]")
        top_k = top_ids.shape[1]
    _bufs(dev, (targets, 8 * M, i64), (logp, 4 * M, f32), (lse, 4 * M, f32), (entropy, 4 * M, f32), (stat, 8 * M, f32),
          (top_ids, 8 * M * top_k, i64), (top_logp, 4 * M * top_k, f32))
    _as_many(targets, M)
    _check("dqt_logprob_fwd",
           load().dqt_logprob_fwd(_addr(X), dtype_code(X), M, V, X.stride(0) if M > 1 else V, _addr(targets),
                                  _addr(logp), _addr(lse), _addr(entropy), _addr(stat), top_k,
                                  _addr(top_ids), _addr(top_logp), _addr(ws), _ws_bytes(dev, ws), _stream(stream)))


def dqt_logprob_bwd(X, targets, stat, dlogp, dX, entropy=None, dent=None, stream=None):
    """dX: [M, V] of X's dtype (X itself is allowed); dlogp, dent: fp32 [M] or None."""
    _unit_stride(X)
    M, V = X.shape
    _unit_stride(dX)
    if dX.dtype != X.dtype or dX.shape != X.shape:
        raise ValueError("dX must have X's dtype and shape")
    f32 = _torch().float32
    _bufs(_here(X, dX), (targets, 8 * M, _torch().int64), (stat, 8 * M, f32), (dlogp, 4 * M, f32),
          (entropy, 4 * M, f32), (dent, 4 * M, f32))
    _as_many(targets, M)
    _check("dqt_logprob_bwd",
           load().dqt_logprob_bwd(_addr(X), dtype_code(X), M, V, X.stride(0) if M > 1 else V, _addr(targets),
                                  _addr(stat), _addr(entropy), _addr(dlogp), _addr(dent), _addr(dX),
                                  dX.stride(0) if M > 1 else V, _stream(stream)))


def attn(q_tokens: int, k_tokens: int, heads: int, kv_heads: int, d: int, q_start=None, k_start=None,
         scale: float | None = None, causal: bool = True) -> DqtAttn:
    """The descriptor of an attention call.  q_start, k_start: device int32
    [n_seq + 1] (kept alive on the descriptor), or None for one sequence of
    all tokens; scale: 1 / sqrt(d) by default."""
    n = {t.numel() - 1 for t in (q_start, k_start) if t is not None} or {1}
    if len(n) != 1:
        raise ValueError("q_start and k_start must have the same length")
    starts = [t for t in (q_start, k_start) if t is not None]
    for t in starts:
        if t.dtype != _torch().int32 or not t.is_contiguous():
            raise ValueError("q_start and k_start must be contiguous int32")
    if starts:
        _here(*starts)
    a = DqtAttn(_addr(q_start), _addr(k_start), q_tokens, k_tokens, n.pop(), heads, kv_heads, d,
                d ** -0.5 if scale is None else scale, int(causal), 0)
    a._keep = (q_start, k_start)
    a._dev = starts[0].get_device() if starts else None
    a._shapes = {"q": (q_tokens, heads, d), "k": (k_tokens, kv_heads, d)}
    return a


_pack_rows = struct.Struct("3q").pack


def _rows(a: DqtAttn, tensors, kinds: str, lse):
    """(Their device, the dqt_rows (as bytes)) of bf16 tensors [q_tokens, heads, d]
    (kind "q") or [k_tokens, kv_heads, d] ("k") with any token and head strides."""
    torch = _torch()
    bf16, shapes = torch.bfloat16, a._shapes
    dev = _here(*tensors)
    _bufs(dev, (lse, 4 * a.heads * a.q_tokens, torch.float32))
    if a._dev is not None and a._dev != dev:
        raise ValueError(f"q_start or k_start on device {a._dev}, the tensors on device {dev}")
    rows = []
    for t, kind in zip(tensors, kinds):
        shape = shapes[kind]
        if t.dtype is not bf16 or t.shape != shape:
            raise ValueError(f"expected a bfloat16 tensor of shape {shape}, got {t.dtype} {tuple(t.shape)}")
        st, sh, sd = t.stride()
        if sd != 1 and t.numel() > 0:
            raise ValueError(f"expected unit last stride, got strides {t.stride()}")
        n, h, d = shape
        # (strides of a dimension of one do not matter)
        rows.append(_pack_rows(t.data_ptr(), st if n > 1 else h * d, sh if h > 1 else d))
    return dev, rows


def dqt_attn_fwd_workspace(a: DqtAttn) -> int:
    return int(load().dqt_attn_fwd_workspace(ctypes.byref(a)))


def dqt_attn_fwd(a: DqtAttn, Q, K, V, O, lse=None, ws=None, stream=None):
    """Q, O: [q_tokens, heads, d]; K, V: [k_tokens, kv_heads, d], bf16 with any
    token and head strides; lse: contiguous fp32 [heads, q_tokens] or None."""
    dev, r = _rows(a, (Q, K, V, O), "qkkq", lse)
    _check("dqt_attn_fwd", load().dqt_attn_fwd(ctypes.byref(a), *r, _addr(lse), _addr(ws), _ws_bytes(dev, ws),
                                               _stream(stream)))


def dqt_attn_bwd_workspace(a: DqtAttn) -> int:
    return int(load().dqt_attn_bwd_workspace(ctypes.byref(a)))


def dqt_attn_bwd(a: DqtAttn, Q, K, V, O, lse, dO, dQ, dK, dV, ws, stream=None):
    """Shapes as dqt_attn_fwd; dO, dQ like Q, dK and dV like K."""
    dev, r = _rows(a, (Q, K, V, O, dO, dQ, dK, dV), "qkkqqqkk", lse)
    _check("dqt_attn_bwd", load().dqt_attn_bwd(ctypes.byref(a), *r[:4], _addr(lse), *r[4:], _addr(ws), _ws_bytes(dev, ws),
                                               _stream(stream)))


def dqt_linear_fwd_workspace(w: DqtWeight) -> int:
    return int(load().dqt_linear_fwd_workspace(ctypes.byref(w)))


def dqt_linear_fwd(w: DqtWeight, Wq, X, M: int, act_q: int, Xq, xdq, Y, ws=None, stream=None,
                   x_t: int | None = None):
    """X may be None when Xq / xdq already hold the quantised input."""
    if x_t is None:
        x_t = dtype_code(X) if X is not None else DQT_F32
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check("dqt_linear_fwd", load().dqt_linear_fwd(ctypes.byref(w), _ptr(Wq), _ptr(X), x_t, M,
                                                   act_q, _ptr(Xq), _ptr(xdq), _ptr(Y),
                                                   dtype_code(Y), _ptr(ws), ws_bytes,
                                                   _stream(stream)))


def workspace(nbytes: int, device="cuda:0"):
    """A zero-filled device buffer of at least nbytes (16-byte aligned), or
    None for 0.  (The library does not depend on a workspace's contents; the
    zero fill only makes unused bytes deterministic.)"""
    if nbytes == 0:
        return None
    torch = _torch()
    return torch.zeros(((nbytes + 15) // 16 * 4,), dtype=torch.float32, device=device)


def dqt_linear_bwd_workspace(w: DqtWeight, M: int) -> int:
    return int(load().dqt_linear_bwd_workspace(ctypes.byref(w), M))


def dqt_linear_bwd(w: DqtWeight, Wq, Xq, act_q: int, xdq, dY, M: int, xt_t: int, dX, dW,
                   ws=None, stream=None, dy_t: int | None = None, dx_t: int | None = None):
    dy_t = dtype_code(dY) if dy_t is None else dy_t
    dx_t = (dtype_code(dX) if dX is not None else DQT_F32) if dx_t is None else dx_t
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check("dqt_linear_bwd", load().dqt_linear_bwd(ctypes.byref(w), _ptr(Wq), _ptr(Xq), act_q,
                                                   _ptr(xdq), _ptr(dY), dy_t, M, xt_t, _ptr(dX),
                                                   dx_t, _ptr(dW), _ptr(ws), ws_bytes,
                                                   _stream(stream)))


def dqt_sr_update(w: DqtWeight, Wq, dW, lr: float, seed: int, step: int, counters=None,
                  stream=None):
    _check("dqt_sr_update", load().dqt_sr_update(ctypes.byref(w), _ptr(Wq), _ptr(dW), lr, seed,
                                                 step, _ptr(counters), _stream(stream)))


def dqt_debug_rng(seed: int, step: int, tensor_id: int, i0: int, out, stream=None):
    _check("dqt_debug_rng", load().dqt_debug_rng(seed, step, tensor_id, i0, out.numel(),
                                                 _ptr(out), _stream(stream)))


def dqt_launch_timer_start(max_launches: int):
    _check("dqt_launch_timer_start", load().dqt_launch_timer_start(max_launches))


def dqt_launch_timer_stop(max_launches: int):
    """Durations (ms) of the GEMM kernel launches timed since the start, in
    issue order, and how many launches were timed."""
    ms = (ctypes.c_float * max(1, max_launches))()
    count = ctypes.c_int32(0)
    _check("dqt_launch_timer_stop", load().dqt_launch_timer_stop(ms, max_launches, ctypes.byref(count)))
    return [float(ms[k]) for k in range(min(count.value, max_launches))], count.value


READ_STREAM_SINK_WORDS = 32768


def dqt_read_stream(src, sink, stream=None):
    """One streaming read of the device tensor src (all its bytes); sink: a
    device int32/uint32 tensor of READ_STREAM_SINK_WORDS words."""
    nbytes = src.numel() * src.element_size()
    assert sink.numel() * sink.element_size() >= 4 * READ_STREAM_SINK_WORDS
    _check("dqt_read_stream", load().dqt_read_stream(_ptr(src), nbytes, _ptr(sink), _stream(stream)))


# ----------------------------------------------------------------- batches

def linear_io(entries):
    """entries: list of dicts with keys w (DqtWeight), Wq, Xq, xdq, Y, dY, dX, dW
    (tensors or None).  Returns a ctypes array of dqt_linear_io; the weight
    descriptors and the tensors are kept alive on the array (it holds raw
    device pointers)."""
    arr = (DqtLinearIO * len(entries))()
    keep = []
    for k, e in enumerate(entries):
        w = e["w"]
        keep.append(w)
        arr[k].w = ctypes.pointer(w)
        for f in ("Wq", "Xq", "xdq", "Y", "dY", "dX", "dW"):
            t = e.get(f)
            setattr(arr[k], f, None if t is None else t.data_ptr())
            if t is not None:
                keep.append(t)
    arr._keep = keep
    return arr


def act_io(entries):
    """entries: list of (X, Xq, xdq) tensors with X [M, K].  Returns a ctypes
    array of dqt_act_io."""
    arr = (DqtActIO * len(entries))()
    for k, (X, Xq, xdq) in enumerate(entries):
        arr[k].X = X.data_ptr()
        arr[k].Xq = Xq.data_ptr()
        arr[k].xdq = xdq.data_ptr()
        arr[k].K = X.shape[1]
        arr[k].reserved = 0
    return arr


def dqt_act_quant_batch(io, x_t: int, M: int, act_q: int, stream=None):
    _check("dqt_act_quant_batch", load().dqt_act_quant_batch(len(io), io, x_t, M, act_q,
                                                             _stream(stream)))


def dqt_linear_fwd_batch_workspace(io) -> int:
    return int(load().dqt_linear_fwd_batch_workspace(len(io), io))


def dqt_linear_fwd_batch(io, M: int, act_q: int, y_t: int, ws=None, stream=None):
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check("dqt_linear_fwd_batch", load().dqt_linear_fwd_batch(len(io), io, M, act_q, y_t, _ptr(ws),
                                                               ws_bytes, _stream(stream)))


NOALLOC_SCRATCH_BYTES = 32 << 20


def dqt_linear_fwd_batch_noalloc(io, M: int, act_q: int, y_t: int, stream=None):
    """dqt_linear_fwd_batch with the library's static per-GPU scratch instead
    of a workspace (the call allocates nothing)."""
    _check("dqt_linear_fwd_batch_noalloc",
           load().dqt_linear_fwd_batch_noalloc(len(io), io, M, act_q, y_t, _stream(stream)))


def dqt_linear_bwd_batch_workspace(io, M: int) -> int:
    return int(load().dqt_linear_bwd_batch_workspace(len(io), io, M))


def dqt_linear_bwd_batch(io, M: int, act_q: int, dy_t: int, xt_t: int, dx_t: int, ws=None,
                         stream=None):
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check("dqt_linear_bwd_batch", load().dqt_linear_bwd_batch(len(io), io, M, act_q, dy_t, xt_t,
                                                               dx_t, _ptr(ws), ws_bytes,
                                                               _stream(stream)))


def dqt_linear_bwd_sr_batch(io, M: int, act_q: int, dy_t: int, xt_t: int, dx_t: int, lr: float,
                            seed: int, step: int, counters=None, ws=None, stream=None):
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check("dqt_linear_bwd_sr_batch",
           load().dqt_linear_bwd_sr_batch(len(io), io, M, act_q, dy_t, xt_t, dx_t, lr, seed, step,
                                          _ptr(counters), _ptr(ws), ws_bytes, _stream(stream)))


DQT_UPD_SR, DQT_UPD_NEAREST, DQT_UPD_FORCE_REMAIN, DQT_UPD_FORCE_CHANGE = 0, 1, 2, 3


def dqt_update_variant_workspace(n: int) -> int:
    return int(load().dqt_update_variant_workspace(n))


def dqt_update_variant_batch(io, lr: float, seed: int, step: int, mode: int, frac: float = 0.2,
                             counters=None, ws=None, stream=None):
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check("dqt_update_variant_batch",
           load().dqt_update_variant_batch(len(io), io, lr, seed, step, mode, frac, _ptr(counters),
                                           _ptr(ws), ws_bytes, _stream(stream)))


def dqt_absmax_requant_batch(io, lr: float, alpha_out, counters=None, ws=None, stream=None):
    """alpha_out: device fp32 [len(io)], receives each tensor's new scale."""
    if ws is None:
        ws = workspace(int(load().dqt_absmax_requant_workspace(len(io))))
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    _check("dqt_absmax_requant_batch",
           load().dqt_absmax_requant_batch(len(io), io, lr, _ptr(alpha_out), _ptr(counters),
                                           _ptr(ws), ws_bytes, _stream(stream)))


class DqtAdamW(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float)]


def adamw(lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
          weight_decay: float = 0.0) -> DqtAdamW:
    return DqtAdamW(lr, beta1, beta2, eps, weight_decay)


def dqt_adamw_sr_update(w, Wq, dW, m, v, hp: DqtAdamW, seed: int, step: int, counters=None,
                        stream=None):
    _check("dqt_adamw_sr_update",
           load().dqt_adamw_sr_update(ctypes.byref(w), _ptr(Wq), _ptr(dW), _ptr(m), _ptr(v),
                                      ctypes.byref(hp), seed, step, _ptr(counters),
                                      _stream(stream)))


def dqt_adamw_sr_update_batch(io, ms, vs, hp: DqtAdamW, seed: int, step: int, counters=None,
                              stream=None):
    """ms, vs: lists of fp32 device tensors (the moments of each entry of io)."""
    n = len(io)
    mp = (ctypes.c_void_p * n)(*[t.data_ptr() for t in ms])
    vp = (ctypes.c_void_p * n)(*[t.data_ptr() for t in vs])
    _check("dqt_adamw_sr_update_batch",
           load().dqt_adamw_sr_update_batch(n, io, mp, vp, ctypes.byref(hp), seed, step,
                                            _ptr(counters), _stream(stream)))


def dqt_sr_update_batch(io, lr: float, seed: int, step: int, counters=None, stream=None):
    _check("dqt_sr_update_batch", load().dqt_sr_update_batch(len(io), io, lr, seed, step,
                                                             _ptr(counters), _stream(stream)))


def dqt_sr_table_bytes(n: int) -> int:
    return int(load().dqt_sr_table_bytes(n))


def dqt_sr_table_build(io) -> np.ndarray:
    """The update table of the entries of io, as host bytes (copy them to the
    device once, e.g. torch.from_numpy(t).to(device))."""
    n = len(io)
    table = np.zeros(max(dqt_sr_table_bytes(n), 1), dtype=np.uint8)
    _check("dqt_sr_table_build", load().dqt_sr_table_build(n, io, table.ctypes.data, table.size))
    return table


def dqt_sr_update_table(io, table, lr: float, seed: int, step: int, counters=None,
                        per_tensor=None, stream=None):
    """table: the device copy of dqt_sr_table_build(io)."""
    _check("dqt_sr_update_table",
           load().dqt_sr_update_table(len(io), io, _ptr(table), lr, seed, step, _ptr(counters),
                                      _ptr(per_tensor), _stream(stream)))


# ----------------------------------------------------------------- host helpers

def dqt_absmean_init(W0: np.ndarray, qmin: int, qmax: int):
    W0 = np.ascontiguousarray(W0, dtype=np.float32)
    q = np.empty(W0.shape, dtype=np.int8)
    alpha = ctypes.c_float()
    _check("dqt_absmean_init", load().dqt_absmean_init(W0.ctypes.data, W0.size, qmin, qmax,
                                                       q.ctypes.data, ctypes.byref(alpha)))
    return q, np.float32(alpha.value)


def dqt_pack_int4(q: np.ndarray) -> np.ndarray:
    q = np.ascontiguousarray(q, dtype=np.int8)
    rows, cols = q.shape
    packed = np.empty((rows, cols // 2), dtype=np.uint8)
    _check("dqt_pack_int4", load().dqt_pack_int4(q.ctypes.data, rows, cols, packed.ctypes.data))
    return packed


def dqt_unpack_int4(packed: np.ndarray, cols: int) -> np.ndarray:
    packed = np.ascontiguousarray(packed, dtype=np.uint8)
    rows = packed.shape[0]
    q = np.empty((rows, cols), dtype=np.int8)
    _check("dqt_unpack_int4", load().dqt_unpack_int4(packed.ctypes.data, rows, cols, q.ctypes.data))
    return q


def dqt_pack_int3(q: np.ndarray) -> np.ndarray:
    q = np.ascontiguousarray(q, dtype=np.int8)
    rows, cols = q.shape
    packed = np.empty((rows, 3 * cols // 8), dtype=np.uint8)
    _check("dqt_pack_int3", load().dqt_pack_int3(q.ctypes.data, rows, cols, packed.ctypes.data))
    return packed


def dqt_unpack_int3(packed: np.ndarray, cols: int) -> np.ndarray:
    packed = np.ascontiguousarray(packed, dtype=np.uint8)
    rows = packed.shape[0]
    q = np.empty((rows, cols), dtype=np.int8)
    _check("dqt_unpack_int3", load().dqt_unpack_int3(packed.ctypes.data, rows, cols, q.ctypes.data))
    return q


def dqt_pack_ternary(q: np.ndarray) -> np.ndarray:
    q = np.ascontiguousarray(q, dtype=np.int8)
    rows, cols = q.shape
    packed = np.empty((rows, cols // 4), dtype=np.uint8)
    _check("dqt_pack_ternary", load().dqt_pack_ternary(q.ctypes.data, rows, cols,
                                                       packed.ctypes.data))
    return packed


def dqt_unpack_ternary(packed: np.ndarray, cols: int) -> np.ndarray:
    packed = np.ascontiguousarray(packed, dtype=np.uint8)
    rows = packed.shape[0]
    q = np.empty((rows, cols), dtype=np.int8)
    _check("dqt_unpack_ternary", load().dqt_unpack_ternary(packed.ctypes.data, rows, cols,
                                                           q.ctypes.data))
    return q
