"""ctypes binding of libhstu (include/hstu.h), argument marshalling only.

Each C entry point has a Python function of the same name that takes
torch tensors (device memory) and passes their data pointers, strides and
the current HIP stream.  Every step of the computation runs in the HIP
kernels of libhstu.so; if the library is missing or fails to load, import
of this module raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libhstu.so")

HSTU_F32, HSTU_BF16 = 0, 1
STATUS = {0: "HSTU_OK", 1: "HSTU_ERR_INVALID_ARGUMENT", 2: "HSTU_ERR_UNSUPPORTED",
          3: "HSTU_ERR_WORKSPACE", 4: "HSTU_ERR_HIP", 5: "HSTU_ERR_DATA"}

EXPORTED = ("hstu_workspace_bytes", "hstu_attn_fwd", "hstu_attn_bwd", "hstu_layer_fwd",
            "hstu_time_bucketize", "hstu_complete_cumsum", "hstu_pair_offsets", "hstu_validate",
            "hstu_last_error", "hstu_abi_version", "hstu_timing_enable", "hstu_timing_read",
            "hstu_timing_reset", "hstu_probe_mfma_bf16", "hstu_layer_bwd",
            "hstu_attn_fwd_cached", "hstu_attn_fwd_cached_workspace_bytes",
            "hstu_proj_workspace_bytes", "hstu_proj_in_fwd",
            "hstu_proj_out_fwd", "hstu_proj_out_bwd", "hstu_proj_in_bwd",
            "hstu_sl_subseq_len", "hstu_sl_keep_numerator", "hstu_sl_workspace_bytes",
            "hstu_stochastic_length", "hstu_gather_rows", "hstu_sl_sparsity",
            "hstu_attn_fwd_noalloc",
            "hstu_rotary_frequencies", "hstu_rotary_fwd", "hstu_rotary_bwd",
            "hstu_cache_write", "hstu_cache_read", "hstu_cache_validate",
            "hstu_attn_fwd_tree_workspace_bytes", "hstu_attn_fwd_tree", "hstu_tree_positions")


class Problem(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("total_tokens", ctypes.c_int64),
                ("max_seq_len", ctypes.c_int32), ("num_heads", ctypes.c_int32),
                ("d_qk", ctypes.c_int32), ("d_v", ctypes.c_int32),
                ("num_time_buckets", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Jagged(ctypes.Structure):
    _fields_ = [("seq_offsets", ctypes.c_void_p), ("timestamps", ctypes.c_void_p),
                ("num_targets", ctypes.c_void_p), ("rab_pos", ctypes.c_void_p),
                ("rab_time", ctypes.c_void_p)]


class CacheDesc(ctypes.Structure):
    _fields_ = [("num_pages", ctypes.c_int64), ("page_size", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("timestamps", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("lengths", ctypes.c_void_p)]


class HstuError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
    lib = ctypes.CDLL(LIB_PATH)
    P, i32, i64, sz, f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
                            ctypes.c_float)
    PP, PJ, PC = (ctypes.POINTER(Problem), ctypes.POINTER(Jagged), ctypes.POINTER(CacheDesc))
    f64 = ctypes.c_double
    sig = {
        "hstu_workspace_bytes": (sz, [PP]),
        "hstu_attn_fwd": (i32, [PP, PJ, P, i64, P, i64, P, i64, P, P, sz, P]),
        "hstu_attn_bwd": (i32, [PP, PJ, P, i64, P, i64, P, i64, P, P, P, P, P, P, P, sz, P]),
        "hstu_layer_fwd": (i32, [PP, PJ, P, i64, P, i64, P, i64, P, i64, P, P, f32, P, P, P, P,
                                 P, sz, P]),
        "hstu_layer_bwd": (i32, [PP, PJ, P, i64, P, i64, P, i64, P, i64, P, P, P, P, P, P,
                                 P, P, P, P, P, P, P, P, P, sz, P]),
        "hstu_attn_fwd_cached": (i32, [PP, PJ, P, i64, P, i64, P, i64, P, P, i64, P, i64, P, i64,
                                       P, P, sz, P]),
        "hstu_time_bucketize": (i32, [i32, i64, i32, P, P, P, i64, P, P]),
        "hstu_complete_cumsum": (i32, [i32, P, P, P]),
        "hstu_pair_offsets": (i32, [i32, P, P, P]),
        "hstu_validate": (i32, [PP, PJ, P]),
        "hstu_last_error": (ctypes.c_char_p, []),
        "hstu_abi_version": (i32, []),
        "hstu_timing_enable": (i32, [i32]),
        "hstu_timing_read": (i32, [ctypes.c_char_p, ctypes.POINTER(ctypes.c_double),
                                   ctypes.POINTER(ctypes.c_int64)]),
        "hstu_timing_reset": (i32, []),
        "hstu_probe_mfma_bf16": (i32, [i32, i32, P, ctypes.POINTER(ctypes.c_double), P]),
        "hstu_proj_workspace_bytes": (sz, [PP, i32]),
        "hstu_attn_fwd_cached_workspace_bytes": (sz, [PP]),
        "hstu_sl_subseq_len": (i32, [i32, ctypes.c_double]),
        "hstu_sl_keep_numerator": (ctypes.c_double, [i32, ctypes.c_double]),
        "hstu_attn_fwd_noalloc": (i32, [PP, PJ, P, i64, P, i64, P, i64, P, P]),
        "hstu_sl_workspace_bytes": (sz, [i32]),
        "hstu_stochastic_length": (i32, [i32, P, P, P, i32, ctypes.c_double, i32, P, P, P, P, P,
                                         sz, P]),
        "hstu_gather_rows": (i32, [P, i64, i64, P, P, i64, P, i64, P]),
        "hstu_sl_sparsity": (i32, [i32, P, i32, ctypes.POINTER(ctypes.c_double),
                                   ctypes.POINTER(ctypes.c_double)]),
        "hstu_proj_in_fwd": (i32, [PP, i32, P, i64, P, P, P, P, P]),
        "hstu_proj_out_fwd": (i32, [PP, i32, P, i64, P, P, P, P, P]),
        "hstu_proj_out_bwd": (i32, [PP, i32, P, i64, P, P, P, P, P, P, sz, P]),
        "hstu_proj_in_bwd": (i32, [PP, i32, P, i64, P, P, P, P, P, P, P, P, P, P, P, sz, P]),
        "hstu_rotary_frequencies": (i32, [i32, f64, i32, f64, f64, f64, f64, P]),
        "hstu_rotary_fwd": (i32, [PP, P, P, P, P, i32, i32, f32, P, i64, P, i64, P, P, P]),
        "hstu_rotary_bwd": (i32, [PP, P, P, P, P, i32, i32, f32, P, i64, P, i64, P, P, P]),
        "hstu_cache_write": (i32, [PP, PC, P, P, P, P, i64, P, i64, P]),
        "hstu_cache_read": (i32, [PP, PC, P, P, P, P, P, P]),
        "hstu_cache_validate": (i32, [PP, PC, P]),
        "hstu_attn_fwd_tree_workspace_bytes": (sz, [PP, PC, i32]),
        "hstu_attn_fwd_tree": (i32, [PP, PJ, PC, P, i32, P, i64, P, i64, P, i64, P, P, sz, P]),
        "hstu_tree_positions": (i32, [i32, i64, i32, P, P, P, P, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


def _check(status: int):
    if status != 0:
        raise HstuError(status, lib.hstu_last_error().decode())


# The marshalling below is on the path of every call; small calls are bound by
# it (attention forward + backward on two sequences of 60 tokens: 46 us of host
# time, 35 us of kernels), so pointers and streams travel as plain integers and
# outputs come from new_empty.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# The handle of the current stream without a Stream object around it.  Both are
# torch's own, undocumented: where one is missing the public call serves.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
        return _raw_stream(_raw_device())
    return torch.cuda.current_stream().cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return HSTU_BF16
    if t.dtype == torch.float32:
        return HSTU_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _row_stride(t: torch.Tensor) -> int:
    """Row stride in elements of a [T, h, d] (or [T, h*d]) view whose rows
    are [h][d]-contiguous."""
    st = t.stride()
    if len(st) == 3:
        if st[2] != 1 or st[1] != t.shape[2]:
            raise ValueError("rows must be [h][d] contiguous")
    elif len(st) == 2:
        if st[1] != 1:
            raise ValueError("rows must be contiguous")
    else:
        raise ValueError("expected a [T, h, d] or [T, h*d] tensor")
    return st[0]


def make_problem(num_seqs, total_tokens, max_seq_len, num_heads, d_qk, d_v, num_time_buckets,
                 dtype) -> Problem:
    return Problem(int(num_seqs), int(total_tokens), int(max_seq_len), int(num_heads), int(d_qk),
                   int(d_v), int(num_time_buckets), int(dtype))


def make_jagged(seq_offsets, timestamps, rab_pos, rab_time, num_targets=None) -> Jagged:
    return Jagged(seq_offsets.data_ptr(), timestamps.data_ptr(),
                  None if num_targets is None else num_targets.data_ptr(),
                  rab_pos.data_ptr(), rab_time.data_ptr())


def problem_for(q, v, seq_offsets, max_seq_len, rab_time) -> Problem:
    T, H, dqk = q.shape
    dv = v.shape[2]
    return make_problem(seq_offsets.numel() - 1, T, max_seq_len, H, dqk, dv, rab_time.numel(),
                        _dtype_code(q))


# ---------------------------------------------------------------- raw names

def hstu_abi_version() -> int:
    return int(lib.hstu_abi_version())


def hstu_last_error() -> str:
    return lib.hstu_last_error().decode()


def hstu_workspace_bytes(problem: Problem) -> int:
    return int(lib.hstu_workspace_bytes(ctypes.byref(problem)))


def workspace(problem: Problem, device=None) -> torch.Tensor:
    n = hstu_workspace_bytes(problem)
    if n == 0:
        raise HstuError(1, "invalid problem")
    return torch.empty(n, dtype=torch.uint8, device=device or "cuda")


def hstu_attn_fwd(q, k, v, seq_offsets, timestamps, rab_pos, rab_time, max_seq_len,
                  num_targets=None, out=None, ws=None, stream=None):
    """O [T, h, d_v] of Eq. 2 (see include/hstu.h)."""
    p = problem_for(q, v, seq_offsets, max_seq_len, rab_time)
    j = make_jagged(seq_offsets, timestamps, rab_pos, rab_time, num_targets)
    if out is None:
        out = q.new_empty((p.total_tokens, p.num_heads, p.d_v))
    if ws is None:
        ws = workspace(p, q.device)
    _check(lib.hstu_attn_fwd(ctypes.byref(p), ctypes.byref(j), _ptr(q), _row_stride(q), _ptr(k),
                             _row_stride(k), _ptr(v), _row_stride(v), _ptr(out), _ptr(ws),
                             ws.numel(), _stream(stream)))
    return out


def hstu_attn_fwd_noalloc(q, k, v, seq_offsets, timestamps, rab_pos, rab_time, max_seq_len, out,
                          num_targets=None, stream=None):
    """hstu_attn_fwd with its scratch in the library's static device array
    (no workspace; `out` [T, h, d_v] is required, nothing is allocated)."""
    p = problem_for(q, v, seq_offsets, max_seq_len, rab_time)
    j = make_jagged(seq_offsets, timestamps, rab_pos, rab_time, num_targets)
    _check(lib.hstu_attn_fwd_noalloc(ctypes.byref(p), ctypes.byref(j), _ptr(q), _row_stride(q),
                                     _ptr(k), _row_stride(k), _ptr(v), _row_stride(v), _ptr(out),
                                     _stream(stream)))
    return out


def hstu_attn_fwd_cached_workspace_bytes(problem: Problem) -> int:
    return int(lib.hstu_attn_fwd_cached_workspace_bytes(ctypes.byref(problem)))


def cached_workspace(problem: Problem, device=None) -> torch.Tensor:
    n = hstu_attn_fwd_cached_workspace_bytes(problem)
    if n == 0:
        raise HstuError(1, "invalid problem")
    return torch.empty(n, dtype=torch.uint8, device=device or "cuda")


def hstu_attn_fwd_cached(q, k, v, seq_offsets, timestamps, k_cache, v_cache, cache_offsets,
                         cache_timestamps, rab_pos, rab_time, max_seq_len, out=None, ws=None,
                         stream=None):
    """O [T, h, d_v] of the candidate rows q, k, v (offsets seq_offsets) against
    the cached history keys and values k_cache, v_cache (offsets
    cache_offsets); see include/hstu.h."""
    p = problem_for(q, v, seq_offsets, max_seq_len, rab_time)
    j = make_jagged(seq_offsets, timestamps, rab_pos, rab_time, None)
    if out is None:
        out = q.new_empty((p.total_tokens, p.num_heads, p.d_v))
    if ws is None:
        ws = cached_workspace(p, q.device)
    _check(lib.hstu_attn_fwd_cached(ctypes.byref(p), ctypes.byref(j), _ptr(q), _row_stride(q),
                                    _ptr(k), _row_stride(k), _ptr(v), _row_stride(v),
                                    _ptr(cache_offsets), _ptr(cache_timestamps),
                                    int(k_cache.shape[0]), _ptr(k_cache), _row_stride(k_cache),
                                    _ptr(v_cache), _row_stride(v_cache), _ptr(out), _ptr(ws),
                                    ws.numel(), _stream(stream)))
    return out


def hstu_attn_bwd(q, k, v, d_out, seq_offsets, timestamps, rab_pos, rab_time, max_seq_len,
                  num_targets=None, grads=None, ws=None, stream=None):
    """(dq, dk, dv, d_rab_pos, d_rab_time) for the loss <O, d_out>."""
    p = problem_for(q, v, seq_offsets, max_seq_len, rab_time)
    j = make_jagged(seq_offsets, timestamps, rab_pos, rab_time, num_targets)
    if grads is None:
        T, H = p.total_tokens, p.num_heads
        grads = (q.new_empty((T, H, p.d_qk)), q.new_empty((T, H, k.shape[2])),
                 q.new_empty((T, H, p.d_v)), torch.empty_like(rab_pos),
                 torch.empty_like(rab_time))
    dq, dk, dv, drp, drt = grads
    if ws is None:
        ws = workspace(p, q.device)
    _check(lib.hstu_attn_bwd(ctypes.byref(p), ctypes.byref(j), _ptr(q), _row_stride(q), _ptr(k),
                             _row_stride(k), _ptr(v), _row_stride(v), _ptr(d_out), _ptr(dq),
                             _ptr(dk), _ptr(dv), _ptr(drp), _ptr(drt), _ptr(ws), ws.numel(),
                             _stream(stream)))
    return grads


def hstu_layer_fwd(q, k, v, u, seq_offsets, timestamps, rab_pos, rab_time, max_seq_len,
                   num_targets=None, ln_weight=None, ln_bias=None, ln_eps=1e-5, attn_out=None,
                   y=None, ln_mean=None, ln_rstd=None, ws=None, stream=None):
    """(attn_out [T, D] fp32, y [T, D], ln_mean [T], ln_rstd [T]) of Eq. 2-3."""
    p = problem_for(q, v, seq_offsets, max_seq_len, rab_time)
    j = make_jagged(seq_offsets, timestamps, rab_pos, rab_time, num_targets)
    T, D = p.total_tokens, p.num_heads * p.d_v
    if attn_out is None:
        attn_out = q.new_empty((T, D), dtype=torch.float32)
    if y is None:
        y = q.new_empty((T, D))
    if ln_mean is None:
        ln_mean = q.new_empty(T, dtype=torch.float32)
    if ln_rstd is None:
        ln_rstd = q.new_empty(T, dtype=torch.float32)
    if ws is None:
        ws = workspace(p, q.device)
    _check(lib.hstu_layer_fwd(ctypes.byref(p), ctypes.byref(j), _ptr(q), _row_stride(q), _ptr(k),
                              _row_stride(k), _ptr(v), _row_stride(v), _ptr(u), _row_stride(u),
                              _ptr(ln_weight), _ptr(ln_bias), float(ln_eps), _ptr(attn_out),
                              _ptr(y), _ptr(ln_mean), _ptr(ln_rstd), _ptr(ws), ws.numel(),
                              _stream(stream)))
    return attn_out, y, ln_mean, ln_rstd


def hstu_layer_bwd(q, k, v, u, attn_out, ln_mean, ln_rstd, d_y, seq_offsets, timestamps,
                   rab_pos, rab_time, max_seq_len, num_targets=None, ln_weight=None,
                   ln_bias=None, want_ln_grads=None, grads=None, ws=None, stream=None):
    """(dq, dk, dv, du, d_ln_weight, d_ln_bias, d_rab_pos, d_rab_time) for the
    loss <Y, d_y> of Eq. 2-3; attn_out, ln_mean, ln_rstd from hstu_layer_fwd.
    d_ln_weight / d_ln_bias are computed when want_ln_grads (default: when
    ln_weight is given), else None."""
    p = problem_for(q, v, seq_offsets, max_seq_len, rab_time)
    j = make_jagged(seq_offsets, timestamps, rab_pos, rab_time, num_targets)
    T, D = p.total_tokens, p.num_heads * p.d_v
    if want_ln_grads is None:
        want_ln_grads = ln_weight is not None
    if grads is None:
        H = q.shape[1]
        grads = (q.new_empty((T, H, p.d_qk)), q.new_empty((T, H, k.shape[2])),
                 q.new_empty((T, H, p.d_v)), q.new_empty((T, D)),
                 q.new_empty(D, dtype=torch.float32) if want_ln_grads else None,
                 q.new_empty(D, dtype=torch.float32) if want_ln_grads else None,
                 torch.empty_like(rab_pos), torch.empty_like(rab_time))
    dq, dk, dv, du, dw, db, drp, drt = grads
    if ws is None:
        ws = workspace(p, q.device)
    _check(lib.hstu_layer_bwd(ctypes.byref(p), ctypes.byref(j), _ptr(q), _row_stride(q), _ptr(k),
                              _row_stride(k), _ptr(v), _row_stride(v), _ptr(u), _row_stride(u),
                              _ptr(attn_out), _ptr(ln_weight), _ptr(ln_bias), _ptr(ln_mean),
                              _ptr(ln_rstd), _ptr(d_y), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(du),
                              _ptr(dw), _ptr(db), _ptr(drp), _ptr(drt), _ptr(ws), ws.numel(),
                              _stream(stream)))
    return grads


def hstu_complete_cumsum(x: torch.Tensor, out=None, stream=None):
    if out is None:
        out = torch.empty(x.numel() + 1, dtype=torch.int64, device=x.device)
    _check(lib.hstu_complete_cumsum(x.numel(), _ptr(x), _ptr(out), _stream(stream)))
    return out


def hstu_pair_offsets(seq_offsets: torch.Tensor, out=None, stream=None):
    if out is None:
        out = torch.empty_like(seq_offsets)
    _check(lib.hstu_pair_offsets(seq_offsets.numel() - 1, _ptr(seq_offsets), _ptr(out),
                                 _stream(stream)))
    return out


def hstu_time_bucketize(seq_offsets, timestamps, num_time_buckets, pair_offsets=None,
                        total_pairs=None, out=None, stream=None):
    """uint8 buckets, one L_b x L_b row-major matrix per sequence."""
    if pair_offsets is None:
        pair_offsets = hstu_pair_offsets(seq_offsets, stream=stream)
    if total_pairs is None:
        total_pairs = int(pair_offsets[-1].item())  # host read, synchronises
    if out is None:
        out = torch.empty(max(total_pairs, 1), dtype=torch.uint8, device=timestamps.device)
    _check(lib.hstu_time_bucketize(seq_offsets.numel() - 1, timestamps.numel(),
                                   int(num_time_buckets), _ptr(seq_offsets), _ptr(timestamps),
                                   _ptr(pair_offsets), int(total_pairs), _ptr(out),
                                   _stream(stream)))
    return out[:total_pairs]


def hstu_validate(seq_offsets, timestamps, rab_pos, rab_time, max_seq_len, num_heads, d_qk, d_v,
                  dtype=HSTU_BF16, num_targets=None, stream=None):
    p = make_problem(seq_offsets.numel() - 1, timestamps.numel(), max_seq_len, num_heads, d_qk,
                     d_v, rab_time.numel(), dtype)
    j = make_jagged(seq_offsets, timestamps, rab_pos, rab_time, num_targets)
    _check(lib.hstu_validate(ctypes.byref(p), ctypes.byref(j), _stream(stream)))


def hstu_timing_enable(on: bool = True):
    _check(lib.hstu_timing_enable(1 if on else 0))


def hstu_timing_reset():
    _check(lib.hstu_timing_reset())


# ------------------------------------------------ linear maps (Eq. 1, Eq. 3)

def proj_problem(x, num_heads, d_qk, d_v) -> Problem:
    """Problem of a projection call: only T, h, d_qk, d_v and the dtype
    matter (one placeholder sequence, N = 1, one time bucket)."""
    return make_problem(1, x.shape[0], 1, num_heads, d_qk, d_v, 1, _dtype_code(x))


def _row_stride2(t: torch.Tensor) -> int:
    if t.dim() == 2 and t.shape[0] == 0:
        return t.shape[1]
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("expected a [T, width] tensor with contiguous rows")
    return t.stride(0)


def hstu_proj_workspace_bytes(p: Problem, d_model: int) -> int:
    return int(lib.hstu_proj_workspace_bytes(ctypes.byref(p), int(d_model)))


def proj_workspace(p: Problem, d_model: int, device=None) -> torch.Tensor:
    n = int(lib.hstu_proj_workspace_bytes(ctypes.byref(p), int(d_model)))
    if n == 0:
        raise HstuError(1, "invalid projection problem")
    return torch.empty(n, dtype=torch.uint8, device=device or "cuda")


def hstu_proj_in_fwd(x, w1, b1, num_heads, d_qk, d_v, z=None, z_pre=None, want_pre=True,
                     stream=None):
    """Eq. 1: returns (z, z_pre), z [T, F] = SiLU(x w1^T + b1) laid out U|V|Q|K."""
    p = proj_problem(x, num_heads, d_qk, d_v)
    F = 2 * num_heads * (d_qk + d_v)
    if z is None:
        z = torch.empty((x.shape[0], F), dtype=x.dtype, device=x.device)
    if z_pre is None and want_pre:
        z_pre = torch.empty_like(z)
    _check(lib.hstu_proj_in_fwd(ctypes.byref(p), int(x.shape[1]), _ptr(x), _row_stride2(x),
                                _ptr(w1), _ptr(b1), _ptr(z), _ptr(z_pre), _stream(stream)))
    return z, z_pre


def split_uvqk(z, num_heads, d_qk, d_v):
    """[T, h, d] views U, V, Q, K of z [T, F] (row stride F)."""
    T = z.shape[0]
    hv, hq = num_heads * d_v, num_heads * d_qk
    F = z.shape[1]

    def view(c0, d):
        return z.as_strided((T, num_heads, d), (F, d, 1), z.storage_offset() + c0)
    return view(0, d_v), view(hv, d_v), view(2 * hv, d_qk), view(2 * hv + hq, d_qk)


def hstu_proj_out_fwd(g, w2, b2, residual, num_heads, d_qk, d_v, y=None, stream=None):
    """Eq. 3's f_2 plus the residual: y [T, D] = g w2^T + b2 + residual."""
    p = proj_problem(g, num_heads, d_qk, d_v)
    D = w2.shape[0]
    if y is None:
        y = torch.empty((g.shape[0], D), dtype=g.dtype, device=g.device)
    _check(lib.hstu_proj_out_fwd(ctypes.byref(p), int(D), _ptr(g), _row_stride2(g), _ptr(w2),
                                 _ptr(b2), _ptr(residual), _ptr(y), _stream(stream)))
    return y


def hstu_proj_out_bwd(g, w2, dy, num_heads, d_qk, d_v, want_db=True, out=None, ws=None,
                      stream=None):
    """Returns (dg, dw2, db2) for the loss <y, dy>."""
    p = proj_problem(g, num_heads, d_qk, d_v)
    D, hv = w2.shape
    if out is None:
        out = (torch.empty((g.shape[0], hv), dtype=g.dtype, device=g.device),
               torch.empty((D, hv), dtype=torch.float32, device=g.device),
               torch.empty(D, dtype=torch.float32, device=g.device) if want_db else None)
    dg, dw2, db2 = out
    if ws is None:
        ws = proj_workspace(p, D, g.device)
    _check(lib.hstu_proj_out_bwd(ctypes.byref(p), int(D), _ptr(g), _row_stride2(g), _ptr(w2),
                                 _ptr(dy), _ptr(dg), _ptr(dw2), _ptr(db2), _ptr(ws), ws.numel(),
                                 _stream(stream)))
    return dg, dw2, db2


def hstu_proj_in_bwd(x, w1, z_pre, du, dv, dq, dk, num_heads, d_qk, d_v, dx_add=None,
                     want_db=True, out=None, ws=None, stream=None):
    """Returns (dx, dw1, db1) for the loss <z, [du|dv|dq|dk]>."""
    p = proj_problem(x, num_heads, d_qk, d_v)
    F, D = w1.shape
    if out is None:
        out = (torch.empty_like(x, memory_format=torch.contiguous_format),
               torch.empty((F, D), dtype=torch.float32, device=x.device),
               torch.empty(F, dtype=torch.float32, device=x.device) if want_db else None)
    dx, dw1, db1 = out
    if ws is None:
        ws = proj_workspace(p, D, x.device)
    _check(lib.hstu_proj_in_bwd(ctypes.byref(p), int(D), _ptr(x), _row_stride2(x), _ptr(w1),
                                _ptr(z_pre), _ptr(du), _ptr(dv), _ptr(dq), _ptr(dk),
                                _ptr(dx_add), _ptr(dx), _ptr(dw1), _ptr(db1), _ptr(ws),
                                ws.numel(), _stream(stream)))
    return dx, dw1, db1


# ------------------------------------------------ Stochastic Length (Eq. 4)

HSTU_SL_GREEDY, HSTU_SL_RANDOM, HSTU_SL_WEIGHTED = 0, 1, 2


def hstu_sl_subseq_len(max_seq_len: int, alpha: float) -> int:
    return int(lib.hstu_sl_subseq_len(int(max_seq_len), float(alpha)))


def hstu_sl_keep_numerator(max_seq_len: int, alpha: float) -> float:
    return float(lib.hstu_sl_keep_numerator(int(max_seq_len), float(alpha)))


def hstu_sl_workspace_bytes(num_seqs: int) -> int:
    return int(lib.hstu_sl_workspace_bytes(int(num_seqs)))


def hstu_stochastic_length(seq_offsets, timestamps, subseq_len, keep_numerator, selection, u_keep,
                           e_rand=None, num_targets=None, out=None, ws=None, stream=None):
    """(new_offsets [B+1], gather [T]) on the device; the first
    new_offsets[B] entries of gather are valid (see include/hstu.h)."""
    B = seq_offsets.numel() - 1
    T = timestamps.numel()
    if out is None:
        out = (torch.empty(B + 1, dtype=torch.int64, device=seq_offsets.device),
               torch.empty(max(T, 1), dtype=torch.int64, device=seq_offsets.device))
    new_offsets, gather = out
    if ws is None:
        ws = torch.empty(int(lib.hstu_sl_workspace_bytes(B)), dtype=torch.uint8,
                         device=seq_offsets.device)
    _check(lib.hstu_stochastic_length(B, _ptr(seq_offsets), _ptr(timestamps), _ptr(num_targets),
                                      int(subseq_len), float(keep_numerator), int(selection),
                                      _ptr(u_keep), _ptr(e_rand),
                                      _ptr(new_offsets), _ptr(gather), _ptr(ws), ws.numel(),
                                      _stream(stream)))
    return new_offsets, gather


def hstu_gather_rows(src, gather, count, max_rows=None, dst=None, stream=None):
    """dst[r] = src[gather[r]] for r < count[0] (a one-element device tensor,
    e.g. new_offsets[-1:]); src rows are its first dimension."""
    rows = src.shape[0]
    row_elems = src.numel() // rows if rows else int(np.prod(src.shape[1:]))
    if max_rows is None:
        max_rows = gather.numel()
    if dst is None:
        dst = torch.empty((max_rows,) + tuple(src.shape[1:]), dtype=src.dtype, device=src.device)
    es = src.element_size()
    _check(lib.hstu_gather_rows(_ptr(src), src.stride(0) * es, row_elems * es, _ptr(gather),
                                _ptr(count), int(max_rows), _ptr(dst), dst.stride(0) * es,
                                _stream(stream)))
    return dst


def hstu_sl_sparsity(seq_offsets_host, max_seq_len):
    """(sparsity, s2) of a batch from host int64 offsets."""
    offs = np.ascontiguousarray(seq_offsets_host, dtype=np.int64)
    sp, s2 = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(lib.hstu_sl_sparsity(len(offs) - 1, offs.ctypes.data_as(ctypes.c_void_p),
                                int(max_seq_len), ctypes.byref(sp), ctypes.byref(s2)))
    return sp.value, s2.value


# ------------------------------------------------ rotary positions

HSTU_ROTARY_HALVES, HSTU_ROTARY_INTERLEAVED = 0, 1
ROTARY_SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}


def _array(name, t, dtype, count=None):
    """Data pointer of a dense device array argument (None stays None)."""
    if t is None:
        return None
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if count is not None and t.numel() != count:
        raise ValueError(f"{name} must have {count} elements, got {t.numel()}")
    return t.data_ptr()


def _offsets(seq_offsets):
    """(pointer, number of sequences) of an offsets array."""
    ptr = _array("seq_offsets", seq_offsets, torch.int64)
    if seq_offsets.numel() < 2:
        raise ValueError("seq_offsets needs an entry for each sequence and one more")
    return ptr, seq_offsets.numel() - 1


def _rows(name, t, shape, dtype):
    """Row stride of a [T, h, d] view of the given shape and dtype."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}, got {tuple(t.shape)}")
    st = t.stride()
    if st[2] != 1 or (shape[1] > 1 and st[1] != shape[2]):
        raise ValueError(f"{name}: rows must be [h][d] contiguous")
    # a single row, or none, has no stride to speak of
    return st[0] if shape[0] > 1 else max(st[0], shape[1] * shape[2])


def _dense_out(name, out, like, shape, dtype):
    if out is None:
        return like.new_empty(shape) if like.dtype == dtype else like.new_empty(shape, dtype=dtype)
    if out.dtype != dtype or out.shape != torch.Size(shape) or not out.is_contiguous():
        raise ValueError(f"{name} must be contiguous {tuple(shape)} of {dtype}")
    return out


def _on_device(*tensors):
    """The launches go to the current device: every array has to lie there."""
    device = _raw_device() if _raw_device is not None else torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:  # -1 on the CPU
            raise ValueError(f"an array is on {t.device}, the current device is cuda:{device}")


def hstu_rotary_frequencies(rot_dim, base=10000.0, scaling="none", factor=1.0, original_len=0.0,
                            low=1.0, high=32.0):
    """Inverse frequencies (numpy float64 [rot_dim / 2], host); scaling: "none",
    "linear", "base" or "parts" (see include/hstu.h)."""
    out = np.empty(max(int(rot_dim) // 2, 0), dtype=np.float64)
    _check(lib.hstu_rotary_frequencies(int(rot_dim), float(base), ROTARY_SCALINGS[scaling],
                                       float(factor), float(original_len), float(low),
                                       float(high), out.ctypes.data_as(ctypes.c_void_p)))
    return out


def _rotary(call, q, k, inv_freq, seq_offsets, num_targets, positions, interleaved, amplitude,
            out, stream):
    one = q if q is not None else k
    if one is None:
        raise ValueError("q and k are both None")
    if one.dim() != 3:
        raise ValueError("expected a [T, h, d] tensor")
    shape, dtype = one.shape, one.dtype
    T, H, d = shape
    code = _dtype_code(one)
    qs = 0 if q is None else _rows("q", q, shape, dtype)
    ks = 0 if k is None else _rows("k", k, shape, dtype)
    freq = _array("inv_freq", inv_freq, torch.float64)
    pos = _array("positions", positions, torch.int64, T)
    offs, B = (None, 1) if seq_offsets is None else _offsets(seq_offsets)
    nt = _array("num_targets", num_targets, torch.int64, B)
    qo, ko = (None, None) if out is None else out
    qo = None if q is None else _dense_out("q output", qo, q, shape, dtype)
    ko = None if k is None else _dense_out("k output", ko, k, shape, dtype)
    _on_device(q, k, inv_freq, positions, seq_offsets, num_targets, qo, ko)
    p = Problem(B, T, 1, H, d, d, 1, code)
    _check(call(ctypes.byref(p), offs, nt, pos, freq, 2 * inv_freq.numel(),
                1 if interleaved else 0, amplitude, _ptr(q), qs, _ptr(k), ks, _ptr(qo), _ptr(ko),
                _stream(stream)))
    return qo, ko


def hstu_rotary_fwd(q, k, inv_freq, seq_offsets=None, num_targets=None, positions=None,
                    interleaved=False, amplitude=1.0, out=None, stream=None):
    """(q', k') dense [T, h, d]: the first 2 * inv_freq.numel() features of each
    head turned by position * inv_freq (float64, device).  Either of q and k may
    be None.  Positions: given, or the index in the sequence (see
    include/hstu.h)."""
    return _rotary(lib.hstu_rotary_fwd, q, k, inv_freq, seq_offsets, num_targets, positions,
                   interleaved, amplitude, out, stream)


def hstu_rotary_bwd(d_q_out, d_k_out, inv_freq, seq_offsets=None, num_targets=None,
                    positions=None, interleaved=False, amplitude=1.0, out=None, stream=None):
    """(dq, dk) for the gradients of hstu_rotary_fwd's outputs."""
    return _rotary(lib.hstu_rotary_bwd, d_q_out, d_k_out, inv_freq, seq_offsets, num_targets,
                   positions, interleaved, amplitude, out, stream)


# ------------------------------------------------ paged cache

HSTU_CACHE_BF16, HSTU_CACHE_E4M3, HSTU_CACHE_INT8 = 0, 1, 2
_CACHE_CODES = {torch.bfloat16: HSTU_CACHE_BF16, torch.float8_e4m3fn: HSTU_CACHE_E4M3,
                torch.int8: HSTU_CACHE_INT8}


class PagedCache:
    """The device arrays of a paged cache (hstu_cache_t in include/hstu.h):
    k [pages, h, page, d_qk], v [pages, h, d_v, page] of bfloat16,
    float8_e4m3fn or int8, k_scale and v_scale [pages, h, page] (None for
    bfloat16), timestamps [pages, page], page_table [B, max_pages] int32,
    lengths [B] int64.  The arrays are the caller's; they are changed in place,
    never exchanged: other arrays are another PagedCache."""

    __slots__ = ("_arrays", "_desc", "_shape")

    def __init__(self, k, v, timestamps, page_table, lengths, k_scale=None, v_scale=None):
        kind = _CACHE_CODES.get(k.dtype)
        if kind is None or v.dtype != k.dtype:
            raise TypeError(f"a cache of {k.dtype} and {v.dtype} is not supported")
        if k.dim() != 4 or v.dim() != 4 or page_table.dim() != 2:
            raise ValueError("k and v have four dimensions, page_table has two")
        pages, heads, page, d_qk = k.shape
        d_v = v.shape[2]
        if v.shape != (pages, heads, d_v, page):
            raise ValueError(f"v must be {(pages, heads, d_v, page)}, got {tuple(v.shape)}")
        if timestamps.shape != (pages, page):
            raise ValueError(f"timestamps must be {(pages, page)}")
        B, width = page_table.shape
        if (k_scale is None) != (kind == HSTU_CACHE_BF16) or (v_scale is None) != (k_scale is None):
            raise ValueError("scales belong to a quantised cache, to both of k and v")
        if k_scale is not None and (k_scale.shape != (pages, heads, page)
                                    or v_scale.shape != (pages, heads, page)):
            raise ValueError(f"scales must be {(pages, heads, page)}")
        device = k.get_device()
        for t in (v, timestamps, page_table, lengths, k_scale, v_scale):
            if t is not None and t.get_device() != device:
                raise ValueError(f"the cache's arrays are on {k.device} and {t.device}")
        self._arrays = (k, v, timestamps, page_table, lengths, k_scale, v_scale)
        self._shape = (B, heads, d_qk, d_v)
        self._desc = CacheDesc(pages, page, width, kind, _array("k", k, k.dtype),
                               _array("v", v, v.dtype),
                               _array("k_scale", k_scale, torch.float32),
                               _array("v_scale", v_scale, torch.float32),
                               _array("timestamps", timestamps, torch.int64),
                               _array("page_table", page_table, torch.int32),
                               _array("lengths", lengths, torch.int64, B))

    k, v, timestamps, page_table, lengths, k_scale, v_scale = (
        property(lambda self, i=i: self._arrays[i]) for i in range(7))


def alloc_cache(num_pages, page_size, num_heads, d_qk, d_v, num_seqs, max_pages,
                dtype=torch.float8_e4m3fn, device=None) -> PagedCache:
    """An empty cache: no user owns a page (page_table -1) or a token."""
    device = device or "cuda"

    def make(dt, *shape):
        return torch.empty(shape, dtype=dt, device=device)
    scales = [None if dtype == torch.bfloat16 else
              make(torch.float32, num_pages, num_heads, page_size) for _ in range(2)]
    return PagedCache(make(dtype, num_pages, num_heads, page_size, d_qk),
                      make(dtype, num_pages, num_heads, d_v, page_size),
                      make(torch.int64, num_pages, page_size),
                      torch.full((num_seqs, max_pages), -1, dtype=torch.int32, device=device),
                      torch.zeros(num_seqs, dtype=torch.int64, device=device), *scales)


def _cache_batch(cache, seq_offsets):
    offs, B = _offsets(seq_offsets)
    if B != cache._shape[0]:
        raise ValueError(f"{B} sequences, but a cache of {cache._shape[0]}")
    return offs, B


def hstu_cache_write(k, v, timestamps, seq_offsets, cache, starts=None, stream=None):
    """Writes rows k [T, h, d_qk], v [T, h, d_v] and their timestamps into the
    cache, token i of sequence b at position starts[b] + i (starts None: i).
    cache.lengths stays as it is."""
    offs, B = _cache_batch(cache, seq_offsets)
    _, H, dqk, dv = cache._shape
    T = k.shape[0]
    code = _dtype_code(k)
    ks = _rows("k", k, (T, H, dqk), k.dtype)
    vs = _rows("v", v, (T, H, dv), k.dtype)
    ts = _array("timestamps", timestamps, torch.int64, T)
    st = _array("starts", starts, torch.int64, B)
    _on_device(k, v, timestamps, seq_offsets, starts, cache.k)
    p = Problem(B, T, 1, H, dqk, dv, 1, code)
    _check(lib.hstu_cache_write(ctypes.byref(p), ctypes.byref(cache._desc), offs, st, ts, _ptr(k),
                                ks, _ptr(v), vs, _stream(stream)))


def hstu_cache_read(cache, seq_offsets, total_tokens, starts=None, dtype=torch.bfloat16, out=None,
                    stream=None):
    """(k [T, h, d_qk], v [T, h, d_v], timestamps [T]): row seq_offsets[b] + i is
    position starts[b] + i of user b (total_tokens = seq_offsets[-1])."""
    offs, B = _cache_batch(cache, seq_offsets)
    _, H, dqk, dv = cache._shape
    T = int(total_tokens)
    st = _array("starts", starts, torch.int64, B)
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype}")
    k, v, ts = (None, None, None) if out is None else out
    k = _dense_out("k", k, cache.k, (T, H, dqk), dtype)
    v = _dense_out("v", v, cache.k, (T, H, dv), dtype)
    ts = _dense_out("timestamps", ts, cache.k, (T,), torch.int64)
    _on_device(seq_offsets, starts, k, v, ts, cache.k)
    p = Problem(B, T, 1, H, dqk, dv, 1, _dtype_code(k))
    _check(lib.hstu_cache_read(ctypes.byref(p), ctypes.byref(cache._desc), offs, st, _ptr(k),
                               _ptr(v), _ptr(ts), _stream(stream)))
    return k, v, ts


def hstu_cache_validate(cache, stream=None):
    """Raises HstuError where lengths or the page table lead out of the pool."""
    B, H, dqk, dv = cache._shape
    _on_device(cache.k)
    p = Problem(B, 0, 1, H, dqk, dv, 1, HSTU_BF16)
    _check(lib.hstu_cache_validate(ctypes.byref(p), ctypes.byref(cache._desc), _stream(stream)))


# ------------------------------------------------ attention of drafted tokens

HSTU_MAX_DRAFT = 1024


def hstu_attn_fwd_tree_workspace_bytes(problem: Problem, cache: PagedCache, max_draft) -> int:
    return int(lib.hstu_attn_fwd_tree_workspace_bytes(ctypes.byref(problem),
                                                      ctypes.byref(cache._desc), int(max_draft)))


def hstu_attn_fwd_tree(q, k, v, seq_offsets, timestamps, cache, rab_pos, rab_time, max_seq_len,
                       max_draft, parents=None, out=None, ws=None, stream=None):
    """O [T, h, d_v] of drafted tokens q, k, v (at most max_draft for each user)
    over the cached tokens and the nodes on their way to the root (parents [T],
    None: all are roots); see include/hstu.h."""
    offs, B = _cache_batch(cache, seq_offsets)
    _, H, dqk, dv = cache._shape
    T, dtype = q.shape[0], q.dtype
    code = _dtype_code(q)
    qs = _rows("q", q, (T, H, dqk), dtype)
    ks = _rows("k", k, (T, H, dqk), dtype)
    vs = _rows("v", v, (T, H, dv), dtype)
    ts = _array("timestamps", timestamps, torch.int64, T)
    par = _array("parents", parents, torch.int64, T)
    rp = _array("rab_pos", rab_pos, torch.float32, 2 * max_seq_len - 1)
    rt = _array("rab_time", rab_time, torch.float32)
    out = _dense_out("out", out, q, (T, H, dv), dtype)
    p = Problem(B, T, max_seq_len, H, dqk, dv, rab_time.numel(), code)
    if ws is None:
        n = hstu_attn_fwd_tree_workspace_bytes(p, cache, max_draft)
        ws = q.new_empty(max(n, 256), dtype=torch.uint8)
    _on_device(q, k, v, seq_offsets, timestamps, parents, rab_pos, rab_time, out, ws, cache.k)
    j = Jagged(offs, ts, None, rp, rt)
    _check(lib.hstu_attn_fwd_tree(ctypes.byref(p), ctypes.byref(j), ctypes.byref(cache._desc), par,
                                  int(max_draft), _ptr(q), qs, _ptr(k), ks, _ptr(v), vs, _ptr(out),
                                  _ptr(ws), ws.numel(), _stream(stream)))
    return out


def hstu_tree_positions(parents, seq_offsets, base, total_tokens, max_draft, out=None,
                        stream=None):
    """int64 [T]: base[b] + depth of each drafted token (parents None: depth 0;
    base None: 0), for hstu_rotary_fwd."""
    offs, B = _offsets(seq_offsets)
    T = int(total_tokens)
    par = _array("parents", parents, torch.int64, T)
    bs = _array("base", base, torch.int64, B)
    out = _dense_out("positions", out, seq_offsets, (T,), torch.int64)
    _on_device(parents, seq_offsets, base, out)
    _check(lib.hstu_tree_positions(B, T, int(max_draft), offs, par, bs, _ptr(out),
                                   _stream(stream)))
    return out


def hstu_probe_mfma_bf16(iters: int, waves_per_simd: int, sink: torch.Tensor, stream=None):
    """Launches the matrix-core rate probe; returns its flop count."""
    flop = ctypes.c_double(0.0)
    _check(lib.hstu_probe_mfma_bf16(int(iters), int(waves_per_simd), _ptr(sink),
                                    ctypes.byref(flop), _stream(stream)))
    return flop.value


def hstu_timing_read(name: str):
    ms = ctypes.c_double(0.0)
    n = ctypes.c_int64(0)
    _check(lib.hstu_timing_read(name.encode(), ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value
