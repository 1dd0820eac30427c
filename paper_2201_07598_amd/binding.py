"""ctypes binding of the C ABI declared in include/okt.h.

Argument marshalling only: every function takes torch CUDA tensors (device
memory) and plain Python scalars, checks dtype / device / contiguity, passes raw
pointers and the current HIP stream, and raises OktError on a non-zero status.
No arithmetic of the method happens here.
"""
from __future__ import annotations

import ctypes
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

c_u32, c_u64, c_sz, c_vp, c_f32, c_f64, c_int = (ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t,
                                                 ctypes.c_void_p, ctypes.c_float, ctypes.c_double,
                                                 ctypes.c_int)

# name -> (restype, argtypes); mirrors include/okt.h
SIGNATURES = {
    "okt_status_string": (ctypes.c_char_p, [c_int]),
    "okt_last_hip_error": (ctypes.c_char_p, []),
    "okt_time_next_kernel": (None, [c_vp, c_vp]),
    "okt_debug_spin_limit": (None, [c_u32]),
    "okt_debug_digit_spin_limit": (None, [c_u32]),
    "okt_debug_slot_min_n": (None, [c_u64]),
    "okt_debug_slot_two_launches": (None, [c_int]),
    "okt_slot_min_n": (c_u64, [c_int]),
    "okt_version": (c_int, []),
    "okt_stream_copy": (c_int, [c_vp, c_vp, c_u64, c_vp]),
    "okt_stream_sum": (c_int, [c_vp, c_u64, c_vp, c_vp]),
    "okt_stream_gather": (c_int, [c_vp, c_vp, c_vp, c_vp, c_u32, c_u32, c_u32, c_vp, c_vp, c_u64, c_vp,
                                  c_sz, c_vp]),
    "okt_workspace_bytes": (c_sz, [c_u64, c_u32]),
    "okt_sparse_reduce_batch_workspace_bytes": (c_sz, [c_u32, c_u32, c_u32]),
    "okt_residual_accumulate": (c_int, [c_vp, c_vp, c_f32, c_u64, c_vp]),
    "okt_topk_threshold_exact": (c_int, [c_vp, c_u64, c_u64, c_vp, c_vp, c_vp, c_sz, c_vp]),
    "okt_threshold_select": (c_int, [c_vp, c_u64, c_vp, c_vp, c_vp, c_u64, c_vp, c_vp, c_sz, c_vp]),
    "okt_threshold_select_noalloc": (c_int, [c_vp, c_u64, c_vp, c_vp, c_vp, c_u64, c_vp, c_vp]),
    "okt_threshold_select_copy": (c_int, [c_vp, c_u64, c_vp, c_vp, c_vp, c_u64, c_vp, c_vp, c_sz, c_vp]),
    "okt_index_intersect_zero": (c_int, [c_vp, c_u64, c_vp, c_vp, c_u64, c_vp, c_vp, c_u64, c_vp, c_vp,
                                         c_vp, c_sz, c_vp]),
    "okt_accumulate_select": (c_int, [c_vp, c_vp, c_f32, c_u64, c_vp, c_vp, c_vp, c_u64, c_vp, c_vp,
                                      c_sz, c_vp]),
    "okt_accumulate_topk_select": (c_int, [c_vp, c_vp, c_f32, c_u64, c_u64, c_vp, c_vp, c_vp, c_vp,
                                           c_u64, c_vp, c_vp, c_sz, c_vp]),
    "okt_coo_threshold_select": (c_int, [c_vp, c_vp, c_vp, c_u64, c_vp, c_vp, c_vp, c_u64, c_vp, c_vp,
                                         c_sz, c_vp]),
    "okt_index_intersect_restore": (c_int, [c_vp, c_u64, c_vp, c_vp, c_vp, c_u64, c_vp, c_vp, c_u64,
                                            c_vp, c_vp, c_vp, c_sz, c_vp]),
    "okt_region_partition": (c_int, [c_vp, c_vp, c_u64, c_u32, c_vp, c_vp, c_vp]),
    "okt_sparse_reduce": (c_int, [c_vp, c_vp, c_vp, c_u32, c_u32, c_u32, c_vp, c_vp, c_u64, c_vp,
                                  c_vp, c_vp, c_sz, c_vp]),
    "okt_sparse_reduce_segments": (c_int, [c_vp, c_vp, c_vp, c_vp, c_u32, c_u32, c_u32, c_vp, c_vp, c_u64,
                                           c_vp, c_vp, c_vp, c_sz, c_vp]),
    "okt_balance_plan": (c_int, [c_vp, c_u32, c_vp, c_u32, c_vp, c_vp]),
    "okt_sparse_reduce_batch": (c_int, [c_vp, c_vp, c_vp, c_vp, c_u32, c_u32, c_u32, c_vp, c_vp,
                                        c_u64, c_vp, c_vp, c_vp, c_sz, c_vp]),
    "okt_dropout": (c_int, [c_vp, c_vp, c_u64, c_int, c_f64, c_vp, c_u32, c_vp]),
    "okt_residual_norm_workspace_bytes": (c_sz, [c_u64, c_u32, c_u64]),
    "okt_residual_norm_forward": (c_int, [c_vp, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp]),
    "okt_residual_norm_backward": (c_int, [c_vp] * 14 + [c_sz, c_vp]),
    "okt_attention_workspace_bytes": (c_sz, [c_u32] * 6),
    "okt_attention_forward": (c_int, [c_vp] * 7 + [c_sz, c_vp]),
    "okt_attention_backward": (c_int, [c_vp] * 11 + [c_sz, c_vp]),
    "okt_norm_rotary_workspace_bytes": (c_sz, [c_u32] * 5),
    "okt_norm_rotary_forward": (c_int, [c_vp] * 6),
    "okt_norm_rotary_backward": (c_int, [c_vp] * 10 + [c_sz, c_vp]),
    "okt_cross_entropy_workspace_bytes": (c_sz, [c_u64, c_u32, c_u32]),
    "okt_cross_entropy_forward": (c_int, [c_vp] * 7 + [c_sz, c_vp]),
    "okt_cross_entropy_backward": (c_int, [c_vp] * 10 + [c_sz, c_vp]),
    "okt_adamw_plan_bytes": (c_sz, [c_vp, c_u32]),
    "okt_adamw_plan": (c_int, [c_vp, c_u32, c_int, c_vp, c_sz, c_vp]),
    "okt_adamw_step": (c_int, [c_vp, c_vp, c_vp]),
}


class OktChunk(ctypes.Structure):
    _fields_ = [("src", c_u32), ("dst", c_u32), ("src_offset", c_u64), ("dst_offset", c_u64),
                ("count", c_u64)]


class OktError(RuntimeError):
    def __init__(self, call: str, status: int, text: str):
        super().__init__(f"{call} failed: {text} (status {status})")
        self.status = status


def library_path() -> str:
    return os.path.join(_HERE, "libokt.so")


def load_library() -> ctypes.CDLL:
    """Load libokt.so (built in-tree by paper_2201_07598_amd.build)."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise OktError("load_library", -100,
                           f"{path} is missing: run `python -m paper_2201_07598_amd.build`")
        # torch first: the library must bind to the HIP runtime torch brings along,
        # the one that owns the streams and the device memory it is handed
        _torch()
        lib = ctypes.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _LIB = lib
    return _LIB


def okt_status_string(status: int) -> str:
    return load_library().okt_status_string(int(status)).decode()


def okt_last_hip_error() -> str:
    return load_library().okt_last_hip_error().decode()


def okt_time_next_kernel(start_event, stop_event) -> None:
    """torch.cuda.Event objects (already recorded once, so that they exist) or None."""
    load_library().okt_time_next_kernel(
        ctypes.c_void_p(start_event.cuda_event if start_event is not None else None),
        ctypes.c_void_p(stop_event.cuda_event if stop_event is not None else None))


def okt_debug_spin_limit(polls: int) -> None:
    """Test hook: polls a wait between workgroups may take (0 = built-in limit)."""
    load_library().okt_debug_spin_limit(int(polls))


def okt_debug_digit_spin_limit(polls: int) -> None:
    """Test hook: the same for the digits of the exact threshold (0 = built-in limit)."""
    load_library().okt_debug_digit_spin_limit(int(polls))


def okt_debug_slot_min_n(n: int) -> None:
    """Test hook: shortest vector that takes the three-pass select (0 = built-in length)."""
    load_library().okt_debug_slot_min_n(int(n))


def okt_debug_slot_two_launches(on: bool) -> None:
    """Test hook: the accumulating calls empty the slots with two launches at any length."""
    load_library().okt_debug_slot_two_launches(1 if on else 0)


def okt_slot_min_n(accumulating: bool = False) -> int:
    """Vectors at least this long take the three-pass form (plain selects, or the
    calls that form the accumulator on the way)."""
    return load_library().okt_slot_min_n(1 if accumulating else 0)


def okt_version() -> int:
    return load_library().okt_version()


def okt_workspace_bytes(n_max: int, P_max: int = 0) -> int:
    return load_library().okt_workspace_bytes(int(n_max), int(P_max))


def okt_sparse_reduce_batch_workspace_bytes(B: int, P: int, max_width: int) -> int:
    return load_library().okt_sparse_reduce_batch_workspace_bytes(int(B), int(P), int(max_width))


# --------------------------------------------------------------------------
_TORCH = None


def _torch():
    """torch, imported with the first call and kept at hand: an import statement costs a
    third of a microsecond each time."""
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


# What a call costs the host beside its launches (2.6 us each) is what short vectors wait
# for: accumulate and select of 1 M elements, two launches and 8.2 us of GPU, took 11.2 us a call with
# 5.7 us of it spent here.  2.6 us were torch.cuda.current_stream(), which builds an
# object from the handle that is wanted; the rest the checks, whose usual outcome is
# decided first.
def _ptr(t, dtype, name, allow_none=False):
    if type(t) is _TORCH.Tensor and t.is_cuda and t.dtype is dtype and t.is_contiguous():
        return t.data_ptr()
    if t is None:
        if allow_none:
            return None
        raise TypeError(f"{name} is required")
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor (device memory)")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream(stream):
    """The handle of `stream`, or of the current stream of the current device."""
    if stream is None:
        return _TORCH._C._cuda_getCurrentRawStream(_TORCH._C._cuda_getDevice())
    return stream.cuda_stream


def _check(call, status):
    if status != 0:
        text = okt_status_string(status)
        if status == -3:
            text += ": " + okt_last_hip_error()
        raise OktError(call, status, text)


# uint64 scalars and uint32 indices on the device are carried in int64 and int32 tensors (same bytes)


def okt_residual_accumulate(grad, residual_inout, lr: float, stream=None) -> None:
    torch = _torch()
    _ptr(residual_inout, torch.float32, "residual_inout")
    _ptr(grad, torch.float32, "grad")
    n = residual_inout.numel()
    if grad.numel() != n:
        raise ValueError("grad and residual must have the same length")
    _check("okt_residual_accumulate", load_library().okt_residual_accumulate(
        _ptr(grad, torch.float32, "grad"), _ptr(residual_inout, torch.float32, "residual_inout"),
        float(lr), n, _stream(stream)))


STREAM_SUM_PARTIALS = 2048     # OKT_STREAM_SUM_PARTIALS


def okt_stream_copy(src, dst, stream=None) -> None:
    """Measurement only: dst[:] = src with the library's plain copy kernel."""
    torch = _torch()
    if src.numel() != dst.numel():
        raise ValueError("src and dst must have the same length")
    _check("okt_stream_copy", load_library().okt_stream_copy(
        _ptr(src, torch.float32, "src"), _ptr(dst, torch.float32, "dst"), src.numel(),
        _stream(stream)))


def okt_stream_sum(src, partials_out, stream=None) -> None:
    """Measurement only: one read of src; STREAM_SUM_PARTIALS fp32 partial sums out."""
    torch = _torch()
    if partials_out.numel() < STREAM_SUM_PARTIALS:
        raise ValueError(f"partials_out needs {STREAM_SUM_PARTIALS} elements")
    _check("okt_stream_sum", load_library().okt_stream_sum(
        _ptr(src, torch.float32, "src"), src.numel(),
        _ptr(partials_out, torch.float32, "partials_out"), _stream(stream)))


def okt_stream_gather(idx_cat, val_cat, chunk_off, lo_hi, B: int, P: int, max_width: int, idx_out,
                      val_out, capacity: int, ws, stream=None) -> None:
    """Measurement only: the batched reduce's reads and writes without its arithmetic."""
    torch = _torch()
    if chunk_off.numel() < B * (P + 1) or lo_hi.numel() < 2 * B:
        raise ValueError("chunk_off needs B*(P+1), lo_hi 2*B elements")
    if idx_out.numel() < B * capacity or val_out.numel() < B * capacity:
        raise ValueError("output buffers need B*capacity elements")
    _check("okt_stream_gather", load_library().okt_stream_gather(
        _ptr(idx_cat, torch.int32, "idx_cat"), _ptr(val_cat, torch.float32, "val_cat"),
        _ptr(chunk_off, torch.int64, "chunk_off"), _ptr(lo_hi, torch.int32, "lo_hi"),
        int(B), int(P), int(max_width),
        _ptr(idx_out, torch.int32, "idx_out"), _ptr(val_out, torch.float32, "val_out"),
        int(capacity), _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(stream)))


def okt_topk_threshold_exact(acc, k: int, threshold_out, count_ge_out, ws, stream=None) -> None:
    torch = _torch()
    if threshold_out.numel() < 1 or count_ge_out.numel() < 1:
        raise ValueError("threshold_out and count_ge_out need one element")
    _check("okt_topk_threshold_exact", load_library().okt_topk_threshold_exact(
        _ptr(acc, torch.float32, "acc"), acc.numel(), int(k),
        _ptr(threshold_out, torch.float32, "threshold_out"),
        _ptr(count_ge_out, torch.int64, "count_ge_out"),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(stream)))


def okt_threshold_select(acc_inout, threshold, idx_out, val_out, nnz_out, ws, capacity=None,
                         stream=None, _call="okt_threshold_select") -> None:
    torch = _torch()
    cap = min(idx_out.numel(), val_out.numel()) if capacity is None else int(capacity)
    if cap > idx_out.numel() or cap > val_out.numel():
        raise ValueError("capacity exceeds the output buffers")
    if nnz_out.numel() < 2 or threshold.numel() < 1:
        raise ValueError("nnz_out needs two elements, threshold one")
    _check(_call, getattr(load_library(), _call)(
        _ptr(acc_inout, torch.float32, "acc_inout"), acc_inout.numel(),
        _ptr(threshold, torch.float32, "threshold"),
        _ptr(idx_out, torch.int32, "idx_out"), _ptr(val_out, torch.float32, "val_out"), cap,
        _ptr(nnz_out, torch.int64, "nnz_out"), _ptr(ws, torch.uint8, "ws"), ws.numel(),
        _stream(stream)))


def okt_threshold_select_noalloc(acc_inout, threshold, idx_out, val_out, nnz_out, capacity=None,
                                 stream=None) -> None:
    """okt_threshold_select on the library's own scan state: no workspace argument."""
    torch = _torch()
    cap = min(idx_out.numel(), val_out.numel()) if capacity is None else int(capacity)
    if cap > idx_out.numel() or cap > val_out.numel():
        raise ValueError("capacity exceeds the output buffers")
    if nnz_out.numel() < 2 or threshold.numel() < 1:
        raise ValueError("nnz_out needs two elements, threshold one")
    _check("okt_threshold_select_noalloc", load_library().okt_threshold_select_noalloc(
        _ptr(acc_inout, torch.float32, "acc_inout"), acc_inout.numel(),
        _ptr(threshold, torch.float32, "threshold"),
        _ptr(idx_out, torch.int32, "idx_out"), _ptr(val_out, torch.float32, "val_out"), cap,
        _ptr(nnz_out, torch.int64, "nnz_out"), _stream(stream)))


def okt_threshold_select_copy(acc, threshold, idx_out, val_out, nnz_out, ws, capacity=None,
                              stream=None) -> None:
    okt_threshold_select(acc, threshold, idx_out, val_out, nnz_out, ws, capacity=capacity,
                         stream=stream, _call="okt_threshold_select_copy")


def okt_accumulate_select(grad, residual_inout, lr: float, threshold, idx_out, val_out, nnz_out, ws,
                          capacity=None, stream=None) -> None:
    torch = _torch()
    _ptr(residual_inout, torch.float32, "residual_inout")
    if grad.numel() != residual_inout.numel():
        raise ValueError("grad and residual must have the same length")
    cap = min(idx_out.numel(), val_out.numel()) if capacity is None else int(capacity)
    if cap > idx_out.numel() or cap > val_out.numel():
        raise ValueError("capacity exceeds the output buffers")
    if nnz_out.numel() < 2 or threshold.numel() < 1:
        raise ValueError("nnz_out needs two elements, threshold one")
    _check("okt_accumulate_select", load_library().okt_accumulate_select(
        _ptr(grad, torch.float32, "grad"), residual_inout.data_ptr(), float(lr),
        residual_inout.numel(), _ptr(threshold, torch.float32, "threshold"),
        _ptr(idx_out, torch.int32, "idx_out"), _ptr(val_out, torch.float32, "val_out"), cap,
        _ptr(nnz_out, torch.int64, "nnz_out"), _ptr(ws, torch.uint8, "ws"), ws.numel(),
        _stream(stream)))


def okt_accumulate_topk_select(grad, residual_inout, lr: float, k: int, threshold_out, count_ge_out,
                               idx_out, val_out, nnz_out, ws, capacity=None, stream=None) -> None:
    torch = _torch()
    _ptr(residual_inout, torch.float32, "residual_inout")
    if grad.numel() != residual_inout.numel():
        raise ValueError("grad and residual must have the same length")
    cap = min(idx_out.numel(), val_out.numel()) if capacity is None else int(capacity)
    if cap > idx_out.numel() or cap > val_out.numel():
        raise ValueError("capacity exceeds the output buffers")
    if nnz_out.numel() < 2 or threshold_out.numel() < 1 or count_ge_out.numel() < 1:
        raise ValueError("nnz_out needs two elements, threshold_out and count_ge_out one")
    _check("okt_accumulate_topk_select", load_library().okt_accumulate_topk_select(
        _ptr(grad, torch.float32, "grad"), residual_inout.data_ptr(), float(lr),
        residual_inout.numel(), int(k), _ptr(threshold_out, torch.float32, "threshold_out"),
        _ptr(count_ge_out, torch.int64, "count_ge_out"),
        _ptr(idx_out, torch.int32, "idx_out"), _ptr(val_out, torch.float32, "val_out"), cap,
        _ptr(nnz_out, torch.int64, "nnz_out"), _ptr(ws, torch.uint8, "ws"), ws.numel(),
        _stream(stream)))


def okt_region_partition(idx, nnz, n: int, R: int, bounds_out, offsets_out, stream=None) -> None:
    torch = _torch()
    if bounds_out.numel() < R + 1 or offsets_out.numel() < R + 1:
        raise ValueError("bounds_out and offsets_out need R+1 elements")
    _check("okt_region_partition", load_library().okt_region_partition(
        _ptr(idx, torch.int32, "idx"), _ptr(nnz, torch.int64, "nnz"), int(n), int(R),
        _ptr(bounds_out, torch.int32, "bounds_out"),
        _ptr(offsets_out, torch.int64, "offsets_out"), _stream(stream)))


def okt_sparse_reduce(idx_cat, val_cat, chunk_off, lo: int, hi: int, idx_out, val_out, nnz_out,
                      ws, dense_out=None, capacity=None, stream=None) -> None:
    torch = _torch()
    P = chunk_off.numel() - 1
    cap = min(idx_out.numel(), val_out.numel()) if capacity is None else int(capacity)
    if cap > idx_out.numel() or cap > val_out.numel():
        raise ValueError("capacity exceeds the output buffers")
    if dense_out is not None and dense_out.numel() < hi - lo:
        raise ValueError("dense_out needs hi-lo elements")
    if nnz_out.numel() < 2 or val_cat.numel() != idx_cat.numel():
        raise ValueError("nnz_out needs two elements; idx_cat and val_cat the same length")
    _check("okt_sparse_reduce", load_library().okt_sparse_reduce(
        _ptr(idx_cat, torch.int32, "idx_cat"), _ptr(val_cat, torch.float32, "val_cat"),
        _ptr(chunk_off, torch.int64, "chunk_off"), P, int(lo), int(hi),
        _ptr(idx_out, torch.int32, "idx_out"), _ptr(val_out, torch.float32, "val_out"), cap,
        _ptr(nnz_out, torch.int64, "nnz_out"),
        _ptr(dense_out, torch.float32, "dense_out", allow_none=True),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(stream)))


def okt_sparse_reduce_batch(idx_cat, val_cat, chunk_off, lo_hi, B: int, P: int, max_width: int,
                            idx_out, val_out, capacity: int, nnz_out, ws, dense_out=None,
                            stream=None) -> None:
    torch = _torch()
    if chunk_off.numel() < B * (P + 1) or lo_hi.numel() < 2 * B or nnz_out.numel() < 2 * B:
        raise ValueError("chunk_off needs B*(P+1), lo_hi and nnz_out 2*B elements")
    if idx_out.numel() < B * capacity or val_out.numel() < B * capacity:
        raise ValueError("output buffers need B*capacity elements")
    if dense_out is not None and dense_out.numel() < B * max_width:
        raise ValueError("dense_out needs B*max_width elements")
    _check("okt_sparse_reduce_batch", load_library().okt_sparse_reduce_batch(
        _ptr(idx_cat, torch.int32, "idx_cat"), _ptr(val_cat, torch.float32, "val_cat"),
        _ptr(chunk_off, torch.int64, "chunk_off"), _ptr(lo_hi, torch.int32, "lo_hi"),
        int(B), int(P), int(max_width),
        _ptr(idx_out, torch.int32, "idx_out"), _ptr(val_out, torch.float32, "val_out"),
        int(capacity), _ptr(nnz_out, torch.int64, "nnz_out"),
        _ptr(dense_out, torch.float32, "dense_out", allow_none=True),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(stream)))


def okt_coo_threshold_select(idx_in, val_in, nnz_in, threshold, idx_out, val_out, nnz_out, ws,
                             max_nnz=None, capacity=None, stream=None) -> None:
    torch = _torch()
    bound = min(idx_in.numel(), val_in.numel()) if max_nnz is None else int(max_nnz)
    if bound > idx_in.numel() or bound > val_in.numel():
        raise ValueError("max_nnz exceeds the input buffers")
    cap = min(idx_out.numel(), val_out.numel()) if capacity is None else int(capacity)
    if cap > idx_out.numel() or cap > val_out.numel():
        raise ValueError("capacity exceeds the output buffers")
    if nnz_out.numel() < 2 or threshold.numel() < 1 or nnz_in.numel() < 1:
        raise ValueError("nnz_out needs two elements, threshold and nnz_in one")
    _check("okt_coo_threshold_select", load_library().okt_coo_threshold_select(
        _ptr(idx_in, torch.int32, "idx_in"), _ptr(val_in, torch.float32, "val_in"),
        _ptr(nnz_in, torch.int64, "nnz_in"), bound, _ptr(threshold, torch.float32, "threshold"),
        _ptr(idx_out, torch.int32, "idx_out"), _ptr(val_out, torch.float32, "val_out"), cap,
        _ptr(nnz_out, torch.int64, "nnz_out"), _ptr(ws, torch.uint8, "ws"), ws.numel(),
        _stream(stream)))


def okt_index_intersect_restore(residual_inout, local_idx, local_val, local_nnz, global_idx,
                                global_nnz, count_out, ws, indexes_out=None, max_local=None,
                                max_global=None, stream=None) -> None:
    torch = _torch()
    bound_l = min(local_idx.numel(), local_val.numel()) if max_local is None else int(max_local)
    bound_g = global_idx.numel() if max_global is None else int(max_global)
    if bound_l > local_idx.numel() or bound_l > local_val.numel() or bound_g > global_idx.numel():
        raise ValueError("max_local / max_global exceed the input buffers")
    if indexes_out is not None and indexes_out.numel() < bound_l:
        raise ValueError("indexes_out needs max_local elements")
    if count_out.numel() < 1 or local_nnz.numel() < 1 or global_nnz.numel() < 1:
        raise ValueError("count_out, local_nnz and global_nnz need one element")
    _check("okt_index_intersect_restore", load_library().okt_index_intersect_restore(
        _ptr(residual_inout, torch.float32, "residual_inout"), residual_inout.numel(),
        _ptr(local_idx, torch.int32, "local_idx"), _ptr(local_val, torch.float32, "local_val"),
        _ptr(local_nnz, torch.int64, "local_nnz"), bound_l,
        _ptr(global_idx, torch.int32, "global_idx"), _ptr(global_nnz, torch.int64, "global_nnz"),
        bound_g, _ptr(indexes_out, torch.int32, "indexes_out", allow_none=True),
        _ptr(count_out, torch.int64, "count_out"), _ptr(ws, torch.uint8, "ws"), ws.numel(),
        _stream(stream)))


def okt_index_intersect_zero(acc_inout, local_idx, local_nnz, global_idx, global_nnz, count_out, ws,
                             indexes_out=None, max_local=None, max_global=None,
                             stream=None) -> None:
    torch = _torch()
    bound_l = local_idx.numel() if max_local is None else int(max_local)
    bound_g = global_idx.numel() if max_global is None else int(max_global)
    if bound_l > local_idx.numel() or bound_g > global_idx.numel():
        raise ValueError("max_local / max_global exceed the input buffers")
    if indexes_out is not None and indexes_out.numel() < bound_l:
        raise ValueError("indexes_out needs max_local elements")
    if count_out.numel() < 1 or local_nnz.numel() < 1 or global_nnz.numel() < 1:
        raise ValueError("count_out, local_nnz and global_nnz need one element")
    _check("okt_index_intersect_zero", load_library().okt_index_intersect_zero(
        _ptr(acc_inout, torch.float32, "acc_inout"), acc_inout.numel(),
        _ptr(local_idx, torch.int32, "local_idx"), _ptr(local_nnz, torch.int64, "local_nnz"),
        bound_l, _ptr(global_idx, torch.int32, "global_idx"),
        _ptr(global_nnz, torch.int64, "global_nnz"), bound_g,
        _ptr(indexes_out, torch.int32, "indexes_out", allow_none=True),
        _ptr(count_out, torch.int64, "count_out"), _ptr(ws, torch.uint8, "ws"), ws.numel(),
        _stream(stream)))


def okt_sparse_reduce_segments(idx_cat, val_cat, seg_begin, seg_end, P: int, lo: int, hi: int,
                               idx_out, val_out, nnz_out, ws, dense_out=None, capacity=None,
                               stream=None) -> None:
    torch = _torch()
    cap = min(idx_out.numel(), val_out.numel()) if capacity is None else int(capacity)
    if cap > idx_out.numel() or cap > val_out.numel():
        raise ValueError("capacity exceeds the output buffers")
    if seg_begin.numel() < P or seg_end.numel() < P:
        raise ValueError("seg_begin and seg_end need P elements")
    if dense_out is not None and dense_out.numel() < hi - lo:
        raise ValueError("dense_out needs hi-lo elements")
    if nnz_out.numel() < 2 or val_cat.numel() != idx_cat.numel():
        raise ValueError("nnz_out needs two elements; idx_cat and val_cat the same length")
    _check("okt_sparse_reduce_segments", load_library().okt_sparse_reduce_segments(
        _ptr(idx_cat, torch.int32, "idx_cat"), _ptr(val_cat, torch.float32, "val_cat"),
        _ptr(seg_begin, torch.int64, "seg_begin"), _ptr(seg_end, torch.int64, "seg_end"),
        int(P), int(lo), int(hi),
        _ptr(idx_out, torch.int32, "idx_out"), _ptr(val_out, torch.float32, "val_out"), cap,
        _ptr(nnz_out, torch.int64, "nnz_out"),
        _ptr(dense_out, torch.float32, "dense_out", allow_none=True),
        _ptr(ws, torch.uint8, "ws"), ws.numel(), _stream(stream)))


def okt_balance_plan(sizes):
    """Host-side: returns (triggered, [(src, dst, src_offset, dst_offset, count), ...])."""
    P = len(sizes)
    h_sizes = (c_u64 * max(P, 1))(*[int(x) for x in sizes])
    plan = (OktChunk * max(2 * P, 1))()
    n = c_u32(0)
    triggered = c_int(0)
    _check("okt_balance_plan", load_library().okt_balance_plan(
        ctypes.cast(h_sizes, c_vp), P, ctypes.cast(plan, c_vp), 2 * P, ctypes.cast(ctypes.pointer(n), c_vp),
        ctypes.cast(ctypes.pointer(triggered), c_vp)))
    return bool(triggered.value), [(c.src, c.dst, c.src_offset, c.dst_offset, c.count)
                                   for c in plan[:n.value]]


# --------------------------------------------------------------------------
# Operators of a layer's training step.  Their arguments travel in structs of the header,
# which are packed here as bytes: members lie in the order of the declaration and every one is
# aligned by what stands before it.
_NORM = struct.Struct("=QIiiffId7Q8Q")          # okt_residual_norm
_ATTENTION = struct.Struct("=6I2ifId3Q24Q")     # okt_attention
_NORM_KINDS = {"layer": 0, "rms": 1}
_DTYPES = {}


def _dtype_code(t, name):
    if not _DTYPES:
        torch = _torch()
        _DTYPES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


def _seed(seed, p):
    if p == 0.0 and seed is None:
        return 0
    if seed is None:
        raise TypeError("seed is required where something is dropped")
    if seed.numel() < 1:
        raise ValueError("seed needs one element")
    return _ptr(seed, _torch().int64, "seed")


def okt_dropout(x, y, p: float, seed, site: int = 0, stream=None) -> None:
    """y = dropout(x); with the gradient of y in place of x, that of x.  seed: int64[1] on
    the device (the bytes of the uint64); y may be x."""
    _torch()
    code = _dtype_code(x, "x")
    if x.numel() != y.numel():
        raise ValueError("x and y must have the same length")
    if seed is None:
        raise TypeError("seed is required")
    _check("okt_dropout", load_library().okt_dropout(
        _ptr(x, x.dtype, "x"), _ptr(y, x.dtype, "y"), x.numel(), code, float(p), _seed(seed, p), int(site),
        _stream(stream)))


# What such a call costs the host is what short sequences wait for, as above: the usual outcome
# of a tensor's checks is decided first, by comparisons alone.
def _rows(t, dtype, shape, name, allow_none=False):
    """(pointer, row stride) of a [rows, width] tensor, rows any distance apart."""
    if t is not None and t.dtype is dtype and t.is_cuda and t.shape == shape:
        step, unit = t.stride()
        if unit == 1 and step >= shape[1]:
            return t.data_ptr(), step if shape[0] > 1 else 0
    if t is None:
        if allow_none:
            return None, 0
        raise TypeError(f"{name} is required")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor (device memory)")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")
    step, unit = t.stride()
    if unit != 1 and shape[1] > 1:
        raise ValueError(f"{name} must have contiguous rows")
    if shape[0] > 1 and step < shape[1]:
        raise ValueError(f"rows of {name} must not overlap")
    return t.data_ptr(), step if shape[0] > 1 else 0


def _parameter(t, numel, name):
    """The address of a float32 parameter on the device, 0 for none."""
    if t is None:
        return 0
    if t.dtype is _TORCH.float32 and t.is_cuda and t.numel() == numel and t.is_contiguous():
        return t.data_ptr()
    if t.numel() != numel:
        raise ValueError(f"{name} needs {numel} elements, got {t.numel()}")
    return _ptr(t, _TORCH.float32, name)


def _norm_struct(dtype, shape, kind, eps, residual_scale, post_weight, post_bias, gate, rows_per_gate,
                 pre_weight, pre_bias, dropout_p, seed, site, strides):
    rows, width = shape
    return _NORM.pack(
        rows, width, _DTYPES[dtype], _NORM_KINDS[kind], eps, residual_scale, site, dropout_p,
        0 if seed is None and dropout_p == 0.0 else _seed(seed, dropout_p),
        0 if post_weight is None else _parameter(post_weight, width, "post_weight"),
        0 if post_bias is None else _parameter(post_bias, width, "post_bias"),
        0 if gate is None else _parameter(gate, _gates(rows, rows_per_gate) * width, "gate"), rows_per_gate,
        0 if pre_weight is None else _parameter(pre_weight, width, "pre_weight"),
        0 if pre_bias is None else _parameter(pre_bias, width, "pre_bias"), *strides)


def _gates(rows, rows_per_gate):
    return max(1, -(-rows // rows_per_gate)) if rows_per_gate else 1


def okt_residual_norm_workspace_bytes(rows: int, width: int, rows_per_gate: int = 0) -> int:
    return load_library().okt_residual_norm_workspace_bytes(int(rows), int(width), int(rows_per_gate))


def okt_residual_norm_forward(u, x, h_out, y_out, stats_out, *, kind: str = "layer", eps: float = 1e-5,
                              residual_scale: float = 1.0, post_weight=None, post_bias=None, gate=None,
                              rows_per_gate: int = 0, pre_weight=None, pre_bias=None,
                              dropout_p: float = 0.0, seed=None, site: int = 0, stream=None) -> None:
    """h = residual_scale x + gate * dropout(norm(u)), y = norm(h) on [rows, width] tensors;
    a norm is there where its weight is.  kind: "layer" or "rms".  h_out may be None, stats_out
    (float32 [rows, 4]) too where no backward pass follows."""
    _dtype_code(u, "u")
    dtype, shape = u.dtype, u.shape
    if len(shape) != 2:
        raise ValueError("u must be [rows, width]")
    pu, su = _rows(u, dtype, shape, "u")
    px, sx = _rows(x, dtype, shape, "x")
    ph, sh = _rows(h_out, dtype, shape, "h_out", True)
    py, sy = _rows(y_out, dtype, shape, "y_out", True)
    if stats_out is not None and stats_out.numel() < 4 * shape[0]:
        raise ValueError("stats_out needs four elements a row")
    op = _norm_struct(dtype, shape, kind, eps, residual_scale, post_weight, post_bias, gate, rows_per_gate,
                         pre_weight, pre_bias, dropout_p, seed, site, (su, sx, sh, sy, 0, 0, 0, 0))
    _check("okt_residual_norm_forward", load_library().okt_residual_norm_forward(
        op, pu, px, ph, py, _ptr(stats_out, _TORCH.float32, "stats_out", True), _stream(stream)))


def okt_residual_norm_backward(u, h, stats, dh, dy, dx_out, du_out, ws, *, dpost_weight=None,
                               dpost_bias=None, dgate=None, dpre_weight=None, dpre_bias=None,
                               kind: str = "layer", eps: float = 1e-5, residual_scale: float = 1.0,
                               post_weight=None, post_bias=None, gate=None, rows_per_gate: int = 0,
                               pre_weight=None, pre_bias=None, dropout_p: float = 0.0, seed=None,
                               site: int = 0, stream=None) -> None:
    """Gradients of x, u and the parameters from those of h (dh, None for zero) and y (dy, None
    without a pre norm).  The parameters' gradients are float32 and are overwritten; None
    leaves one out."""
    if du_out is None or du_out.dim() != 2:
        raise ValueError("du_out must be [rows, width]")
    _dtype_code(du_out, "du_out")
    dtype, shape = du_out.dtype, du_out.shape
    pu, su = _rows(u, dtype, shape, "u", True)
    ph, sh = _rows(h, dtype, shape, "h", True)
    pdh, sdh = _rows(dh, dtype, shape, "dh", True)
    pdy, sdy = _rows(dy, dtype, shape, "dy", True)
    pdx, sdx = _rows(dx_out, dtype, shape, "dx_out")
    pdu, sdu = _rows(du_out, dtype, shape, "du_out")
    rows, width = shape
    if stats.numel() < 4 * rows:
        raise ValueError("stats needs four elements a row")
    op = _norm_struct(dtype, shape, kind, eps, residual_scale, post_weight, post_bias, gate, rows_per_gate,
                      pre_weight, pre_bias, dropout_p, seed, site, (su, 0, sh, 0, sdh, sdy, sdx, sdu))
    _check("okt_residual_norm_backward", load_library().okt_residual_norm_backward(
        op, pu, ph, _ptr(stats, _TORCH.float32, "stats"), pdh, pdy, pdx, pdu,
        _parameter(dpost_weight, width, "dpost_weight"), _parameter(dpost_bias, width, "dpost_bias"),
        0 if dgate is None else _parameter(dgate, _gates(rows, rows_per_gate) * width, "dgate"),
        _parameter(dpre_weight, width, "dpre_weight"), _parameter(dpre_bias, width, "dpre_bias"),
        _ptr(ws, _TORCH.uint8, "ws"), ws.numel(), _stream(stream)))


def okt_attention_workspace_bytes(batch: int, heads: int, kv_heads: int, q_len: int, k_len: int,
                                  head_dim: int) -> int:
    return load_library().okt_attention_workspace_bytes(int(batch), int(heads), int(kv_heads), int(q_len),
                                                        int(k_len), int(head_dim))


def _heads(t, dtype, shape, name):
    """(pointer, (batch stride, length stride, head stride)) of a [batch, length, heads, dim]
    tensor."""
    if t.dtype is dtype and t.is_cuda and t.shape == shape:
        strides = t.stride()
        if strides[3] == 1:
            return t.data_ptr(), strides[:3]
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor (device memory)")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must have contiguous head vectors")


def _lengths(t, batch, name):
    if t is None:
        return 0
    if t.numel() != batch:
        raise ValueError(f"{name} needs one element a sequence")
    return _ptr(t, _TORCH.int32, name)


_NO_STRIDES = (0,) * 12


def _attention_struct(dtype, shape, keys, causal, scale, dropout_p, seed, site, q_lens, k_lens, strides):
    batch, q_len, heads, dim = shape
    return _ATTENTION.pack(
        batch, heads, keys[2], q_len, keys[1], dim, _DTYPES[dtype], 1 if causal else 0,
        dim ** -0.5 if scale is None else scale, site, dropout_p,
        0 if seed is None and dropout_p == 0.0 else _seed(seed, dropout_p),
        0 if q_lens is None else _lengths(q_lens, batch, "q_lens"),
        0 if k_lens is None else _lengths(k_lens, batch, "k_lens"), *strides)


def _attention_inputs(q, k, v):
    _dtype_code(q, "q")
    dtype, shape, keys = q.dtype, q.shape, k.shape
    if len(shape) != 4 or len(keys) != 4:
        raise ValueError("q, k and v must be [batch, length, heads, head_dim]")
    if keys[0] != shape[0] or keys[3] != shape[3]:
        raise ValueError("q and k must agree in batch and head_dim")
    pq, sq = _heads(q, dtype, shape, "q")
    pk, sk = _heads(k, dtype, keys, "k")
    pv, sv = _heads(v, dtype, keys, "v")
    return dtype, shape, keys, pq, pk, pv, sq + sk + sv


def okt_attention_forward(q, k, v, o_out, lse_out, ws=None, *, causal: bool = False, scale=None,
                          q_lens=None, k_lens=None, dropout_p: float = 0.0, seed=None, site: int = 0,
                          stream=None) -> None:
    """o = dropout(softmax(scale q k' over the visible keys)) v on [batch, length, heads, head_dim]
    tensors, the last axis contiguous, other strides multiples of 8; scale defaults to head_dim ** -0.5.  q_lens, k_lens: int32 [batch] on the
    device, the sequences' own lengths.  lse_out (float32 [batch, heads, q_len]) may be None where
    no backward pass follows."""
    dtype, shape, keys, pq, pk, pv, strides = _attention_inputs(q, k, v)
    po, so = _heads(o_out, dtype, shape, "o_out")
    if lse_out is not None and lse_out.numel() != shape[0] * shape[1] * shape[2]:
        raise ValueError("lse_out must be [batch, heads, q_len]")
    op = _attention_struct(dtype, shape, keys, causal, scale, dropout_p, seed, site, q_lens, k_lens,
                           strides + so + _NO_STRIDES)
    _check("okt_attention_forward", load_library().okt_attention_forward(
        op, pq, pk, pv, po, _ptr(lse_out, _TORCH.float32, "lse_out", True),
        _ptr(ws, _TORCH.uint8, "ws", True), 0 if ws is None else ws.numel(), _stream(stream)))


def okt_attention_backward(q, k, v, o, lse, do, dq_out, dk_out, dv_out, ws, *, causal: bool = False,
                           scale=None, q_lens=None, k_lens=None, dropout_p: float = 0.0, seed=None,
                           site: int = 0, stream=None) -> None:
    """Gradients of q, k and v from that of o, with o and lse of the forward pass and the same
    options (seed and site above all)."""
    dtype, shape, keys, pq, pk, pv, strides = _attention_inputs(q, k, v)
    po, so = _heads(o, dtype, shape, "o")
    pdo, sdo = _heads(do, dtype, shape, "do")
    pdq, sdq = _heads(dq_out, dtype, shape, "dq_out")
    pdk, sdk = _heads(dk_out, dtype, keys, "dk_out")
    pdv, sdv = _heads(dv_out, dtype, keys, "dv_out")
    if lse.numel() != shape[0] * shape[1] * shape[2]:
        raise ValueError("lse must be [batch, heads, q_len]")
    op = _attention_struct(dtype, shape, keys, causal, scale, dropout_p, seed, site, q_lens, k_lens,
                           strides + so + sdo + sdq + sdk + sdv)
    _check("okt_attention_backward", load_library().okt_attention_backward(
        op, pq, pk, pv, po, _ptr(lse, _TORCH.float32, "lse"), pdo, pdq, pdk, pdv,
        _ptr(ws, _TORCH.uint8, "ws"), ws.numel(), _stream(stream)))


# --------------------------------------------------------------------------
# Where a call's tensors lie: all on the current device, whose stream it is enqueued on.
def _stream_for(stream, *tensors):
    device = _TORCH._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError(f"tensors must be on the current device ({device}), got one on {t.device}")
    if stream is None:
        return _TORCH._C._cuda_getCurrentRawStream(device)
    if stream.device_index != device:
        raise ValueError(f"stream must be of the current device ({device}), got {stream.device}")
    return stream.cuda_stream


# --------------------------------------------------------------------------
# Norms and rotation of heads
_ROTARY = struct.Struct("=6I2ifi2I128sQQ2Q2Q18Q")    # okt_norm_rotary


def okt_norm_rotary_workspace_bytes(batch: int, length: int, heads: int, kv_heads: int, head_dim: int) -> int:
    return load_library().okt_norm_rotary_workspace_bytes(int(batch), int(length), int(heads), int(kv_heads), int(head_dim))


def _positions(t, batch, length, axes):
    """(pointer, batch stride, token stride) of int32 [batch, length, axes] or [length, axes]; one axis may be left out."""
    if t is None:
        return 0, 0, 0
    if t.dtype is _TORCH.int32 and t.is_cuda and t.shape == (batch, length, axes):
        strides = t.stride()
        if axes == 1 or strides[2] == 1:
            return t.data_ptr(), strides[0], strides[1]
    if not t.is_cuda:
        raise TypeError("positions must be a CUDA tensor (device memory)")
    if t.dtype is not _TORCH.int32:
        raise TypeError(f"positions must have dtype {_TORCH.int32}, got {t.dtype}")
    if axes == 1 and (t.dim() == 1 or (t.dim() == 2 and t.shape == (batch, length) and t.shape != (length, 1))):
        t = t.unsqueeze(-1)
    if t.shape != (batch, length, axes) and t.shape != (length, axes):
        raise ValueError(f"positions must have the shape {(batch, length, axes)} or {(length, axes)}, got {tuple(t.shape)}")
    if axes > 1 and t.stride(-1) != 1:
        raise ValueError("positions must have contiguous axes")
    strides = t.stride()
    return t.data_ptr(), strides[0] if t.dim() == 3 else 0, strides[-2]


_NO_HEADS = (0, 0, 0)


def _rotary_struct(dtype, shape, kv_heads, inv_freq, positions, axis_of_pair, adjacent, kind, eps, q_weight, k_weight, strides):
    batch, length, heads, dim = shape
    pairs = 0 if inv_freq is None else inv_freq.numel()
    axes = 1
    table = b""
    if axis_of_pair is not None:
        if len(axis_of_pair) != pairs:
            raise ValueError(f"axis_of_pair needs one axis a pair ({pairs}), got {len(axis_of_pair)}")
        table = bytes(axis_of_pair)
        axes = 1 if table.count(0) == pairs else max(table) + 1
    if positions is not None:
        places = positions.shape
        # two sizes are [batch, length] where they can be and one axis turns all pairs, else [length, axes]
        if len(places) == 3 or (len(places) == 2 and (axes > 1 or (places[0] == length and places != (batch, length)))):
            axes = max(axes, places[-1])
    at, by_batch, by_token = _positions(positions, batch, length, axes)
    return _ROTARY.pack(
        batch, length, heads, kv_heads, dim, 2 * pairs, _DTYPES[dtype], _NORM_KINDS[kind], eps, 1 if adjacent else 0, axes, 0, table,
        0 if inv_freq is None else _parameter(inv_freq, pairs, "inv_freq"), at, by_batch, by_token,
        _parameter(q_weight, dim, "q_weight"), _parameter(k_weight, dim, "k_weight"), *strides)


def okt_norm_rotary_forward(q, k, q_out, k_out, inv_freq, *, positions=None, axis_of_pair=None, adjacent: bool = False,
                            kind: str = "rms", eps: float = 1e-6, q_weight=None, k_weight=None, stream=None) -> None:
    """Norm (where there is a weight) and rotation of every head of [batch, length, heads, head_dim] tensors, the last axis
    contiguous.  k and k_out may be None.  inv_freq: float32, one frequency a pair, so 2 * inv_freq.numel() leading elements of a head
    are rotated (None: none).  positions: int32 [batch, length, axes] or [length, axes] on the device (of one axis [batch, length] or
    [length], too), None for the place in the
    sequence; axis_of_pair: which axis turns each pair (a sequence of numbers; None: the first).  Outputs may be their inputs."""
    _dtype_code(q, "q")
    dtype, shape = q.dtype, q.shape
    if len(shape) != 4:
        raise ValueError("q and k must be [batch, length, heads, head_dim]")
    pq, sq = _heads(q, dtype, shape, "q")
    po, so = _heads(q_out, dtype, shape, "q_out")
    pk, sk, pko, sko, kv_heads = 0, _NO_HEADS, 0, _NO_HEADS, 0
    if k is not None:
        keys = k.shape
        if len(keys) != 4 or keys[0] != shape[0] or keys[1] != shape[1] or keys[3] != shape[3]:
            raise ValueError("q and k must agree in batch, length and head_dim")
        kv_heads = keys[2]
        pk, sk = _heads(k, dtype, keys, "k")
        pko, sko = _heads(k_out, dtype, keys, "k_out")
    op = _rotary_struct(dtype, shape, kv_heads, inv_freq, positions, axis_of_pair, adjacent, kind, eps, q_weight, k_weight,
                        (*sq, *sk, *so, *sko, *_NO_HEADS, *_NO_HEADS))
    handle = _stream_for(stream, q, k, q_out, k_out, inv_freq, positions, q_weight, k_weight)
    _check("okt_norm_rotary_forward", load_library().okt_norm_rotary_forward(op, pq, pk, po, pko, handle))


def okt_norm_rotary_backward(q, k, dq, dk, dq_out, dk_out, inv_freq, ws=None, *, dq_weight_out=None, dk_weight_out=None,
                             positions=None, axis_of_pair=None, adjacent: bool = False, kind: str = "rms", eps: float = 1e-6,
                             q_weight=None, k_weight=None, stream=None) -> None:
    """Gradients of q, k and the weights from those of the outputs, dq and dk, with the options of the forward pass.  q and k as
    the forward pass read them (None where there is no weight).  dq_out may be dq, dk_out dk."""
    _dtype_code(dq, "dq")
    dtype, shape = dq.dtype, dq.shape
    if len(shape) != 4:
        raise ValueError("dq and dk must be [batch, length, heads, head_dim]")
    pd, sd = _heads(dq, dtype, shape, "dq")
    po, so = _heads(dq_out, dtype, shape, "dq_out")
    if q is None and q_weight is not None:
        raise TypeError("q is required where it has a norm")
    pq, sq = (0, _NO_HEADS) if q is None else _heads(q, dtype, shape, "q")
    pk, sk, pdk, sdk, pko, sko, kv_heads = 0, _NO_HEADS, 0, _NO_HEADS, 0, _NO_HEADS, 0
    if dk is not None:
        keys = dk.shape
        if len(keys) != 4 or keys[0] != shape[0] or keys[1] != shape[1] or keys[3] != shape[3]:
            raise ValueError("dq and dk must agree in batch, length and head_dim")
        kv_heads = keys[2]
        if k is None and k_weight is not None:
            raise TypeError("k is required where it has a norm")
        pk, sk = (0, _NO_HEADS) if k is None else _heads(k, dtype, keys, "k")
        pdk, sdk = _heads(dk, dtype, keys, "dk")
        pko, sko = _heads(dk_out, dtype, keys, "dk_out")
    op = _rotary_struct(dtype, shape, kv_heads, inv_freq, positions, axis_of_pair, adjacent, kind, eps, q_weight, k_weight,
                        (*sq, *sk, *so, *sko, *sd, *sdk))
    dim = shape[3]
    handle = _stream_for(stream, q, k, dq, dk, dq_out, dk_out, inv_freq, positions, q_weight, k_weight, dq_weight_out, dk_weight_out, ws)
    _check("okt_norm_rotary_backward", load_library().okt_norm_rotary_backward(
        op, pq, pk, pd, pdk, po, pko, _parameter(dq_weight_out, dim, "dq_weight_out"), _parameter(dk_weight_out, dim, "dk_weight_out"),
        _ptr(ws, _TORCH.uint8, "ws", True), 0 if ws is None else ws.numel(), handle))


# --------------------------------------------------------------------------
# Cross entropy over a vocabulary
_CROSS_ENTROPY = struct.Struct("=Q2I2i2IQ4Q")        # okt_cross_entropy


def okt_cross_entropy_workspace_bytes(rows: int, width: int, vocab: int) -> int:
    return load_library().okt_cross_entropy_workspace_bytes(int(rows), int(width), int(vocab))


def _cross_entropy_inputs(h, weight, labels):
    if h.dtype not in (_torch().bfloat16, _TORCH.float16):
        raise TypeError(f"h must be bfloat16 or float16, got {h.dtype}")
    _dtype_code(h, "h")
    if h.dim() != 2 or weight.dim() != 2:
        raise ValueError("h must be [rows, width] and weight [vocab, width]")
    rows, width = h.shape
    if weight.shape[1] != width:
        raise ValueError("h and weight must agree in width")
    ph, sh = _rows(h, h.dtype, h.shape, "h")
    pw, sw = _rows(weight, h.dtype, weight.shape, "weight")
    if labels.numel() != rows:
        raise ValueError(f"labels needs one element a row ({rows}), got {labels.numel()}")
    return rows, width, weight.shape[0], ph, sh, pw, sw, _ptr(labels, _TORCH.int64, "labels")


def _per_row(t, rows, name, allow_none=False):
    if t is not None and t.numel() != rows:
        raise ValueError(f"{name} needs one element a row ({rows}), got {t.numel()}")
    return _ptr(t, _TORCH.float32, name, allow_none)


def okt_cross_entropy_forward(h, weight, labels, loss_out, lse_out, ws, *, bias=None, stream=None) -> None:
    """loss = logsumexp(h weight' + bias) - the label's logit for every row of h [rows, width] (bfloat16 or float16), weight
    [vocab, width]; labels int64 [rows]; 0 for a row whose label is not in the vocabulary.  loss_out and
    lse_out float32 [rows]; lse_out may be None where no backward pass follows; bias float32 [vocab]."""
    rows, width, vocab, ph, sh, pw, sw, py = _cross_entropy_inputs(h, weight, labels)
    op = _CROSS_ENTROPY.pack(rows, width, vocab, _DTYPES[h.dtype], _DTYPES[h.dtype], 1, 0, _parameter(bias, vocab, "bias"), sh, sw, 0, 0)
    ploss, plse = _per_row(loss_out, rows, "loss_out"), _per_row(lse_out, rows, "lse_out", True)
    pws = _ptr(ws, _TORCH.uint8, "ws")
    handle = _stream_for(stream, h, weight, labels, loss_out, lse_out, ws, bias)
    _check("okt_cross_entropy_forward", load_library().okt_cross_entropy_forward(op, ph, pw, py, ploss, plse, pws, ws.numel(), handle))


def okt_cross_entropy_backward(h, weight, labels, lse, dloss, dh_out, dweight_out, ws, *, bias=None, dbias_out=None,
                               stream=None) -> None:
    """Gradients of h, weight and bias from that of the loss: dloss float32 [rows], or one value for all rows (one element, or
    expanded from one).  dh_out is of h's type, dweight_out of that or float32; either may be None."""
    rows, width, vocab, ph, sh, pw, sw, py = _cross_entropy_inputs(h, weight, labels)
    f32 = _TORCH.float32
    if not dloss.is_cuda:
        raise TypeError("dloss must be a CUDA tensor (device memory)")
    if dloss.dtype is not f32:
        raise TypeError(f"dloss must have dtype {f32}, got {dloss.dtype}")
    if dloss.numel() != rows and dloss.numel() != 1:
        raise ValueError(f"dloss needs one element a row ({rows}) or one, got {dloss.numel()}")
    one = dloss.numel() == 1 or all(s == 0 for s in dloss.stride())
    if not one and not dloss.is_contiguous():
        raise TypeError("dloss must be contiguous, or one value for all rows")
    pdh, sdh = _rows(dh_out, h.dtype, h.shape, "dh_out", True)
    wide = dweight_out is not None and dweight_out.dtype is f32
    pdw, sdw = _rows(dweight_out, f32 if wide else h.dtype, weight.shape, "dweight_out", True)
    op = _CROSS_ENTROPY.pack(rows, width, vocab, _DTYPES[h.dtype], 0 if wide else _DTYPES[h.dtype], 0 if one else 1, 0,
                             _parameter(bias, vocab, "bias"), sh, sw, sdh, sdw)
    plse, pdb, pws = _per_row(lse, rows, "lse"), _parameter(dbias_out, vocab, "dbias_out"), _ptr(ws, _TORCH.uint8, "ws")
    handle = _stream_for(stream, h, weight, labels, lse, dloss, dh_out, dweight_out, dbias_out, bias, ws)
    _check("okt_cross_entropy_backward", load_library().okt_cross_entropy_backward(
        op, ph, pw, py, plse, dloss.data_ptr(), pdh, pdw, pdb, pws, ws.numel(), handle))


# --------------------------------------------------------------------------
# AdamW over many tensors
_ADAMW_TENSOR = struct.Struct("=7QQ2d4i")       # okt_adamw_tensor
_ADAMW = struct.Struct("=2IiI4d5Q")             # okt_adamw
ADAMW_BLOCK = 256                               # OKT_ADAMW_BLOCK


class AdamWPlan:
    """What okt_adamw_step needs of its tensors, on their device; keeps them alive.  To be made again when one of
    them moves (okt_adamw_plan), a gradient too, so gradients are to be written in place; their contents may change at will."""

    def __init__(self, device_bytes, tensors, chunks, state, held):
        self.device_bytes, self.tensors, self.chunks, self.state, self.held = device_bytes, tensors, chunks, state, held


def okt_adamw_plan_bytes(lengths) -> int:
    """Bytes of the plan of tensors of such lengths; 0 if they are out of range."""
    table = b"".join(_ADAMW_TENSOR.pack(*(0,) * 7, int(n), 0.0, 1.0, 0, 0, 1, 0) for n in lengths)
    return load_library().okt_adamw_plan_bytes(table, len(lengths))


def _each(value, count, name):
    """One number for all tensors, or one for each."""
    if isinstance(value, (int, float)):
        return [float(value)] * count
    value = [float(x) for x in value]
    if len(value) != count:
        raise ValueError(f"{name} needs one value a tensor ({count}), got {len(value)}")
    return value


def _adamw_refuse(params, grads, ms, vs, m_scales, v_scales, copies, lengths, blocks, state_type, device):
    """Says which tensor is not what a plan needs."""
    torch = _TORCH
    for i, (n, b) in enumerate(zip(lengths, blocks)):
        parts = [(params[i], None, "params", n), (grads[i], None, "grads", n), (ms[i], state_type, "ms", n), (vs[i], state_type, "vs", n)]
        if m_scales is not None:
            parts += [(m_scales[i], torch.float32, "m_scales", b), (v_scales[i], torch.float32, "v_scales", b)]
        if copies is not None and copies[i] is not None:
            parts.append((copies[i], None, "copies", n))
        for t, dtype, name, numel in parts:
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name}[{i}] is required")
            if dtype is None:
                _dtype_code(t, f"{name}[{i}]")
            _ptr(t, dtype or t.dtype, f"{name}[{i}]")
            if t.numel() != numel:
                raise ValueError(f"{name}[{i}] needs {numel} elements, got {t.numel()}")
            if t.device != device:
                raise ValueError(f"{name}[{i}] must be on {device}, got {t.device}")
            if name == "copies" and t.dtype is torch.float32:
                raise TypeError(f"copies[{i}] must be bfloat16 or float16")


def okt_adamw_plan(params, grads, ms, vs, *, m_scales=None, v_scales=None, copies=None, weight_decay=0.0,
                   rate_scale=1.0) -> AdamWPlan:
    """The plan of okt_adamw_step over lists of tensors, which are contiguous and on one device: params and grads float32,
    bfloat16 or float16; the averages ms and vs float32, or float8_e4m3fn with a float32 scale for every ADAMW_BLOCK
    elements in m_scales and v_scales (v is the square of what vs stands for); copies, if given, bfloat16
    or float16 (or None for a tensor without one).  weight_decay and rate_scale: one for all or one a tensor.  Copies the plan to the device,
    on the current stream."""
    torch = _torch()
    count = len(params)
    if count == 0:
        raise ValueError("params must not be empty")
    lists = {"grads": grads, "ms": ms, "vs": vs, "m_scales": m_scales, "v_scales": v_scales, "copies": copies}
    for name, tensors in lists.items():
        if tensors is not None and len(tensors) != count:
            raise ValueError(f"{name} needs one tensor a parameter ({count}), got {len(tensors)}")
    for name in ("grads", "ms", "vs"):
        if lists[name] is None:
            raise TypeError(f"{name} is required")
    state_type = ms[0].dtype
    if state_type not in (torch.float32, torch.float8_e4m3fn):
        raise TypeError(f"ms and vs must be float32 or float8_e4m3fn, got {state_type}")
    eight = state_type == torch.float8_e4m3fn
    if eight != (m_scales is not None) or eight != (v_scales is not None):
        raise TypeError("m_scales and v_scales belong to averages in float8_e4m3fn, both of them")
    decays, rates = _each(weight_decay, count, "weight_decay"), _each(rate_scale, count, "rate_scale")
    device, held = params[0].device, [*params, *grads, *ms, *vs]
    scales = [*m_scales, *v_scales] if eight else []
    held += scales
    held += [c for c in copies or () if c is not None]
    lengths = [p.numel() if isinstance(p, torch.Tensor) else 0 for p in params]
    blocks = [-(-n // ADAMW_BLOCK) for n in lengths]

    def fine(tensors, types, numels):
        """The usual outcome, decided by comparisons alone."""
        return all(type(t) is torch.Tensor and t.device == device and t.is_contiguous() for t in tensors) and device.type == "cuda" and (
            {t.dtype for t in tensors} <= types and [t.numel() for t in tensors] == numels)

    floats, one = {torch.float32, torch.bfloat16, torch.float16}, {state_type}
    whole = all(fine(x, t, n) for x, t, n in ((params, floats, lengths), (grads, floats, lengths), (ms, one, lengths), (vs, one, lengths)))
    whole = whole and (not eight or all(fine(x, {torch.float32}, blocks) for x in (m_scales, v_scales)))
    there = [] if copies is None else [(c, n) for c, n in zip(copies, lengths) if c is not None]
    whole = whole and fine([c for c, _ in there], floats - {torch.float32}, [n for _, n in there])
    if not whole:
        _adamw_refuse(params, grads, ms, vs, m_scales, v_scales, copies, lengths, blocks, state_type, device)
    _dtype_code(params[0], "params[0]")

    def places(tensors):
        return [0] * count if tensors is None else [0 if t is None else t.data_ptr() for t in tensors]

    codes = lambda tensors: [_DTYPES[t.dtype] for t in tensors]  # noqa: E731
    copy_codes = [1] * count if copies is None else [1 if c is None else _DTYPES[c.dtype] for c in copies]
    packed = [_ADAMW_TENSOR.pack(*row, 0) for row in zip(
        places(params), places(grads), places(ms), places(vs), places(copies), places(m_scales), places(v_scales), lengths, decays, rates,
        codes(params), codes(grads), copy_codes)]
    table, lib = b"".join(packed), load_library()
    nbytes = lib.okt_adamw_plan_bytes(table, count)
    host, chunks = torch.empty(max(nbytes, 256), dtype=torch.uint8), c_u32(0)
    _check("okt_adamw_plan", lib.okt_adamw_plan(table, count, 1 if eight else 0, host.data_ptr(), nbytes,
                                                ctypes.cast(ctypes.pointer(chunks), c_vp)))
    return AdamWPlan(host.to(device), count, chunks.value, 1 if eight else 0, held)


def okt_adamw_step(plan: AdamWPlan, step, *, lr, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, grad_scale=None,
                   skip=None, seed=None, site: int = 0, stream=None) -> None:
    """One AdamW step over the plan's tensors.  step: int64[1] on the device, counted from 1 (the caller counts); lr: a number
    or float32[1] on the device; grad_scale, skip: float32[1] on the device or None - gradients are
    multiplied by the one, and nothing is changed where the other is not 0; seed: int64[1] on the device, for averages in 8 bits."""
    f32, i64 = _TORCH.float32, _TORCH.int64
    on_device = not isinstance(lr, (int, float))
    for t, name in ((step, "step"), (lr if on_device else None, "lr"), (grad_scale, "grad_scale"), (skip, "skip"), (seed, "seed")):
        if t is not None and t.numel() < 1:
            raise ValueError(f"{name} needs one element")
    op = _ADAMW.pack(plan.tensors, plan.chunks, plan.state, site, 0.0 if on_device else lr, beta1, beta2, eps,
                     _ptr(step, i64, "step"), _ptr(lr, f32, "lr") if on_device else 0, _ptr(grad_scale, f32, "grad_scale", True) or 0,
                     _ptr(skip, f32, "skip", True) or 0, _ptr(seed, i64, "seed", True) or 0)
    handle = _stream_for(stream, plan.device_bytes, step, lr if on_device else None, grad_scale, skip, seed)
    _check("okt_adamw_step", load_library().okt_adamw_step(op, plan.device_bytes.data_ptr(), handle))
