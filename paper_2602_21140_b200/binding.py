"""Python binding of the C ABI in ``include/moe_route.h``.

Argument marshalling only: every step of the path runs in the CUDA kernels of
``csrc/libmoe_route.so``.  PyTorch supplies device memory and streams.  If the
compiled library is missing the import of any ``moe_*`` name fails loudly;
there is no CPU or PyTorch fallback.

Two layers:
  * ``moe_route_init`` ... ``moe_route_destroy``: one function per C entry point,
    same names, taking raw pointers / ctypes structs.
  * ``MoeRouter``: a small convenience class that owns a context and the output
    tensors of a dispatch, and passes ``tensor.data_ptr()`` and the current
    stream to the functions above.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass, field

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "csrc", "libmoe_route.so")
_lib_handle = None

MOE_OK = 0
MOE_ERR_INVALID_ARG = 1
MOE_ERR_CUDA = 2
MOE_ERR_INSUFFICIENT_EXPERTS = 3
MOE_ERR_CAPACITY = 4
MOE_ERR_DEVICE_TIMEOUT = 5
MOE_SCORE_SOFTMAX = 0
MOE_SCORE_SIGMOID = 1
MOE_ROUTE_DENSE_TP = 2
MOE_DTYPE_BF16, MOE_DTYPE_F16, MOE_DTYPE_F32 = range(3)
# options of moe_set_tuning (include/moe_route.h, moe_tuning_option)
(MOE_TUNE_PDL, MOE_TUNE_SCATTER_IMPL, MOE_TUNE_SCATTER_BULK_STAGES, MOE_TUNE_SCATTER_BULK_CTAS_PER_SM,
 MOE_TUNE_SCATTER_BLOCKS_PER_SM, MOE_TUNE_SCATTER_UNROLL, MOE_TUNE_COMBINE_IMPL, MOE_TUNE_COMBINE_CHUNK,
 MOE_TUNE_COMBINE_STAGES, MOE_TUNE_COMBINE_WARPS, MOE_TUNE_COMBINE_CTAS_PER_SM,
 MOE_TUNE_ROUTE_LANES_PER_TOKEN, MOE_TUNE_ROUTE_TOKENS_PER_TILE, MOE_TUNE_SPIN_LIMIT,
 MOE_TUNE_ROUTE_PREFETCH, MOE_TUNE_SCATTER_STORE_POLICY) = range(16)

EXPORTED_SYMBOLS = (
    "moe_route_init", "moe_set_failed_ranks", "moe_update_replica_map", "moe_dispatch",
    "moe_combine", "moe_step_host", "moe_step_host_async", "moe_set_timing_event", "moe_get_device_status", "moe_plan_routing_state",
    "moe_workspace_bytes", "moe_route_destroy", "moe_status_string", "moe_permute_static",
    "moe_set_failed_experts", "moe_compact_ranks", "moe_set_rank_order",
    "moe_ep_attach", "moe_ep_route", "moe_ep_scatter", "moe_ep_combine", "moe_ep_plan_host",
    "moe_set_tuning", "moe_debug_skip_ticket",
    "moe_mx_scale_pitch", "moe_mx_quantize", "moe_mx_dequantize", "moe_mx_dispatch", "moe_mx_expert_product",
    "moe_mx_expert_gated", "moe_combine_backward", "moe_dispatch_backward",
    "moe_expert_product", "moe_expert_gated", "moe_expert_rows_backward", "moe_expert_gated_backward", "moe_expert_weight_backward",
    "moe_kept_dequantize", "moe_rms_norm", "moe_rms_norm_backward", "moe_rms_norm_backward_workspace", "moe_redispatch",
)


class MoeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {moe_status_string(status)}")


class moe_config(ctypes.Structure):
    _fields_ = [("num_experts", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("max_tokens", ctypes.c_int32),
                ("num_ranks", ctypes.c_int32), ("slots_per_rank", ctypes.c_int32),
                ("max_replicas", ctypes.c_int32), ("score_func", ctypes.c_int32),
                ("n_group", ctypes.c_int32), ("topk_group", ctypes.c_int32),
                ("replica_policy", ctypes.c_int32), ("route_scale", ctypes.c_float)]


class moe_dispatch_out(ctypes.Structure):
    _fields_ = [("topk_ids", ctypes.c_void_p), ("topk_weights", ctypes.c_void_p),
                ("topk_slot", ctypes.c_void_p), ("slot_counts", ctypes.c_void_p),
                ("slot_offsets", ctypes.c_void_p), ("rank_counts", ctypes.c_void_p),
                ("rank_offsets", ctypes.c_void_p), ("dst_row", ctypes.c_void_p),
                ("src_index", ctypes.c_void_p), ("send_buf", ctypes.c_void_p)]


class moe_ep_group(ctypes.Structure):
    _fields_ = [("world", ctypes.c_int32), ("rank", ctypes.c_int32),
                ("recv_bufs", ctypes.POINTER(ctypes.c_void_p)), ("recv_rows", ctypes.c_int64)]


def library_path() -> str:
    return _LIB_PATH


def _lib():
    global _lib_handle
    if _lib_handle is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                f"{_LIB_PATH} is missing: build it with "
                "`python -m paper_2602_21140_b200.build` (needs nvcc); there is no fallback path")
        lib = ctypes.CDLL(_LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        lib.moe_route_init.restype = ctypes.c_int
        lib.moe_route_init.argtypes = [ctypes.POINTER(moe_config), vp, vp, vp, vp, ctypes.POINTER(vp)]
        lib.moe_set_failed_ranks.restype = ctypes.c_int
        lib.moe_set_failed_ranks.argtypes = [vp, vp, i32, vp]
        lib.moe_set_failed_experts.restype = ctypes.c_int
        lib.moe_set_failed_experts.argtypes = [vp, vp, i32, vp]
        lib.moe_compact_ranks.restype = ctypes.c_int
        lib.moe_compact_ranks.argtypes = [i32, vp, i32, i32, i32, vp, ctypes.POINTER(i32)]
        lib.moe_set_rank_order.restype = ctypes.c_int
        lib.moe_set_rank_order.argtypes = [vp, vp, i32, vp]
        lib.moe_update_replica_map.restype = ctypes.c_int
        lib.moe_update_replica_map.argtypes = [vp, vp, vp]
        lib.moe_dispatch.restype = ctypes.c_int
        lib.moe_dispatch.argtypes = [vp, vp, vp, i32, ctypes.POINTER(moe_dispatch_out), vp]
        lib.moe_combine.restype = ctypes.c_int
        lib.moe_combine.argtypes = [vp, vp, i32, vp, vp]
        lib.moe_step_host.restype = ctypes.c_int
        lib.moe_step_host.argtypes = [vp, vp, vp, i32, ctypes.POINTER(moe_dispatch_out), vp, vp, vp, vp, vp]
        lib.moe_step_host_async.restype = ctypes.c_int
        lib.moe_step_host_async.argtypes = [vp, vp, vp, i32, ctypes.POINTER(moe_dispatch_out), vp, vp, vp, vp, vp]
        lib.moe_set_timing_event.restype = ctypes.c_int
        lib.moe_set_timing_event.argtypes = [vp, vp]
        lib.moe_get_device_status.restype = ctypes.c_int
        lib.moe_get_device_status.argtypes = [vp, ctypes.POINTER(i32)]
        lib.moe_plan_routing_state.restype = ctypes.c_int
        lib.moe_plan_routing_state.argtypes = [ctypes.POINTER(moe_config), vp, vp, i32, vp, vp,
                                               ctypes.POINTER(i32)]
        lib.moe_workspace_bytes.restype = ctypes.c_size_t
        lib.moe_workspace_bytes.argtypes = [ctypes.POINTER(moe_config)]
        lib.moe_route_destroy.restype = ctypes.c_int
        lib.moe_route_destroy.argtypes = [vp]
        lib.moe_permute_static.restype = ctypes.c_int
        lib.moe_permute_static.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp]
        lib.moe_ep_attach.restype = ctypes.c_int
        lib.moe_ep_attach.argtypes = [vp, ctypes.POINTER(moe_ep_group), vp]
        lib.moe_ep_route.restype = ctypes.c_int
        lib.moe_ep_route.argtypes = [vp, vp, i32, ctypes.POINTER(moe_dispatch_out), vp]
        lib.moe_ep_scatter.restype = ctypes.c_int
        lib.moe_ep_scatter.argtypes = [vp, vp, i32, vp, vp, vp]
        lib.moe_ep_combine.restype = ctypes.c_int
        lib.moe_ep_combine.argtypes = [vp, i32, vp, vp]
        lib.moe_ep_plan_host.restype = ctypes.c_int
        lib.moe_ep_plan_host.argtypes = [vp, i32, i32, i32, vp, vp]
        lib.moe_set_tuning.restype = ctypes.c_int
        lib.moe_set_tuning.argtypes = [vp, i32, i32]
        lib.moe_debug_skip_ticket.restype = ctypes.c_int
        lib.moe_debug_skip_ticket.argtypes = [vp]
        lib.moe_mx_scale_pitch.restype = i32
        lib.moe_mx_scale_pitch.argtypes = [i32]
        lib.moe_mx_quantize.restype = ctypes.c_int
        lib.moe_mx_quantize.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp]
        lib.moe_mx_dequantize.restype = ctypes.c_int
        lib.moe_mx_dequantize.argtypes = [vp, vp, i64, i32, vp, i32, i64, vp]
        lib.moe_mx_dispatch.restype = ctypes.c_int
        lib.moe_mx_dispatch.argtypes = [vp, vp, vp, i32, ctypes.POINTER(moe_dispatch_out), vp, vp, vp]
        lib.moe_mx_expert_product.restype = ctypes.c_int
        lib.moe_mx_expert_product.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, i32, i32, vp, vp]
        lib.moe_mx_expert_gated.restype = ctypes.c_int
        lib.moe_mx_expert_gated.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, i32, i32, vp, vp, vp]
        lib.moe_combine_backward.restype = ctypes.c_int
        lib.moe_combine_backward.argtypes = [vp, vp, vp, i32, vp, vp, vp]
        lib.moe_dispatch_backward.restype = ctypes.c_int
        lib.moe_dispatch_backward.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp]
        lib.moe_expert_product.restype = ctypes.c_int
        lib.moe_expert_product.argtypes = [vp, vp, i64, vp, vp, vp, i32, i32, vp, vp]
        lib.moe_expert_gated.restype = ctypes.c_int
        lib.moe_expert_gated.argtypes = [vp, vp, i64, vp, vp, vp, i32, i32, vp, vp, vp, vp]
        lib.moe_expert_rows_backward.restype = ctypes.c_int
        lib.moe_expert_rows_backward.argtypes = [vp, vp, i64, vp, vp, vp, i32, i32, vp, vp]
        lib.moe_expert_gated_backward.restype = ctypes.c_int
        lib.moe_expert_gated_backward.argtypes = [vp, vp, i64, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp]
        lib.moe_expert_weight_backward.restype = ctypes.c_int
        lib.moe_expert_weight_backward.argtypes = [vp, vp, vp, i64, vp, vp, i32, i32, vp, i32, i32, vp]
        lib.moe_kept_dequantize.restype = ctypes.c_int
        lib.moe_kept_dequantize.argtypes = [vp, vp, i64, i32, vp, i32, i64, vp]
        lib.moe_rms_norm.restype = ctypes.c_int
        lib.moe_rms_norm.argtypes = [vp, i64, vp, i64, i32, i64, i32, vp, i32, ctypes.c_float, vp, vp, vp, vp, vp, vp]
        lib.moe_rms_norm_backward_workspace.restype = ctypes.c_size_t
        lib.moe_rms_norm_backward_workspace.argtypes = [i64, i32]
        lib.moe_rms_norm_backward.restype = ctypes.c_int
        lib.moe_rms_norm_backward.argtypes = [vp, vp, vp, vp, i32, i64, i32, vp, i32, vp, vp, vp, ctypes.c_size_t, vp]
        lib.moe_redispatch.restype = ctypes.c_int
        lib.moe_redispatch.argtypes = [vp, vp, vp, i32, vp, vp]
        lib.moe_status_string.restype = ctypes.c_char_p
        lib.moe_status_string.argtypes = [ctypes.c_int]
        _lib_handle = lib
    return _lib_handle


def _np_ptr(a: np.ndarray | None):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a), dtype=np.int32)


def _f32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a), dtype=np.float32)


# --------------------------------------------------------------------------
# one function per C entry point
# --------------------------------------------------------------------------

def moe_status_string(status: int) -> str:
    return _lib().moe_status_string(int(status)).decode()


def moe_workspace_bytes(cfg: moe_config) -> int:
    return int(_lib().moe_workspace_bytes(ctypes.byref(cfg)))


def moe_plan_routing_state(cfg: moe_config, slot_to_expert, failed_ranks):
    """Host-only remap planning.  Returns (status, rank_alive u32[], replica_table i32[E,max_rep], n_available)."""
    s2e = _i32(slot_to_expert)
    fr = _i32(list(failed_ranks))
    words = (cfg.num_ranks + 31) // 32
    alive = np.zeros(max(words, 1), np.uint32)
    table = np.full((max(cfg.num_experts, 1), max(cfg.max_replicas, 1)), -1, np.int32)
    n_avail = ctypes.c_int32(0)
    st = _lib().moe_plan_routing_state(ctypes.byref(cfg), _np_ptr(s2e), _np_ptr(fr) if fr.size else None,
                                       fr.size, _np_ptr(alive), _np_ptr(table), ctypes.byref(n_avail))
    return st, alive, table, int(n_avail.value)


def moe_route_init(cfg: moe_config, slot_to_expert, bias, slot_scale, cuda_stream: int = 0):
    """Returns (status, ctx handle or None)."""
    s2e = _i32(slot_to_expert)
    b = None if bias is None else _f32(bias)
    sc = _f32(slot_scale)
    if s2e.size != cfg.num_ranks * cfg.slots_per_rank or sc.size != s2e.size:
        return MOE_ERR_INVALID_ARG, None
    if b is not None and b.size != cfg.num_experts:
        return MOE_ERR_INVALID_ARG, None
    ctx = ctypes.c_void_p()
    st = _lib().moe_route_init(ctypes.byref(cfg), _np_ptr(s2e), _np_ptr(b), _np_ptr(sc),
                               ctypes.c_void_p(cuda_stream), ctypes.byref(ctx))
    return st, (ctx if st == MOE_OK else None)


def moe_set_failed_ranks(ctx, ranks, cuda_stream: int = 0) -> int:
    r = _i32(list(ranks))
    return _lib().moe_set_failed_ranks(ctx, _np_ptr(r) if r.size else None, r.size,
                                       ctypes.c_void_p(cuda_stream))


def moe_set_failed_experts(ctx, mask, cuda_stream: int = 0) -> int:
    """mask: iterable of num_experts flags (non-zero = lost), or None / empty to clear."""
    m = np.zeros(0, np.uint8) if mask is None else np.ascontiguousarray(np.asarray(mask) != 0, dtype=np.uint8)
    return _lib().moe_set_failed_experts(ctx, _np_ptr(m) if m.size else None, m.size,
                                         ctypes.c_void_p(cuda_stream))


def moe_compact_ranks(num_ranks: int, failed_ranks, switched_rank: int = -1, replaced_rank: int = -1):
    """Host-only rank compaction.  Returns (status, list of physical ranks in new logical order)."""
    fr = _i32(list(failed_ranks))
    out = np.full(max(num_ranks, 1), -1, np.int32)
    n = ctypes.c_int32(0)
    st = _lib().moe_compact_ranks(num_ranks, _np_ptr(fr) if fr.size else None, fr.size, switched_rank,
                                  replaced_rank, _np_ptr(out), ctypes.byref(n))
    return st, out[: n.value].tolist()


def moe_set_rank_order(ctx, logical_to_physical, cuda_stream: int = 0) -> int:
    o = _i32(list(logical_to_physical))
    return _lib().moe_set_rank_order(ctx, _np_ptr(o) if o.size else None, o.size, ctypes.c_void_p(cuda_stream))


def moe_update_replica_map(ctx, slot_to_expert, cuda_stream: int = 0) -> int:
    s2e = _i32(slot_to_expert)
    return _lib().moe_update_replica_map(ctx, _np_ptr(s2e), ctypes.c_void_p(cuda_stream))


def moe_dispatch(ctx, logits_ptr: int, x_ptr: int, T: int, out: moe_dispatch_out,
                 cuda_stream: int = 0) -> int:
    return _lib().moe_dispatch(ctx, ctypes.c_void_p(logits_ptr), ctypes.c_void_p(x_ptr), T,
                               ctypes.byref(out), ctypes.c_void_p(cuda_stream))


def moe_combine(ctx, expert_buf_ptr: int, T: int, y_ptr: int, cuda_stream: int = 0) -> int:
    return _lib().moe_combine(ctx, ctypes.c_void_p(expert_buf_ptr), T, ctypes.c_void_p(y_ptr),
                              ctypes.c_void_p(cuda_stream))


def moe_step_host(ctx, logits_host_ptr: int, x_host_ptr: int, T: int, out: moe_dispatch_out,
                  logits_dev_ptr: int, x_dev_ptr: int, y_dev_ptr: int, y_host_ptr: int,
                  cuda_stream: int = 0) -> int:
    vp = ctypes.c_void_p
    return _lib().moe_step_host(ctx, vp(logits_host_ptr), vp(x_host_ptr), T, ctypes.byref(out),
                                vp(logits_dev_ptr), vp(x_dev_ptr), vp(y_dev_ptr), vp(y_host_ptr),
                                vp(cuda_stream))


def moe_step_host_async(ctx, logits_host_ptr: int, x_host_ptr: int, T: int, out: moe_dispatch_out,
                        logits_dev_ptr: int, x_dev_ptr: int, y_dev_ptr: int, y_host_ptr: int,
                        cuda_stream: int = 0) -> int:
    vp = ctypes.c_void_p
    return _lib().moe_step_host_async(ctx, vp(logits_host_ptr), vp(x_host_ptr), T, ctypes.byref(out),
                                      vp(logits_dev_ptr), vp(x_dev_ptr), vp(y_dev_ptr), vp(y_host_ptr),
                                      vp(cuda_stream))


def moe_set_timing_event(ctx, cuda_event: int) -> int:
    return _lib().moe_set_timing_event(ctx, ctypes.c_void_p(cuda_event) if cuda_event else None)


def moe_set_tuning(ctx, option: int, value: int) -> int:
    return _lib().moe_set_tuning(ctx, int(option), int(value))


def moe_debug_skip_ticket(ctx) -> int:
    return _lib().moe_debug_skip_ticket(ctx)


def moe_get_device_status(ctx):
    code = ctypes.c_int32(0)
    st = _lib().moe_get_device_status(ctx, ctypes.byref(code))
    return st, int(code.value)


def moe_permute_static(topk_slot_ptr: int, n_assign: int, num_ranks: int, slots_per_rank: int,
                       slot_counts_ptr: int, slot_offsets_ptr: int, rank_counts_ptr: int,
                       rank_offsets_ptr: int, dst_row_ptr: int, src_index_ptr: int,
                       cuda_stream: int = 0) -> int:
    """Count / scan / stable permutation from caller-owned device buffers, using only the
    library's built-in scratch array: for callers that are not able to allocate device
    memory (see include/moe_route.h).  All pointer arguments are raw device addresses."""
    vp = ctypes.c_void_p
    return _lib().moe_permute_static(vp(topk_slot_ptr), n_assign, num_ranks, slots_per_rank,
                                     vp(slot_counts_ptr), vp(slot_offsets_ptr), vp(rank_counts_ptr),
                                     vp(rank_offsets_ptr), vp(dst_row_ptr), vp(src_index_ptr),
                                     vp(cuda_stream))


def moe_ep_attach(ctx, world: int, rank: int, recv_buf_ptrs, recv_rows: int, cuda_stream: int = 0) -> int:
    """recv_buf_ptrs: `world` raw device addresses, usable from the calling GPU."""
    ptrs = (ctypes.c_void_p * max(world, 1))(*[int(a) for a in recv_buf_ptrs])
    group = moe_ep_group(world, rank, ctypes.cast(ptrs, ctypes.POINTER(ctypes.c_void_p)), recv_rows)
    return _lib().moe_ep_attach(ctx, ctypes.byref(group), ctypes.c_void_p(cuda_stream))


def moe_ep_route(ctx, logits_ptr: int, T: int, out: moe_dispatch_out, cuda_stream: int = 0) -> int:
    return _lib().moe_ep_route(ctx, ctypes.c_void_p(logits_ptr), T, ctypes.byref(out),
                               ctypes.c_void_p(cuda_stream))


def moe_ep_scatter(ctx, x_ptr: int, T: int, counts_all_ptr: int, recv_slot_offsets_ptr: int,
                   cuda_stream: int = 0) -> int:
    vp = ctypes.c_void_p
    return _lib().moe_ep_scatter(ctx, vp(x_ptr), T, vp(counts_all_ptr), vp(recv_slot_offsets_ptr),
                                 vp(cuda_stream))


def moe_ep_combine(ctx, T: int, y_ptr: int, cuda_stream: int = 0) -> int:
    return _lib().moe_ep_combine(ctx, T, ctypes.c_void_p(y_ptr), ctypes.c_void_p(cuda_stream))


def moe_ep_plan_host(counts_all, rank: int):
    """Host-only layout of the exchange.  counts_all: [world, P] ints.
    Returns (status, src_base i32[P], recv_slot_offsets i32[P/world + 1])."""
    c = _i32(counts_all)
    world, P = c.shape
    src_base = np.zeros(P, np.int32)
    recv_off = np.zeros(P // max(world, 1) + 1, np.int32)
    st = _lib().moe_ep_plan_host(_np_ptr(c), world, rank, P, _np_ptr(src_base), _np_ptr(recv_off))
    return st, src_base, recv_off


def moe_mx_scale_pitch(cols: int) -> int:
    return int(_lib().moe_mx_scale_pitch(cols))


def moe_mx_quantize(x_ptr: int, dtype: int, rows: int, cols: int, row_stride: int, codes_ptr: int, scales_ptr: int,
                    cuda_stream: int = 0) -> int:
    return _lib().moe_mx_quantize(x_ptr, dtype, rows, cols, row_stride, codes_ptr, scales_ptr, cuda_stream)


def moe_mx_dequantize(codes_ptr: int, scales_ptr: int, rows: int, cols: int, y_ptr: int, dtype: int, row_stride: int,
                      cuda_stream: int = 0) -> int:
    return _lib().moe_mx_dequantize(codes_ptr, scales_ptr, rows, cols, y_ptr, dtype, row_stride, cuda_stream)


def moe_mx_dispatch(ctx, logits_ptr: int, x_ptr: int, T: int, out: moe_dispatch_out, send_codes_ptr: int,
                    send_scales_ptr: int, cuda_stream: int = 0) -> int:
    return _lib().moe_mx_dispatch(ctx, logits_ptr, x_ptr, T, ctypes.byref(out), send_codes_ptr, send_scales_ptr, cuda_stream)


def moe_mx_expert_product(ctx, a_codes_ptr: int, a_scales_ptr: int, rows: int, slot_counts_ptr: int, slot_offsets_ptr: int,
                          w_codes_ptr: int, w_scales_ptr: int, n_out: int, n_in: int, y_ptr: int, cuda_stream: int = 0) -> int:
    return _lib().moe_mx_expert_product(ctx, a_codes_ptr, a_scales_ptr, rows, slot_counts_ptr, slot_offsets_ptr, w_codes_ptr,
                                        w_scales_ptr, n_out, n_in, y_ptr, cuda_stream)


def moe_mx_expert_gated(ctx, a_codes_ptr: int, a_scales_ptr: int, rows: int, slot_counts_ptr: int, slot_offsets_ptr: int,
                        w_codes_ptr: int, w_scales_ptr: int, n_hidden: int, n_in: int, h_codes_ptr: int, h_scales_ptr: int,
                        cuda_stream: int = 0) -> int:
    return _lib().moe_mx_expert_gated(ctx, a_codes_ptr, a_scales_ptr, rows, slot_counts_ptr, slot_offsets_ptr, w_codes_ptr,
                                      w_scales_ptr, n_hidden, n_in, h_codes_ptr, h_scales_ptr, cuda_stream)


def moe_combine_backward(ctx, expert_buf_ptr: int, dy_ptr: int, T: int, d_expert_buf_ptr: int, d_weights_ptr: int,
                         cuda_stream: int = 0) -> int:
    return _lib().moe_combine_backward(ctx, expert_buf_ptr, dy_ptr, T, d_expert_buf_ptr, d_weights_ptr, cuda_stream)


def moe_dispatch_backward(ctx, logits_ptr: int, d_send_buf_ptr: int, d_weights_ptr: int, T: int, dx_ptr: int,
                          d_logits_ptr: int, cuda_stream: int = 0) -> int:
    """d_weights_ptr and d_logits_ptr may both be 0; logits_ptr may be 0 for softmax scores if no token ran out of experts."""
    return _lib().moe_dispatch_backward(ctx, logits_ptr or None, d_send_buf_ptr, d_weights_ptr or None, T, dx_ptr,
                                        d_logits_ptr or None, cuda_stream)


def moe_kept_dequantize(codes_ptr: int, scales_ptr: int, rows: int, cols: int, y_ptr: int, dtype: int, row_stride: int,
                       cuda_stream: int = 0) -> int:
    return _lib().moe_kept_dequantize(codes_ptr, scales_ptr, rows, cols, y_ptr, dtype, row_stride, cuda_stream)


def moe_rms_norm(x_ptr: int, x_stride: int, residual_ptr: int, residual_stride: int, dtype: int, rows: int, cols: int, weight_ptr: int,
                 weight_dtype: int, eps: float, h_ptr: int, y_ptr: int, rstd_ptr: int, codes_ptr: int, scales_ptr: int,
                 cuda_stream: int = 0) -> int:
    """residual_ptr, h_ptr, rstd_ptr may be 0, and codes_ptr and scales_ptr together (include/moe_route.h)."""
    return _lib().moe_rms_norm(x_ptr, x_stride, residual_ptr or None, residual_stride, dtype, rows, cols, weight_ptr, weight_dtype, eps,
                               h_ptr or None, y_ptr, rstd_ptr or None, codes_ptr or None, scales_ptr or None, cuda_stream)


def moe_rms_norm_backward_workspace(rows: int, cols: int) -> int:
    return int(_lib().moe_rms_norm_backward_workspace(rows, cols))


def moe_rms_norm_backward(dy_ptr: int, dh_ptr: int, h_ptr: int, rstd_ptr: int, dtype: int, rows: int, cols: int, weight_ptr: int,
                          weight_dtype: int, dx_ptr: int, d_weight_ptr: int, workspace_ptr: int, workspace_bytes: int,
                          cuda_stream: int = 0) -> int:
    """dh_ptr may be 0."""
    return _lib().moe_rms_norm_backward(dy_ptr, dh_ptr or None, h_ptr, rstd_ptr, dtype, rows, cols, weight_ptr, weight_dtype, dx_ptr,
                                        d_weight_ptr, workspace_ptr, workspace_bytes, cuda_stream)


@functools.lru_cache(maxsize=256)
def _norm_workspace(rows: int, cols: int) -> int:
    return moe_rms_norm_backward_workspace(rows, cols)


def moe_redispatch(ctx, codes_ptr: int, scales_ptr: int, T: int, send_buf_ptr: int, cuda_stream: int = 0) -> int:
    return _lib().moe_redispatch(ctx, codes_ptr, scales_ptr, T, send_buf_ptr, cuda_stream)


def moe_expert_product(ctx, a_ptr: int, rows: int, slot_counts_ptr: int, slot_offsets_ptr: int, w_ptr: int, n_out: int, n_in: int,
                       y_ptr: int, cuda_stream: int = 0) -> int:
    return _lib().moe_expert_product(ctx, a_ptr, rows, slot_counts_ptr, slot_offsets_ptr, w_ptr, n_out, n_in, y_ptr, cuda_stream)


def moe_expert_gated(ctx, a_ptr: int, rows: int, slot_counts_ptr: int, slot_offsets_ptr: int, w_ptr: int, n_hidden: int, n_in: int,
                     h_ptr: int, z_ptr: int = 0, z_scales_ptr: int = 0, cuda_stream: int = 0) -> int:
    """z_ptr and z_scales_ptr may both be 0 (nothing is kept), or z_scales_ptr alone (kept in bf16)."""
    return _lib().moe_expert_gated(ctx, a_ptr, rows, slot_counts_ptr, slot_offsets_ptr, w_ptr, n_hidden, n_in, h_ptr, z_ptr or None,
                                   z_scales_ptr or None, cuda_stream)


def moe_expert_rows_backward(ctx, dy_ptr: int, rows: int, slot_counts_ptr: int, slot_offsets_ptr: int, w_ptr: int, n_out: int, n_in: int,
                             da_ptr: int, cuda_stream: int = 0) -> int:
    return _lib().moe_expert_rows_backward(ctx, dy_ptr, rows, slot_counts_ptr, slot_offsets_ptr, w_ptr, n_out, n_in, da_ptr, cuda_stream)


def moe_expert_gated_backward(ctx, dy_ptr: int, rows: int, slot_counts_ptr: int, slot_offsets_ptr: int, w_ptr: int, n_out: int,
                              n_hidden: int, z_ptr: int, z_scales_ptr: int, dz_ptr: int, h_ptr: int, cuda_stream: int = 0) -> int:
    """z_scales_ptr may be 0: z is bf16."""
    return _lib().moe_expert_gated_backward(ctx, dy_ptr, rows, slot_counts_ptr, slot_offsets_ptr, w_ptr, n_out, n_hidden, z_ptr,
                                            z_scales_ptr or None, dz_ptr, h_ptr, cuda_stream)


def moe_expert_weight_backward(ctx, dy_ptr: int, a_ptr: int, rows: int, slot_counts_ptr: int, slot_offsets_ptr: int, n_out: int,
                               n_in: int, dw_ptr: int, dtype: int, add: int, cuda_stream: int = 0) -> int:
    return _lib().moe_expert_weight_backward(ctx, dy_ptr, a_ptr, rows, slot_counts_ptr, slot_offsets_ptr, n_out, n_in, dw_ptr, dtype,
                                             add, cuda_stream)


def moe_route_destroy(ctx) -> int:
    return _lib().moe_route_destroy(ctx)


# --------------------------------------------------------------------------
# convenience layer over torch tensors
# --------------------------------------------------------------------------

@dataclass
class DispatchBuffers:
    """Device tensors written by one dispatch (caller-owned, reusable)."""
    topk_ids: torch.Tensor
    topk_weights: torch.Tensor
    topk_slot: torch.Tensor
    slot_counts: torch.Tensor
    slot_offsets: torch.Tensor
    rank_counts: torch.Tensor
    rank_offsets: torch.Tensor
    dst_row: torch.Tensor
    src_index: torch.Tensor
    send_buf: torch.Tensor | None      # None: the buffers of a dispatch with 4-bit rows

    def as_struct(self) -> moe_dispatch_out:
        return moe_dispatch_out(self.topk_ids.data_ptr(), self.topk_weights.data_ptr(), self.topk_slot.data_ptr(),
                                self.slot_counts.data_ptr(), self.slot_offsets.data_ptr(), self.rank_counts.data_ptr(),
                                self.rank_offsets.data_ptr(), self.dst_row.data_ptr(), self.src_index.data_ptr(),
                                None if self.send_buf is None else self.send_buf.data_ptr())


@dataclass
class MxRows:
    """4-bit rows (format: include/moe_route.h): any leading dimensions, contiguous."""
    codes: torch.Tensor      # uint8 [..., cols / 2]
    scales: torch.Tensor     # uint8 [..., moe_mx_scale_pitch(cols)]

    @property
    def cols(self) -> int:
        return 2 * self.codes.shape[-1]


@dataclass
class Mx8Rows:
    """8-bit rows (format: include/moe_route.h), in which activations are kept for a backward pass: any leading
    dimensions, contiguous."""
    codes: torch.Tensor      # uint8 [..., cols]
    scales: torch.Tensor     # uint8 [..., moe_mx_scale_pitch(cols)]

    @property
    def cols(self) -> int:
        return self.codes.shape[-1]


_DTYPE_CODE = {torch.bfloat16: MOE_DTYPE_BF16, torch.float16: MOE_DTYPE_F16, torch.float32: MOE_DTYPE_F32}


def _require(ok: bool, where: str) -> None:
    if not ok:
        raise MoeError(MOE_ERR_INVALID_ARG, where)


def _mx_pitch(cols: int) -> int:
    return (cols // 32 + 15) // 16 * 16


def _is_mx(m: MxRows, index: int, lead=None) -> bool:
    """4-bit rows on CUDA device `index`, of leading shape `lead` where one is given."""
    c, s = m.codes, m.scales
    cs, ss = c.shape, s.shape
    return (c.dtype is torch.uint8 and s.dtype is torch.uint8 and c.is_contiguous() and s.is_contiguous() and c.is_cuda and s.is_cuda
            and c.get_device() == index and s.get_device() == index and len(cs) > 0 and cs[-1] % 16 == 0 and cs[:-1] == ss[:-1]
            and ss[-1] == _mx_pitch(2 * cs[-1]) and (lead is None or cs[:-1] == lead))


def _span(t: torch.Tensor):
    """Address and bytes of a contiguous tensor, none where there is no tensor."""
    return (0, 0) if t is None else (t.data_ptr(), t.numel() * t.element_size())


def _apart(outputs, inputs) -> bool:
    """Whether outputs share no byte with inputs or with one another, each given by its address and its bytes."""
    spans = [(at, at + size, True) for at, size in outputs if size]
    if not spans:
        return True
    spans += [(at, at + size, False) for at, size in inputs if size]
    spans.sort()
    any_end = out_end = 0                                      # of those that begin before
    for at, end, out in spans:
        if at < out_end or (out and at < any_end):
            return False
        if end > any_end:
            any_end = end
        if out and end > out_end:
            out_end = end
    return True


def _aligned16(*addresses) -> bool:
    together = 0
    for a in addresses:
        together |= a
    return together & 15 == 0


@functools.lru_cache(maxsize=256)
def _network_status(n: int, n_in: int, cols: int, n_out: int, slots: int, grads: bool = False) -> int:
    """What the C calls of a gated network on n rows, or of its gradients, say to its sizes (rows of n_in, two projections of
    cols / 2, n_out)."""
    if n_in < 8 or n_in % 8 or cols < 32 or cols % 32 or n_out < 8 or n_out % 8:
        return MOE_ERR_INVALID_ARG
    most, tiles = 1 << 30, 1 << 29                              # expert_product_fits, weight_grad_fits in csrc/expert_product.h
    for a, b in ((cols, n_in), (n_out, cols // 2)):
        if max(n, a, b) > most or a * b * 2 >= 1 << 39 or (max(a, b) + 127) // 128 * (slots + n // 32) >= tiles:
            return MOE_ERR_CAPACITY
        if grads and ((a + 255) // 256 * ((b + 255) // 256) >= tiles // slots or a * b * 4 >= 1 << 39):
            return MOE_ERR_CAPACITY
    return MOE_OK


def _is_mx8(m: Mx8Rows, index: int, shape) -> bool:
    """8-bit rows of the given logical shape on CUDA device `index`."""
    shape = tuple(shape)
    return (isinstance(m, Mx8Rows) and shape[-1] > 0 and shape[-1] % 32 == 0 and _is_dense(m.codes, torch.uint8, shape, index)
            and _is_dense(m.scales, torch.uint8, (*shape[:-1], _mx_pitch(shape[-1])), index))


def _is_dense(t: torch.Tensor, dtype: torch.dtype, shape, index: int) -> bool:
    return t.dtype is dtype and t.shape == shape and t.get_device() == index >= 0 and t.is_contiguous()   # (-1 on the CPU)


# The current stream of a device as the integer that the C entry points take.  (torch.cuda.current_stream builds
# an object first: 3 of the 15 microseconds that a small call takes on the host.)
def _raw_stream(index: int) -> int:
    return torch._C._cuda_getCurrentRawStream(index)


def _on_device(index: int, call, *args) -> int:
    """call(*args) with that device current (a kernel launch needs its stream's device)."""
    if torch._C._cuda_getDevice() == index:
        return call(*args)
    with torch.cuda.device(index):
        return call(*args)


def mx_empty(*shape, device="cuda") -> MxRows:
    """Uninitialised 4-bit rows of the given logical shape (last dimension: elements of a row)."""
    lead, cols = shape[:-1], shape[-1]
    _require(cols > 0 and cols % 32 == 0, "mx_empty")
    return MxRows(torch.empty((*lead, cols // 2), dtype=torch.uint8, device=device),
                  torch.empty((*lead, _mx_pitch(cols)), dtype=torch.uint8, device=device))


def mx8_empty(*shape, device="cuda") -> Mx8Rows:
    """Uninitialised 8-bit rows of the given shape (last dimension: elements of a row)."""
    lead, cols = shape[:-1], shape[-1]
    _require(cols > 0 and cols % 32 == 0, "mx8_empty")
    return Mx8Rows(torch.empty((*lead, cols), dtype=torch.uint8, device=device),
                   torch.empty((*lead, _mx_pitch(cols)), dtype=torch.uint8, device=device))


def _mx_like(x: torch.Tensor, lead, cols: int) -> MxRows:
    """As mx_empty, on the device of ``x``."""
    return MxRows(x.new_empty((*lead, cols // 2), dtype=torch.uint8), x.new_empty((*lead, _mx_pitch(cols)), dtype=torch.uint8))


def mx_quantize(x: torch.Tensor, out: MxRows | None = None) -> MxRows:
    """Rows of ``x`` ([..., cols], bf16 / fp16 / fp32) in 4 bits, on the current stream of its device.
    A 2-D ``x`` may have any row stride that keeps its rows 16-byte aligned; others are contiguous."""
    shape, code = x.shape, _DTYPE_CODE.get(x.dtype)
    _require(x.is_cuda and code is not None and len(shape) > 0 and shape[-1] > 0 and shape[-1] % 32 == 0, "mx_quantize")
    cols, index, stride = shape[-1], x.get_device(), shape[-1]
    if not x.is_contiguous():
        _require(len(shape) == 2 and x.stride(1) == 1, "mx_quantize")
        stride = x.stride(0)
    if out is None:
        out = _mx_like(x, shape[:-1], cols)
    else:
        _require(_is_mx(out, index, shape[:-1]) and out.cols == cols, "mx_quantize")
    st = _on_device(index, moe_mx_quantize, x.data_ptr(), code, x.numel() // cols, cols, stride, out.codes.data_ptr(),
                    out.scales.data_ptr(), _raw_stream(index))
    if st != MOE_OK:
        raise MoeError(st, "moe_mx_quantize")
    return out


def mx_dequantize(m: MxRows, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that 4-bit rows stand for."""
    index = m.codes.get_device()
    _require(dtype in _DTYPE_CODE and _is_mx(m, index) and m.codes.shape[-1] > 0, "mx_dequantize")
    shape, cols = (*m.codes.shape[:-1], m.cols), m.cols
    stride = cols
    if out is None:
        out = m.codes.new_empty(shape, dtype=dtype)
    else:
        flat = out.is_contiguous()
        _require(out.shape == shape and out.dtype is dtype and out.is_cuda and out.get_device() == index
                 and (flat or (out.dim() == 2 and out.stride(1) == 1)), "mx_dequantize")
        stride = cols if flat else out.stride(0)
    st = _on_device(index, moe_mx_dequantize, m.codes.data_ptr(), m.scales.data_ptr(), out.numel() // cols, cols, out.data_ptr(),
                    _DTYPE_CODE[dtype], stride, _raw_stream(index))
    if st != MOE_OK:
        raise MoeError(st, "moe_mx_dequantize")
    return out


def mx8_dequantize(m: Mx8Rows, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that 8-bit rows stand for."""
    index, shape, cols = m.codes.get_device(), m.codes.shape, m.cols
    _require(dtype in _DTYPE_CODE and len(shape) > 0 and _is_mx8(m, index, shape), "mx8_dequantize")
    stride = cols
    if out is None:
        out = m.codes.new_empty(shape, dtype=dtype)
    else:
        flat = out.is_contiguous()
        _require(out.shape == shape and out.dtype is dtype and out.is_cuda and out.get_device() == index
                 and (flat or (out.dim() == 2 and out.stride(1) == 1)), "mx8_dequantize")
        stride = cols if flat else out.stride(0)
    st = _on_device(index, moe_kept_dequantize, m.codes.data_ptr(), m.scales.data_ptr(), out.numel() // cols, cols, out.data_ptr(),
                    _DTYPE_CODE[dtype], stride, _raw_stream(index))
    if st != MOE_OK:
        raise MoeError(st, "moe_kept_dequantize")
    return out


@dataclass
class RmsNormOut:
    """What a norm writes; reusable as its ``out``."""
    y: torch.Tensor                  # the normed rows
    h: torch.Tensor                  # x + residual, x itself without a residual
    rstd: torch.Tensor               # fp32, one per row
    y8: Mx8Rows | None = None        # the normed rows in 8 bits (a call that does not keep them leaves these as they were)
    # An x that a call put into h is the caller's and no later call's output, unless the caller puts it there: which one it
    # is, and the buffer whose place it took.
    lent: torch.Tensor | None = field(default=None, repr=False, compare=False)
    own_h: torch.Tensor | None = field(default=None, repr=False, compare=False)

    def __setattr__(self, name, value):
        if name == "h":
            self.__dict__["lent"] = None
        self.__dict__[name] = value


def _row_stride(t: torch.Tensor, cols: int) -> int:
    """Elements from row to row of [..., cols], or -1: a 2-D tensor may have gaps between its rows, others are contiguous."""
    if t.is_contiguous():
        return cols
    return t.stride(0) if t.dim() == 2 and t.stride(1) == 1 else -1


def rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: torch.Tensor | None = None, eps: float = 1e-6, keep: bool = False,
             out: RmsNormOut | None = None) -> RmsNormOut:
    """Root-mean-square norm of ``x`` + ``residual`` ([..., cols], bf16 / fp16 / fp32) times ``weight`` (any of these types), on the
    current stream of its device.  ``keep``: also in 8 bits, for a backward pass.  ``out.h`` may be ``residual``
    itself, where the caller has put it there."""
    shape, dtype, index = x.shape, x.dtype, x.get_device()
    code, w_code = _DTYPE_CODE.get(dtype), _DTYPE_CODE.get(weight.dtype)
    _require(index >= 0 and code is not None and w_code is not None and len(shape) > 0 and shape[-1] > 0, "rms_norm")
    cols, x_stride, r_stride = shape[-1], _row_stride(x, shape[-1]), 0
    ok = (x_stride >= 0 and weight.get_device() == index and weight.dim() == 1 and weight.shape[0] == cols and weight.is_contiguous())
    if residual is not None:
        r_stride = _row_stride(residual, cols)
        ok = ok and r_stride >= 0 and residual.shape == shape and residual.dtype is dtype and residual.get_device() == index
    _require(ok, "rms_norm")
    # (empty_like of a contiguous tensor: a third of the time on the host that a shape takes)
    like = x if x_stride == cols and x.is_contiguous() else None
    if out is None:
        y8 = Mx8Rows(x.new_empty(shape, dtype=torch.uint8), x.new_empty((*shape[:-1], _mx_pitch(cols)), dtype=torch.uint8)) if keep else None
        h = None
        out = RmsNormOut.__new__(RmsNormOut)                    # (its __init__: 1 of the 14 microseconds that a small call takes on the host)
        out.__dict__.update(y=x.new_empty(shape) if like is None else torch.empty_like(like), y8=y8,
                            rstd=torch.empty(shape[:-1], dtype=torch.float32, device=x.device))
    else:
        h = out.h if out.lent is None else out.own_h
        _require(_is_dense(out.y, dtype, shape, index) and (residual is None or h is None or _is_dense(h, dtype, shape, index))
                 and _is_dense(out.rstd, torch.float32, shape[:-1], index) and (not keep or _is_mx8(out.y8, index, shape)), "rms_norm")
    r_ptr, h_ptr = 0, 0
    if residual is not None:
        if h is None:
            h = x.new_empty(shape) if like is None else torch.empty_like(like)
        r_ptr, h_ptr = residual.data_ptr(), h.data_ptr()
    c_ptr, s_ptr = (out.y8.codes.data_ptr(), out.y8.scales.data_ptr()) if keep else (0, 0)
    st = _on_device(index, moe_rms_norm, x.data_ptr(), x_stride, r_ptr, r_stride, code, x.numel() // cols, cols, weight.data_ptr(), w_code, eps,
                    h_ptr, out.y.data_ptr(), out.rstd.data_ptr(), c_ptr, s_ptr, _raw_stream(index))
    if st != MOE_OK:
        raise MoeError(st, "moe_rms_norm")
    out.__dict__.update(h=x if residual is None else h, lent=x if residual is None else None, own_h=h)
    return out


def rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, rstd: torch.Tensor, weight: torch.Tensor, dh: torch.Tensor | None = None,
                      dx: torch.Tensor | None = None, d_weight: torch.Tensor | None = None):
    """Gradient of rms_norm: (dx, d_weight), dx by x and by the residual alike, d_weight in fp32.  ``h`` and ``rstd``: of the
    forward; ``dh``: the gradient that comes to h past the norm.  ``dx`` may be dy, dh or h itself."""
    shape, dtype, index = dy.shape, dy.dtype, dy.get_device()
    code = _DTYPE_CODE.get(dtype)
    _require(index >= 0 and code is not None and len(shape) > 0 and shape[-1] > 0, "rms_norm_backward")
    cols = shape[-1]
    n = dy.numel() // cols
    dx = torch.empty_like(dy) if dx is None else dx
    d_weight = torch.empty(cols, dtype=torch.float32, device=dy.device) if d_weight is None else d_weight
    _require(dy.is_contiguous() and _is_dense(h, dtype, shape, index) and _is_dense(dx, dtype, shape, index)
             and (dh is None or _is_dense(dh, dtype, shape, index)) and _is_dense(rstd, torch.float32, shape[:-1], index)
             and weight.dtype in _DTYPE_CODE and _is_dense(weight, weight.dtype, (cols,), index)
             and _is_dense(d_weight, torch.float32, (cols,), index), "rms_norm_backward")
    ws = torch.empty(_norm_workspace(n, cols), dtype=torch.uint8, device=dy.device)
    st = _on_device(index, moe_rms_norm_backward, dy.data_ptr(), 0 if dh is None else dh.data_ptr(), h.data_ptr(), rstd.data_ptr(), code, n,
                    cols, weight.data_ptr(), _DTYPE_CODE[weight.dtype], dx.data_ptr(), d_weight.data_ptr(), ws.data_ptr(), ws.numel(),
                    _raw_stream(index))
    if st != MOE_OK:
        raise MoeError(st, "moe_rms_norm_backward")
    return dx, d_weight


def make_config(num_experts, top_k, hidden, max_tokens, num_ranks, slots_per_rank, max_replicas=2,
                score_func=MOE_SCORE_SOFTMAX, n_group=1, topk_group=1, route_scale=1.0) -> moe_config:
    return moe_config(num_experts, top_k, hidden, max_tokens, num_ranks, slots_per_rank,
                      max_replicas, score_func, n_group, topk_group, 0, route_scale)


class MoeRouter:
    """Owns one library context on a CUDA device."""

    def __init__(self, cfg: moe_config, slot_to_expert, bias, slot_scale, device="cuda:0"):
        self.cfg = cfg
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise RuntimeError("MoeRouter needs a CUDA device; there is no CPU path")
        if self.device.index is None:            # the device that is current now is the context's from here on
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._ctx = None
        self._latest = None      # what the context still points at: see _keep
        with torch.cuda.device(self.device):
            st, ctx = moe_route_init(cfg, slot_to_expert, bias, slot_scale, self._stream())
        if st != MOE_OK:
            raise MoeError(st, "moe_route_init")
        self._ctx = ctx

    # -- helpers ----------------------------------------------------------
    def _stream(self) -> int:
        return torch.cuda.current_stream(self.device).cuda_stream

    def _keep(self, out: DispatchBuffers, status: int) -> None:
        """Hold the buffers that a later combine or gradient of this dispatch reads: the context has their addresses,
        and the caller may drop ``out`` (mx_step returns y alone).  A call that was refused changed nothing."""
        if status not in (MOE_ERR_INVALID_ARG, MOE_ERR_CAPACITY):
            self._latest = (out.topk_ids, out.topk_weights, out.topk_slot, out.dst_row)

    @property
    def num_slots(self) -> int:
        return self.cfg.num_ranks * self.cfg.slots_per_rank

    def alloc_outputs(self, T: int, send_buf: bool = True) -> DispatchBuffers:
        c, dev = self.cfg, self.device
        n = T * c.top_k
        i32 = dict(dtype=torch.int32, device=dev)
        return DispatchBuffers(
            topk_ids=torch.empty((T, c.top_k), **i32),
            topk_weights=torch.empty((T, c.top_k), dtype=torch.float32, device=dev),
            topk_slot=torch.empty((T, c.top_k), **i32),
            slot_counts=torch.empty(self.num_slots, **i32),
            slot_offsets=torch.empty(self.num_slots + 1, **i32),
            rank_counts=torch.empty(c.num_ranks, **i32),
            rank_offsets=torch.empty(c.num_ranks + 1, **i32),
            dst_row=torch.empty(n, **i32),
            src_index=torch.empty(n, **i32),
            send_buf=torch.empty((n, c.hidden), dtype=torch.bfloat16, device=dev) if send_buf else None)

    # -- recovery -----------------------------------------------------------
    def set_failed_ranks(self, ranks) -> None:
        st = moe_set_failed_ranks(self._ctx, ranks, self._stream())
        if st != MOE_OK:
            raise MoeError(st, "moe_set_failed_ranks")

    def set_failed_experts(self, mask) -> None:
        st = moe_set_failed_experts(self._ctx, mask, self._stream())
        if st != MOE_OK:
            raise MoeError(st, "moe_set_failed_experts")

    def set_rank_order(self, logical_to_physical) -> None:
        st = moe_set_rank_order(self._ctx, logical_to_physical, self._stream())
        if st != MOE_OK:
            raise MoeError(st, "moe_set_rank_order")

    def update_replica_map(self, slot_to_expert) -> None:
        st = moe_update_replica_map(self._ctx, slot_to_expert, self._stream())
        if st != MOE_OK:
            raise MoeError(st, "moe_update_replica_map")

    # -- hot path -----------------------------------------------------------
    def dispatch(self, logits: torch.Tensor, x: torch.Tensor, out: DispatchBuffers | None = None) -> DispatchBuffers:
        T = logits.shape[0]
        assert logits.dtype == torch.float32 and logits.is_contiguous() and logits.shape[1] == self.cfg.num_experts
        assert x.dtype == torch.bfloat16 and x.is_contiguous() and tuple(x.shape) == (T, self.cfg.hidden)
        if out is None:
            out = self.alloc_outputs(T)
        struct = out.as_struct()
        st = moe_dispatch(self._ctx, logits.data_ptr(), x.data_ptr(), T, struct, self._stream())
        self._keep(out, st)
        if st != MOE_OK:
            raise MoeError(st, "moe_dispatch")
        return out

    def combine(self, expert_buf: torch.Tensor, T: int, y: torch.Tensor | None = None) -> torch.Tensor:
        assert expert_buf.dtype == torch.bfloat16 and expert_buf.is_contiguous()
        if y is None:
            y = torch.empty((T, self.cfg.hidden), dtype=torch.bfloat16, device=self.device)
        st = moe_combine(self._ctx, expert_buf.data_ptr(), T, y.data_ptr(), self._stream())
        if st != MOE_OK:
            raise MoeError(st, "moe_combine")
        return y

    # -- 4-bit rows: dispatch and the experts' products ----------------------
    def _index(self) -> int:
        return self.device.index

    def mx_dispatch(self, logits: torch.Tensor, x: torch.Tensor, out: DispatchBuffers | None = None,
                    rows: MxRows | None = None):
        """As dispatch, with a send buffer of 4-bit rows.  Returns (buffers, rows)."""
        c, dev = self.cfg, self._index()
        T, H = x.shape[0], c.hidden
        _require(_is_dense(logits, torch.float32, (T, c.num_experts), dev) and _is_dense(x, torch.bfloat16, (T, H), dev), "mx_dispatch")
        if out is None:
            out = self.alloc_outputs(T, send_buf=False)
        else:
            _require(self._outputs_ok(out, T, dev), "mx_dispatch")
        if rows is None:
            rows = _mx_like(x, (T * c.top_k,), H)
        else:
            _require(_is_mx(rows, dev, (T * c.top_k,)) and rows.cols == H, "mx_dispatch")
        st = moe_mx_dispatch(self._ctx, logits.data_ptr(), x.data_ptr(), T, out.as_struct(), rows.codes.data_ptr(),
                             rows.scales.data_ptr(), _raw_stream(dev))
        self._keep(out, st)
        if st != MOE_OK:
            raise MoeError(st, "moe_mx_dispatch")
        return out, rows

    def _outputs_ok(self, out: DispatchBuffers, T: int, dev: int) -> bool:
        """The index buffers have room for a dispatch of T tokens (send_buf is not among them): the C call takes their
        sizes on trust.  (2 of the 12 microseconds that a small call takes on the host.)"""
        c = self.cfg
        R, n, i32, weights = c.num_ranks, T * c.top_k, torch.int32, out.topk_weights
        P = R * c.slots_per_rank
        if weights.dtype is not torch.float32:
            return False
        for t, least in ((weights, n), (out.topk_ids, n), (out.topk_slot, n), (out.dst_row, n), (out.src_index, n), (out.slot_counts, P),
                         (out.slot_offsets, P + 1), (out.rank_counts, R), (out.rank_offsets, R + 1)):
            if t.numel() < least or not t.is_contiguous() or t.get_device() != dev or (t.dtype is not i32 and t is not weights):
                return False
        return True

    def _index_spans(self, out: DispatchBuffers, T: int):
        """What a dispatch of T tokens uses of its index buffers."""
        c = self.cfg
        R, n = 4 * c.num_ranks, 4 * T * c.top_k
        P = R * c.slots_per_rank
        return [(out.topk_ids.data_ptr(), n), (out.topk_weights.data_ptr(), n), (out.topk_slot.data_ptr(), n), (out.slot_counts.data_ptr(), P),
                (out.slot_offsets.data_ptr(), P + 4), (out.rank_counts.data_ptr(), R), (out.rank_offsets.data_ptr(), R + 4),
                (out.dst_row.data_ptr(), n), (out.src_index.data_ptr(), n)]

    def _segments_ok(self, rows: MxRows, slot_counts, slot_offsets, weight: MxRows, dev: int) -> bool:
        P, w = self.num_slots, weight.codes.shape
        return (_is_mx(rows, dev) and len(rows.codes.shape) == 2 and _is_mx(weight, dev) and len(w) == 3 and w[0] == P
                and w[2] == rows.codes.shape[1] and _is_dense(slot_counts, torch.int32, (P,), dev)
                and slot_offsets.dim() == 1 and slot_offsets.shape[0] >= P
                and _is_dense(slot_offsets, torch.int32, slot_offsets.shape, dev))

    def mx_expert_product(self, rows: MxRows, slot_counts: torch.Tensor, slot_offsets: torch.Tensor, weight: MxRows,
                          y: torch.Tensor | None = None) -> torch.Tensor:
        """y[r] = weight[slot of r] @ rows[r]: weight [P, n_out, cols] and rows [n, cols] in 4 bits, y [n, n_out] bf16."""
        dev = self._index()
        _require(self._segments_ok(rows, slot_counts, slot_offsets, weight, dev), "mx_expert_product")
        n, n_out = rows.codes.shape[0], weight.codes.shape[1]
        if y is None:
            y = rows.codes.new_empty((n, n_out), dtype=torch.bfloat16)
        else:
            _require(_is_dense(y, torch.bfloat16, (n, n_out), dev), "mx_expert_product")
        st = moe_mx_expert_product(self._ctx, rows.codes.data_ptr(), rows.scales.data_ptr(), n, slot_counts.data_ptr(),
                                   slot_offsets.data_ptr(), weight.codes.data_ptr(), weight.scales.data_ptr(), n_out, rows.cols,
                                   y.data_ptr(), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_mx_expert_product")
        return y

    def mx_expert_gated(self, rows: MxRows, slot_counts: torch.Tensor, slot_offsets: torch.Tensor, gate_up: MxRows,
                        out: MxRows | None = None) -> MxRows:
        """silu(gate) * up in 4 bits.  gate_up [P, 2 * n_hidden, cols]: row 2i is the gate of feature i, row 2i + 1 its up-projection."""
        dev = self._index()
        _require(self._segments_ok(rows, slot_counts, slot_offsets, gate_up, dev) and gate_up.codes.shape[1] % 64 == 0
                 and gate_up.codes.shape[1] > 0, "mx_expert_gated")
        n, n_hidden = rows.codes.shape[0], gate_up.codes.shape[1] // 2
        if out is None:
            out = _mx_like(rows.codes, (n,), n_hidden)
        else:
            _require(_is_mx(out, dev, (n,)) and out.cols == n_hidden, "mx_expert_gated")
        st = moe_mx_expert_gated(self._ctx, rows.codes.data_ptr(), rows.scales.data_ptr(), n, slot_counts.data_ptr(),
                                 slot_offsets.data_ptr(), gate_up.codes.data_ptr(), gate_up.scales.data_ptr(), n_hidden, rows.cols,
                                 out.codes.data_ptr(), out.scales.data_ptr(), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_mx_expert_gated")
        return out

    def mx_expert_ffn(self, rows: MxRows, slot_counts: torch.Tensor, slot_offsets: torch.Tensor, gate_up: MxRows, down: MxRows,
                      y: torch.Tensor | None = None, hidden: MxRows | None = None) -> torch.Tensor:
        """The gated feed-forward expert of every slot on its rows: mx_expert_gated, then mx_expert_product."""
        hidden = self.mx_expert_gated(rows, slot_counts, slot_offsets, gate_up, hidden)
        return self.mx_expert_product(hidden, slot_counts, slot_offsets, down, y)

    def mx_step(self, logits: torch.Tensor, x: torch.Tensor, gate_up: MxRows, down: MxRows, out: DispatchBuffers | None = None,
                y: torch.Tensor | None = None) -> torch.Tensor:
        """One whole layer: 4-bit dispatch, the experts, and the combine (times slot_scale, as always)."""
        H, P, g, d = self.cfg.hidden, self.num_slots, gate_up.codes.shape, down.codes.shape
        # before the first launch: the combine takes the size of y on trust, and a step that is refused halfway has
        # already replaced the latest dispatch
        _require(len(g) == 3 and g[1] > 0 and g[1] % 64 == 0 and tuple(g) == (P, g[1], H // 2) and tuple(d) == (P, H, g[1] // 4)
                 and (y is None or _is_dense(y, torch.bfloat16, (x.shape[0], H), self._index())), "mx_step")
        out, rows = self.mx_dispatch(logits, x, out)
        buf = self.mx_expert_ffn(rows, out.slot_counts, out.slot_offsets, gate_up, down)
        return _on_device(self._index(), self.combine, buf, x.shape[0], y)

    # -- gradients of the routed step ----------------------------------------
    def combine_backward(self, expert_buf: torch.Tensor, dy: torch.Tensor, d_expert_buf: torch.Tensor | None = None,
                         d_weights: torch.Tensor | None = None):
        """Gradients of the latest combine by its rows and its gate weights: (d_expert_buf, d_weights)."""
        c, T, dev = self.cfg, dy.shape[0], self._index()
        H, k = c.hidden, c.top_k
        ok = _is_dense(expert_buf, torch.bfloat16, (T * k, H), dev) and _is_dense(dy, torch.bfloat16, (T, H), dev)
        if d_expert_buf is None:
            d_expert_buf = torch.empty_like(expert_buf)
        else:
            ok = ok and _is_dense(d_expert_buf, torch.bfloat16, (T * k, H), dev)
        if d_weights is None:
            d_weights = dy.new_empty((T, k), dtype=torch.float32)
        else:
            ok = ok and _is_dense(d_weights, torch.float32, (T, k), dev)
        _require(ok, "combine_backward")
        st = moe_combine_backward(self._ctx, expert_buf.data_ptr(), dy.data_ptr(), T, d_expert_buf.data_ptr(),
                                  d_weights.data_ptr(), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_combine_backward")
        return d_expert_buf, d_weights

    def dispatch_backward(self, logits: torch.Tensor | None, d_send_buf: torch.Tensor, d_weights: torch.Tensor | None = None,
                          dx: torch.Tensor | None = None, d_logits: torch.Tensor | None = None):
        """Gradients of the latest dispatch: (dx, d_logits).  d_logits is None without d_weights.  ``logits``: those of the
        dispatch; None is for softmax scores when no -inf mask left a token with fewer than top_k experts."""
        c, dev = self.cfg, self._index()
        T = d_send_buf.shape[0] // c.top_k
        H, k, E = c.hidden, c.top_k, c.num_experts
        ok = _is_dense(d_send_buf, torch.bfloat16, (T * k, H), dev)
        if dx is None:
            dx = d_send_buf.new_empty((T, H))
        else:
            ok = ok and _is_dense(dx, torch.bfloat16, (T, H), dev)
        if d_weights is not None:
            ok = ok and _is_dense(d_weights, torch.float32, (T, k), dev)
            if d_logits is None:
                d_logits = d_weights.new_empty((T, E))
        if d_logits is not None:
            ok = ok and _is_dense(d_logits, torch.float32, (T, E), dev)
        ok = ok and (logits is None or _is_dense(logits, torch.float32, (T, E), dev))
        _require(ok, "dispatch_backward")
        st = moe_dispatch_backward(self._ctx, 0 if logits is None else logits.data_ptr(), d_send_buf.data_ptr(),
                                   0 if d_weights is None else d_weights.data_ptr(), T, dx.data_ptr(),
                                   0 if d_logits is None else d_logits.data_ptr(), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_dispatch_backward")
        return dx, d_logits

    # -- experts in 16 bits and their gradients --------------------------------
    # (Outside autograd, as all of the binding: results carry no graph, and gradients are calls of their own.)
    def redispatch(self, x8: Mx8Rows, send_buf: torch.Tensor | None = None) -> torch.Tensor:
        """The send buffer [T * k, H] of the latest dispatch once more, from its tokens' rows [T, H] in 8 bits."""
        c, dev = self.cfg, self._index()
        T, H = x8.codes.shape[0], c.hidden
        _require(H % 32 == 0 and _is_mx8(x8, dev, (T, H)), "redispatch")
        if send_buf is None:
            send_buf = x8.codes.new_empty((T * c.top_k, H), dtype=torch.bfloat16)
        else:
            _require(_is_dense(send_buf, torch.bfloat16, (T * c.top_k, H), dev), "redispatch")
        st = moe_redispatch(self._ctx, x8.codes.data_ptr(), x8.scales.data_ptr(), T, send_buf.data_ptr(), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_redispatch")
        return send_buf

    def _expert_ok(self, rows: torch.Tensor, cols: int, slot_counts, slot_offsets, weight: torch.Tensor, dev: int) -> bool:
        """Rows [n, cols] and one matrix [P, n_out, n_in] per slot, in bf16."""
        P = self.num_slots
        return (rows.dim() == 2 and weight.dim() == 3 and weight.shape[0] == P and _is_dense(rows, torch.bfloat16, (rows.shape[0], cols), dev)
                and _is_dense(weight, torch.bfloat16, weight.shape, dev) and self._slots_ok(slot_counts, slot_offsets, dev))

    def _slots_ok(self, slot_counts: torch.Tensor, slot_offsets: torch.Tensor, dev: int) -> bool:
        P = self.num_slots
        return (_is_dense(slot_counts, torch.int32, (P,), dev) and slot_offsets.dim() == 1 and slot_offsets.shape[0] >= P
                and _is_dense(slot_offsets, torch.int32, slot_offsets.shape, dev))

    @staticmethod
    def _kept_ok(z, n: int, cols: int, dev: int) -> bool:
        if z is None:
            return False
        return _is_mx8(z, dev, (n, cols)) if isinstance(z, Mx8Rows) else _is_dense(z, torch.bfloat16, (n, cols), dev)

    @staticmethod
    def _kept_spans(z):
        return [_span(z.codes), _span(z.scales)] if isinstance(z, Mx8Rows) else [_span(z)]

    @staticmethod
    def _kept_ptrs(z):
        return (z.codes.data_ptr(), z.scales.data_ptr()) if isinstance(z, Mx8Rows) else (0 if z is None else z.data_ptr(), 0)

    def expert_product(self, rows: torch.Tensor, slot_counts: torch.Tensor, slot_offsets: torch.Tensor, weight: torch.Tensor,
                       y: torch.Tensor | None = None) -> torch.Tensor:
        """y[r] = weight[slot of r] @ rows[r]: weight [P, n_out, cols], rows [n, cols], y [n, n_out], all bf16."""
        dev = self._index()
        _require(weight.dim() == 3 and self._expert_ok(rows, weight.shape[2], slot_counts, slot_offsets, weight, dev), "expert_product")
        n, (_, n_out, n_in) = rows.shape[0], weight.shape
        if y is None:
            y = rows.new_empty((n, n_out))
        else:
            _require(_is_dense(y, torch.bfloat16, (n, n_out), dev), "expert_product")
        st = moe_expert_product(self._ctx, rows.data_ptr(), n, slot_counts.data_ptr(), slot_offsets.data_ptr(), weight.data_ptr(), n_out,
                                n_in, y.data_ptr(), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_expert_product")
        return y

    def expert_gated(self, rows: torch.Tensor, slot_counts: torch.Tensor, slot_offsets: torch.Tensor, gate_up: torch.Tensor,
                     h: torch.Tensor | None = None, z: "torch.Tensor | Mx8Rows | None" = None) -> torch.Tensor:
        """silu(gate) * up [n, n_hidden].  gate_up [P, 2 * n_hidden, cols]: row 2i is the gate of feature i, row 2i + 1 its
        up-projection.  ``z`` [n, 2 * n_hidden]: bf16 or 8-bit rows that keep the projections for the backward pass."""
        dev = self._index()
        _require(gate_up.dim() == 3 and gate_up.shape[1] > 0 and gate_up.shape[1] % 32 == 0
                 and self._expert_ok(rows, gate_up.shape[2], slot_counts, slot_offsets, gate_up, dev), "expert_gated")
        n, (_, cols, n_in) = rows.shape[0], gate_up.shape
        if h is None:
            h = rows.new_empty((n, cols // 2))
        _require(_is_dense(h, torch.bfloat16, (n, cols // 2), dev) and (z is None or self._kept_ok(z, n, cols, dev)), "expert_gated")
        st = moe_expert_gated(self._ctx, rows.data_ptr(), n, slot_counts.data_ptr(), slot_offsets.data_ptr(), gate_up.data_ptr(),
                              cols // 2, n_in, h.data_ptr(), *self._kept_ptrs(z), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_expert_gated")
        return h

    def expert_ffn(self, rows: torch.Tensor, slot_counts: torch.Tensor, slot_offsets: torch.Tensor, gate_up: torch.Tensor,
                   down: torch.Tensor, y: torch.Tensor | None = None, h: torch.Tensor | None = None,
                   z: "torch.Tensor | Mx8Rows | None" = None) -> torch.Tensor:
        """The gated feed-forward expert of every slot on its rows: expert_gated, then expert_product, refused before the
        first launch where either would be, and where an output shares a byte with an input of either (``y`` may take the place
        of ``rows``) or with another output."""
        dev, n, bf16 = self._index(), rows.shape[0], torch.bfloat16
        P, cols, n_in = gate_up.shape if gate_up.dim() == 3 else (0, 0, 0)
        n_out, n_hidden = down.shape[1] if down.dim() == 3 else 0, cols // 2
        _require(P == self.num_slots and cols > 0 and cols % 32 == 0 and _is_dense(gate_up, bf16, (P, cols, n_in), dev)
                 and _is_dense(down, bf16, (P, n_out, n_hidden), dev) and _is_dense(rows, bf16, (n, n_in), dev)
                 and self._slots_ok(slot_counts, slot_offsets, dev) and (z is None or self._kept_ok(z, n, cols, dev))
                 and (y is None or _is_dense(y, bf16, (n, n_out), dev)) and (h is None or _is_dense(h, bf16, (n, n_hidden), dev)), "expert_ffn")
        st = _network_status(n, n_in, cols, n_out, P)
        if st != MOE_OK:
            raise MoeError(st, "expert_ffn")
        if n:
            r_ptr, g_ptr, d_ptr = rows.data_ptr(), gate_up.data_ptr(), down.data_ptr()
            ok = (r_ptr | g_ptr | d_ptr) & 15 == 0
            if y is not None or h is not None or z is not None:
                kept, h_span, y_span = self._kept_spans(z), _span(h), _span(y)
                ok = (ok and _aligned16(h_span[0], y_span[0], *[at for at, _ in kept])
                      and _apart((y_span, h_span, *kept), ((g_ptr, P * cols * n_in * 2), (d_ptr, P * n_out * n_hidden * 2),
                                                           (slot_counts.data_ptr(), 4 * P), (slot_offsets.data_ptr(), 4 * P)))
                      and _apart((h_span, *kept), ((r_ptr, n * n_in * 2),)))
            _require(ok, "expert_ffn")
        return self._expert_ffn(rows, slot_counts, slot_offsets, gate_up, down, y, h, z)

    def _expert_ffn(self, rows, slot_counts, slot_offsets, gate_up, down, y, h, z) -> torch.Tensor:
        """expert_ffn of arguments that have been looked at."""
        n, (_, cols, n_in), n_out, n_hidden = rows.shape[0], gate_up.shape, down.shape[1], gate_up.shape[1] // 2
        if h is None:
            h = rows.new_empty((n, n_hidden))
        if y is None:
            y = torch.empty_like(rows) if n_out == n_in else rows.new_empty((n, n_out))
        counts, offsets, stream = slot_counts.data_ptr(), slot_offsets.data_ptr(), _raw_stream(self._index())
        st = moe_expert_gated(self._ctx, rows.data_ptr(), n, counts, offsets, gate_up.data_ptr(), n_hidden, n_in, h.data_ptr(),
                              *self._kept_ptrs(z), stream)
        if st == MOE_OK:
            st = moe_expert_product(self._ctx, h.data_ptr(), n, counts, offsets, down.data_ptr(), n_out, n_hidden, y.data_ptr(), stream)
        if st != MOE_OK:
            raise MoeError(st, "expert_ffn")
        return y

    def expert_rows_backward(self, dy: torch.Tensor, slot_counts: torch.Tensor, slot_offsets: torch.Tensor, weight: torch.Tensor,
                             d_rows: torch.Tensor | None = None) -> torch.Tensor:
        """Gradient of expert_product by its rows: dy [n, n_out] -> [n, cols]."""
        dev = self._index()
        _require(weight.dim() == 3 and self._expert_ok(dy, weight.shape[1], slot_counts, slot_offsets, weight, dev), "expert_rows_backward")
        n, (_, n_out, n_in) = dy.shape[0], weight.shape
        if d_rows is None:
            d_rows = dy.new_empty((n, n_in))
        else:
            _require(_is_dense(d_rows, torch.bfloat16, (n, n_in), dev), "expert_rows_backward")
        st = moe_expert_rows_backward(self._ctx, dy.data_ptr(), n, slot_counts.data_ptr(), slot_offsets.data_ptr(), weight.data_ptr(),
                                      n_out, n_in, d_rows.data_ptr(), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_expert_rows_backward")
        return d_rows

    def expert_gated_backward(self, dy: torch.Tensor, slot_counts: torch.Tensor, slot_offsets: torch.Tensor, down: torch.Tensor,
                              z: "torch.Tensor | Mx8Rows", dz: torch.Tensor | None = None, h: torch.Tensor | None = None):
        """From the gradient of an expert's output [n, n_out] and the kept projections: (dz [n, 2 * n_hidden], h [n, n_hidden]),
        the projections' gradient and the hidden rows of the forward pass."""
        dev = self._index()
        _require(down.dim() == 3 and down.shape[2] > 0 and down.shape[2] % 16 == 0 and self._expert_ok(dy, down.shape[1], slot_counts, slot_offsets, down, dev),
                 "expert_gated_backward")
        n, (_, n_out, n_hidden) = dy.shape[0], down.shape
        dz = dy.new_empty((n, 2 * n_hidden)) if dz is None else dz
        h = dy.new_empty((n, n_hidden)) if h is None else h
        _require(_is_dense(dz, torch.bfloat16, (n, 2 * n_hidden), dev) and _is_dense(h, torch.bfloat16, (n, n_hidden), dev)
                 and self._kept_ok(z, n, 2 * n_hidden, dev), "expert_gated_backward")
        st = moe_expert_gated_backward(self._ctx, dy.data_ptr(), n, slot_counts.data_ptr(), slot_offsets.data_ptr(), down.data_ptr(),
                                       n_out, n_hidden, *self._kept_ptrs(z), dz.data_ptr(), h.data_ptr(), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_expert_gated_backward")
        return dz, h

    def expert_weight_backward(self, dy: torch.Tensor, rows: torch.Tensor, slot_counts: torch.Tensor, slot_offsets: torch.Tensor,
                               d_weight: torch.Tensor | None = None, add: bool = False, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        """Gradient of expert_product by its matrices: dy [n, n_out], rows [n, cols] -> [P, n_out, cols] in bf16 or fp32 (``dtype``
        where no ``d_weight`` is given); with ``add`` (fp32) added to ``d_weight``.  Copies of one expert have one each."""
        dev, P = self._index(), self.num_slots
        _require(dy.dim() == 2 and rows.dim() == 2 and _is_dense(dy, torch.bfloat16, dy.shape, dev)
                 and _is_dense(rows, torch.bfloat16, (dy.shape[0], rows.shape[1]), dev) and self._slots_ok(slot_counts, slot_offsets, dev)
                 and not (add and d_weight is None), "expert_weight_backward")
        shape = (P, dy.shape[1], rows.shape[1])
        if d_weight is None:
            _require(dtype in (torch.bfloat16, torch.float32), "expert_weight_backward")
            d_weight = dy.new_empty(shape, dtype=dtype)
        _require(d_weight.dtype in (torch.bfloat16, torch.float32) and _is_dense(d_weight, d_weight.dtype, shape, dev), "expert_weight_backward")
        st = moe_expert_weight_backward(self._ctx, dy.data_ptr(), rows.data_ptr(), dy.shape[0], slot_counts.data_ptr(),
                                        slot_offsets.data_ptr(), shape[1], shape[2], d_weight.data_ptr(), _DTYPE_CODE[d_weight.dtype],
                                        int(add), _raw_stream(dev))
        if st != MOE_OK:
            raise MoeError(st, "moe_expert_weight_backward")
        return d_weight

    def expert_ffn_backward(self, dy: torch.Tensor, rows: torch.Tensor, slot_counts: torch.Tensor, slot_offsets: torch.Tensor,
                            gate_up: torch.Tensor, down: torch.Tensor, z: "torch.Tensor | Mx8Rows", d_rows: torch.Tensor | None = None,
                            d_gate_up: torch.Tensor | None = None, d_down: torch.Tensor | None = None, add: bool = False,
                            grad_dtype: torch.dtype = torch.bfloat16):
        """Gradients of expert_ffn with the projections ``z`` that it kept: (d_rows, d_gate_up, d_down).  ``add``: as in
        expert_weight_backward, for both matrices.  Refused before the first launch where one of the four operators would be, and
        where a given output shares a byte with an input of any of them."""
        dev, n, bf16, f32 = self._index(), dy.shape[0], torch.bfloat16, torch.float32
        P, cols, n_in = gate_up.shape if gate_up.dim() == 3 else (0, 0, 0)
        n_out, n_hidden = down.shape[1] if down.dim() == 3 else 0, cols // 2
        apart = ((d_rows is None and d_gate_up is None and d_down is None)
                 or _apart((_span(d_rows), _span(d_gate_up), _span(d_down)),
                           (*[_span(t) for t in (dy, rows, gate_up, down, slot_counts, slot_offsets)], *self._kept_spans(z))))
        add_ok = not add or (d_gate_up is not None and d_down is not None and d_gate_up.dtype is f32 and d_down.dtype is f32)
        if d_gate_up is None:
            d_gate_up = torch.empty_like(gate_up, dtype=grad_dtype) if grad_dtype is not bf16 else torch.empty_like(gate_up)
        if d_down is None:
            d_down = torch.empty_like(down, dtype=grad_dtype) if grad_dtype is not bf16 else torch.empty_like(down)
        g_type, d_type = d_gate_up.dtype, d_down.dtype
        _require(P == self.num_slots and cols > 0 and cols % 32 == 0 and _is_dense(gate_up, bf16, (P, cols, n_in), dev)
                 and _is_dense(down, bf16, (P, n_out, n_hidden), dev) and _is_dense(dy, bf16, (n, n_out), dev) and _is_dense(rows, bf16, (n, n_in), dev)
                 and self._slots_ok(slot_counts, slot_offsets, dev) and self._kept_ok(z, n, cols, dev)
                 and (d_rows is None or _is_dense(d_rows, bf16, (n, n_in), dev)) and g_type in (bf16, f32) and d_type in (bf16, f32)
                 and _is_dense(d_gate_up, g_type, (P, cols, n_in), dev) and _is_dense(d_down, d_type, (P, n_out, n_hidden), dev)
                 and add_ok and apart, "expert_ffn_backward")
        st = _network_status(n, n_in, cols, n_out, P, True)
        if st != MOE_OK:
            raise MoeError(st, "expert_ffn_backward")
        _require(_aligned16(d_gate_up.data_ptr(), d_down.data_ptr())
                 and (n == 0 or _aligned16(dy.data_ptr(), rows.data_ptr(), gate_up.data_ptr(), down.data_ptr(), 0 if d_rows is None else d_rows.data_ptr(),
                                           *self._kept_ptrs(z))), "expert_ffn_backward")
        if d_rows is None:
            d_rows = torch.empty_like(rows)
        dz, h = dy.new_empty((n, cols)), dy.new_empty((n, n_hidden))
        ctx, counts, offsets, stream = self._ctx, slot_counts.data_ptr(), slot_offsets.data_ptr(), _raw_stream(dev)
        dy_ptr, dz_ptr, h_ptr, add = dy.data_ptr(), dz.data_ptr(), h.data_ptr(), int(add)
        st = moe_expert_gated_backward(ctx, dy_ptr, n, counts, offsets, down.data_ptr(), n_out, n_hidden, *self._kept_ptrs(z), dz_ptr, h_ptr, stream)
        if st == MOE_OK:
            st = moe_expert_weight_backward(ctx, dy_ptr, h_ptr, n, counts, offsets, n_out, n_hidden, d_down.data_ptr(), _DTYPE_CODE[d_type], add, stream)
        if st == MOE_OK:
            st = moe_expert_weight_backward(ctx, dz_ptr, rows.data_ptr(), n, counts, offsets, cols, n_in, d_gate_up.data_ptr(), _DTYPE_CODE[g_type], add,
                                            stream)
        if st == MOE_OK:
            st = moe_expert_rows_backward(ctx, dz_ptr, n, counts, offsets, gate_up.data_ptr(), cols, n_in, d_rows.data_ptr(), stream)
        if st != MOE_OK:
            raise MoeError(st, "expert_ffn_backward")
        return d_rows, d_gate_up, d_down

    def _networks_ok(self, gate_up: torch.Tensor, down: torch.Tensor) -> bool:
        H, P, dev = self.cfg.hidden, self.num_slots, self._index()
        return (gate_up.dim() == 3 and gate_up.shape[1] > 0 and gate_up.shape[1] % 32 == 0
                and _is_dense(gate_up, torch.bfloat16, (P, gate_up.shape[1], H), dev)
                and _is_dense(down, torch.bfloat16, (P, H, gate_up.shape[1] // 2), dev))

    def expert_step(self, logits: torch.Tensor, x: torch.Tensor, gate_up: torch.Tensor, down: torch.Tensor,
                    out: DispatchBuffers | None = None, y: torch.Tensor | None = None, buf: torch.Tensor | None = None,
                    z: "torch.Tensor | Mx8Rows | None" = None) -> torch.Tensor:
        """One whole layer with experts in 16 bits: dispatch, the experts, and the combine (times slot_scale, as always).
        For expert_step_backward keep ``out``, the experts' outputs ``buf`` [T * k, H] and their projections ``z``.  Outputs share no
        byte with inputs, matrices, ``out`` or one another, but ``y`` may take the place of ``x``, and ``buf`` and ``y`` that of the
        send buffer (a backward pass then needs its rows in 8 bits)."""
        T, H, k, dev = x.shape[0], self.cfg.hidden, self.cfg.top_k, self._index()
        # before the first launch: dispatch and combine take the sizes of their buffers on trust
        _require(self._networks_ok(gate_up, down) and _is_dense(x, torch.bfloat16, (T, H), dev)
                 and _is_dense(logits, torch.float32, (T, self.cfg.num_experts), dev)
                 and (y is None or _is_dense(y, torch.bfloat16, (T, H), dev)) and (buf is None or _is_dense(buf, torch.bfloat16, (T * k, H), dev))
                 and (z is None or self._kept_ok(z, T * k, gate_up.shape[1], dev))
                 and (out is None or (self._outputs_ok(out, T, dev) and out.send_buf is not None
                                      and _is_dense(out.send_buf, torch.bfloat16, (T * k, H), dev))), "expert_step")
        st = _network_status(T * k, H, gate_up.shape[1], H, self.num_slots)
        if st != MOE_OK:
            raise MoeError(st, "expert_step")
        if T:
            P, cols, _ = gate_up.shape
            w = [(gate_up.data_ptr(), P * cols * H * 2), (down.data_ptr(), P * cols * H)]
            kept, outs, send = self._kept_spans(z), [_span(y), _span(buf)], _span(None if out is None else out.send_buf)
            _require(_aligned16(send[0], *[at for at, _ in (*w, *kept, *outs)])
                     and ((y is None and buf is None and z is None)
                          or (_apart((*outs, *kept), (*w, (logits.data_ptr(), T * self.cfg.num_experts * 4), *([] if out is None else self._index_spans(out, T))))
                              and _apart(kept, (send,)) and _apart((outs[1], *kept), ((x.data_ptr(), T * H * 2),)))), "expert_step")
        out = _on_device(dev, self.dispatch, logits, x, out)
        buf = self._expert_ffn(out.send_buf, out.slot_counts, out.slot_offsets, gate_up, down, buf, None, z)
        return _on_device(dev, self.combine, buf, T, y)

    def expert_step_backward(self, logits: torch.Tensor, dy: torch.Tensor, rows: "torch.Tensor | Mx8Rows", out: DispatchBuffers,
                             buf: torch.Tensor, z: "torch.Tensor | Mx8Rows", gate_up: torch.Tensor, down: torch.Tensor,
                             d_gate_up: torch.Tensor | None = None, d_down: torch.Tensor | None = None, add: bool = False,
                             grad_dtype: torch.dtype = torch.bfloat16):
        """Gradients of the latest expert_step: (dx, d_logits, d_gate_up, d_down).  ``rows``: its send buffer (where ``buf`` has
        not taken its place), or its tokens' rows x in 8 bits (rms_norm's ``y8``).  d_logits is None for dense-FFN routing,
        whose weights are constants.  Refused before a gradient is written where any of its operators would be."""
        T, H, E, dev, score = dy.shape[0], self.cfg.hidden, self.cfg.num_experts, self._index(), self.cfg.score_func
        # the gradients of combine and dispatch take the context's latest dispatch: it has to be this one
        _require(self._latest is not None and self._latest[3] is out.dst_row
                 and self._networks_ok(gate_up, down) and _is_dense(dy, torch.bfloat16, (T, H), dev) and self._outputs_ok(out, T, dev)
                 and self._kept_ok(z, T * self.cfg.top_k, gate_up.shape[1], dev)
                 and (score != MOE_SCORE_SIGMOID if logits is None else _is_dense(logits, torch.float32, (T, E), dev))
                 and (isinstance(rows, Mx8Rows) or _apart((_span(buf),), (_span(rows),)))
                 and ((d_gate_up is None and d_down is None)
                      or _apart((_span(d_gate_up), _span(d_down)),
                                (_span(logits), _span(dy), _span(buf), *self._kept_spans(rows), *self._index_spans(out, T)))),
                 "expert_step_backward")
        d_buf, d_weights = self.combine_backward(buf, dy)
        if isinstance(rows, Mx8Rows):
            rows = self.redispatch(rows)
        d_rows, d_gate_up, d_down = self.expert_ffn_backward(d_buf, rows, out.slot_counts, out.slot_offsets, gate_up, down, z, None,
                                                             d_gate_up, d_down, add, grad_dtype)
        if self.cfg.score_func == MOE_ROUTE_DENSE_TP:
            d_weights = None
        dx, d_logits = self.dispatch_backward(logits, d_rows, d_weights)
        return dx, d_logits, d_gate_up, d_down

    # -- expert parallelism over several GPUs -------------------------------
    def ep_attach(self, world: int, rank: int, recv_buf_ptrs, recv_rows: int) -> None:
        st = moe_ep_attach(self._ctx, world, rank, recv_buf_ptrs, recv_rows, self._stream())
        if st != MOE_OK:
            raise MoeError(st, "moe_ep_attach")

    def ep_route(self, logits: torch.Tensor, out: DispatchBuffers) -> DispatchBuffers:
        T = logits.shape[0]
        assert logits.dtype == torch.float32 and logits.is_contiguous() and logits.shape[1] == self.cfg.num_experts
        st = moe_ep_route(self._ctx, logits.data_ptr(), T, out.as_struct(), self._stream())
        self._keep(out, st)
        if st != MOE_OK:
            raise MoeError(st, "moe_ep_route")
        return out

    def ep_scatter(self, x: torch.Tensor, counts_all: torch.Tensor, recv_slot_offsets: torch.Tensor) -> None:
        T = x.shape[0]
        assert x.dtype == torch.bfloat16 and x.is_contiguous() and x.shape[1] == self.cfg.hidden
        assert counts_all.dtype == torch.int32 and counts_all.is_contiguous()
        assert recv_slot_offsets.dtype == torch.int32 and recv_slot_offsets.is_contiguous()
        st = moe_ep_scatter(self._ctx, x.data_ptr(), T, counts_all.data_ptr(),
                            recv_slot_offsets.data_ptr(), self._stream())
        if st != MOE_OK:
            raise MoeError(st, "moe_ep_scatter")

    def ep_combine(self, T: int, y: torch.Tensor | None = None) -> torch.Tensor:
        if y is None:
            y = torch.empty((T, self.cfg.hidden), dtype=torch.bfloat16, device=self.device)
        st = moe_ep_combine(self._ctx, T, y.data_ptr(), self._stream())
        if st != MOE_OK:
            raise MoeError(st, "moe_ep_combine")
        return y

    def step_host(self, logits_host: torch.Tensor, x_host: torch.Tensor, out: DispatchBuffers,
                  logits_dev: torch.Tensor, x_dev: torch.Tensor, y_dev: torch.Tensor,
                  y_host: torch.Tensor) -> None:
        T = logits_host.shape[0]
        st = moe_step_host(self._ctx, logits_host.data_ptr(), x_host.data_ptr(), T, out.as_struct(),
                           logits_dev.data_ptr(), x_dev.data_ptr(), y_dev.data_ptr(),
                           y_host.data_ptr(), self._stream())
        self._keep(out, st)
        if st != MOE_OK:
            raise MoeError(st, "moe_step_host")

    def step_host_async(self, logits_host: torch.Tensor, x_host: torch.Tensor, out: DispatchBuffers,
                        logits_dev: torch.Tensor, x_dev: torch.Tensor, y_dev: torch.Tensor,
                        y_host: torch.Tensor) -> None:
        """As step_host, but returns once the work is enqueued on the current stream."""
        T = logits_host.shape[0]
        st = moe_step_host_async(self._ctx, logits_host.data_ptr(), x_host.data_ptr(), T, out.as_struct(),
                                 logits_dev.data_ptr(), x_dev.data_ptr(), y_dev.data_ptr(),
                                 y_host.data_ptr(), self._stream())
        self._keep(out, st)
        if st != MOE_OK:
            raise MoeError(st, "moe_step_host_async")

    def set_timing_event(self, event: "torch.cuda.Event | None") -> None:
        """Record `event` between the routing and the scatter kernel of every dispatch."""
        handle = 0
        if event is not None:
            event.record(torch.cuda.current_stream(self.device))   # forces creation of the handle
            handle = event.cuda_event
        st = moe_set_timing_event(self._ctx, handle)
        if st != MOE_OK:
            raise MoeError(st, "moe_set_timing_event")

    def set_tuning(self, option: int, value: int) -> None:
        """Override one launch choice of the context (see moe_tuning_option); -1 = automatic."""
        st = moe_set_tuning(self._ctx, option, value)
        if st != MOE_OK:
            raise MoeError(st, "moe_set_tuning")

    def device_status(self) -> int:
        st, code = moe_get_device_status(self._ctx)
        if st != MOE_OK:
            raise MoeError(st, "moe_get_device_status")
        return code

    def close(self) -> None:
        if self._ctx is not None:
            moe_route_destroy(self._ctx)
            self._ctx = self._latest = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def config_for_workload(wl, max_tokens: int | None = None, hidden: int | None = None,
                        route_scale: float = 1.0) -> moe_config:
    """moe_config for one of ``workloads.WORKLOADS`` (shape bookkeeping only)."""
    return make_config(num_experts=wl.E, top_k=wl.k, hidden=wl.H if hidden is None else hidden,
                       max_tokens=wl.T if max_tokens is None else max_tokens, num_ranks=wl.R,
                       slots_per_rank=wl.S, max_replicas=wl.max_replicas, score_func=wl.score_func,
                       n_group=wl.n_group, topk_group=wl.topk_group, route_scale=route_scale)
