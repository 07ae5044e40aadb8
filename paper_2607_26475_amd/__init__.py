"""Python binding of libckv (critical-KV selection and sparse decode attention
on MI355X).

Argument marshalling only: every function passes raw pointers, sizes and the
current HIP stream to the C ABI declared in ``include/ckv.h`` and raises
``CkvError`` on a non-zero status.  All computation happens in the HIP
kernels of ``libckv.so``; there is no fallback.  torch is used for device
memory, pinned host memory and streams.

The library must have been built first (``python paper_2607_26475_amd/build.py``
or ``__graft_entry__.build()``); importing this package without it raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

__all__ = [
    "CkvError", "Shape", "shape_for", "workspace_bytes", "workspace",
    "score_keys", "select_topk", "gather_kv", "sparse_decode_attn",
    "critical_kv_attn", "critical_kv_attn_noalloc", "NOALLOC_SCRATCH_BYTES", "corrected_attn", "chunk_landmarks", "select_chunks",
    "chunked_kv_attn", "dual_token_attn", "reconstruct_keys", "corrected_attn_lowrank",
    "MAX_RANK", "ABI_VERSION", "profile_begin", "profile_end", "abi_version",
    "Layer", "layer_array", "Pipeline", "status_str", "LIB_PATH",
    "SRC_DEVICE", "SRC_HOST_PINNED", "ENTRY_SELECT_TOPK",
    "ENTRY_SPARSE_DECODE_ATTN", "ENTRY_CRITICAL_KV_ATTN", "ENTRY_CORRECTED_ATTN", "ENTRY_DUAL_TOKEN_ATTN", "ENTRY_DECODE_STEP",
    "EXPORTS", "probe_read_rows", "probe_sink_words", "PROBE_STANDALONE", "PROBE_ROW_HALVES",
    "PROBE_HEAD_HALVES", "set_debug", "set_one_launch_same_step", "ONE_LAUNCH_OFF",
    "ONE_LAUNCH_ROW_HALVES", "ONE_LAUNCH_HEAD_HALVES",
    "Rope", "rope_for", "rope_frequencies", "Rows", "rows_for", "rope_rows",
    "ROPE_HALF", "ROPE_INTERLEAVED", "ROPE_BF16", "ROPE_F32", "ROPE_PLAIN", "ROPE_LINEAR",
    "ROPE_BASE", "ROPE_BANDS", "ROPE_RAMP", "PagedCache", "paged_cache_for", "paged_write",
    "paged_read", "paged_score_keys", "paged_decode_attn", "CACHE_BF16", "CACHE_E4M3",
    "CACHE_E2M1", "ENTRY_PAGED_DECODE_ATTN", "paged_landmarks", "select_blocks",
    "paged_block_attn", "blocks_workspace", "blocks_workspace_bytes",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libckv.so")

SRC_DEVICE, SRC_HOST_PINNED = 0, 1
ENTRY_SELECT_TOPK, ENTRY_SPARSE_DECODE_ATTN, ENTRY_CRITICAL_KV_ATTN = 1, 2, 3
ENTRY_CORRECTED_ATTN, ENTRY_DUAL_TOKEN_ATTN, ENTRY_DECODE_STEP = 4, 5, 6
ENTRY_PAGED_DECODE_ATTN = 7  # workspace_bytes: k is the number of query tokens
PROBE_STANDALONE, PROBE_ROW_HALVES, PROBE_HEAD_HALVES = 0, 1, 2
EXPORTS = ("ckv_abi_version", "ckv_status_str", "ckv_last_error_detail",
           "ckv_workspace_bytes", "ckv_score_keys", "ckv_select_topk",
           "ckv_gather_kv", "ckv_sparse_decode_attn", "ckv_critical_kv_attn",
           "ckv_critical_kv_attn_noalloc",
           "ckv_corrected_attn", "ckv_chunk_landmarks", "ckv_select_chunks",
           "ckv_chunked_kv_attn", "ckv_dual_token_attn", "ckv_reconstruct_keys",
           "ckv_corrected_attn_lowrank",
           "ckv_kernel_name", "ckv_profile_begin", "ckv_profile_begin_sampled",
           "ckv_profile_end", "ckv_profile_end_n",
           "ckv_pipeline_create", "ckv_pipeline_destroy", "ckv_pipeline_set_gather_width",
           "ckv_pipeline_set_checks",
           "ckv_pipeline_prime",
           "ckv_decode_step", "ckv_probe_read_rows", "ckv_probe_sink_words", "ckv_set_debug",
           "ckv_set_one_launch_same_step", "ckv_rope_rows", "ckv_rope_frequencies",
           "ckv_paged_write", "ckv_paged_read", "ckv_paged_score_keys",
           "ckv_paged_decode_attn", "ckv_paged_landmarks", "ckv_select_blocks",
           "ckv_paged_block_attn", "ckv_blocks_workspace_bytes")
KERNEL_COUNT = 28
MAX_RANK = 4096
ABI_VERSION = 9  # CKV_ABI_VERSION of include/ckv.h that this binding marshals for


class CkvError(RuntimeError):
    def __init__(self, fn: str, status: int, detail: str):
        super().__init__(f"{fn}: {status_str(status)} ({status}): {detail}")
        self.status = status


class KernelStats(ctypes.Structure):
    """Mirror of ``ckv_kernel_stats``."""
    _fields_ = [("launches", ctypes.c_int64), ("total_ms", ctypes.c_double),
                ("max_ms", ctypes.c_double)]


class Layer(ctypes.Structure):
    """Mirror of ``ckv_layer``."""
    _fields_ = [(name, ctypes.c_void_p) for name in (
        "q_att", "q_sel", "k_score", "k_src", "v_src", "idx_prev", "n_sel_prev",
        "idx_next", "n_sel_next", "out", "idx_true", "n_true", "hits")] + [
        ("lr_rank", ctypes.c_int32), ("lr_u", ctypes.c_void_p), ("lr_w", ctypes.c_void_p),
        ("chunk", ctypes.c_int32), ("landmarks", ctypes.c_void_p),
        ("k_local", ctypes.c_void_p), ("v_local", ctypes.c_void_p),
        ("out_spec", ctypes.c_void_p)]


class Shape(ctypes.Structure):
    """Mirror of ``ckv_shape``."""
    _fields_ = [("batch", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_ctx", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("key_row_stride", ctypes.c_int64),
                ("kv_row_stride", ctypes.c_int64)]


class Rope(ctypes.Structure):
    """Mirror of ``ckv_rope``."""
    _fields_ = [("inv_freq", ctypes.c_void_p), ("head_dim", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("type", ctypes.c_int32), ("inverse", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class RopeScaling(ctypes.Structure):
    """Mirror of ``ckv_rope_scaling``."""
    _fields_ = [("kind", ctypes.c_int32), ("orig_ctx", ctypes.c_int32),
                ("factor", ctypes.c_double), ("low", ctypes.c_double),
                ("high", ctypes.c_double)]


class Rows(ctypes.Structure):
    """Mirror of ``ckv_rows``."""
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p),
                ("src_token_stride", ctypes.c_int64), ("src_head_stride", ctypes.c_int64),
                ("dst_token_stride", ctypes.c_int64), ("dst_head_stride", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class PagedCache(ctypes.Structure):
    """Mirror of ``ckv_paged_cache``."""
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("k_exps", ctypes.c_void_p), ("v_exps", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("kind", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("table_stride", ctypes.c_int32)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run "
                          "`python paper_2607_26475_amd/build.py` first")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    sp = ctypes.POINTER(Shape)
    sig = {
        "ckv_abi_version": (ctypes.c_int, []),
        "ckv_status_str": (ctypes.c_char_p, [ctypes.c_int]),
        "ckv_last_error_detail": (ctypes.c_char_p, []),
        "ckv_workspace_bytes": (ctypes.c_int, [sp, i32, ctypes.c_int, ctypes.POINTER(sz)]),
        "ckv_score_keys": (ctypes.c_int, [sp, vp, vp, vp, ctypes.c_float, vp, vp]),
        "ckv_select_topk": (ctypes.c_int, [sp, vp, vp, i32, vp, vp, vp, sz, vp]),
        "ckv_gather_kv": (ctypes.c_int, [sp, vp, vp, ctypes.c_int, vp, vp, i32, vp, vp, vp]),
        "ckv_sparse_decode_attn": (ctypes.c_int, [sp, vp, vp, vp, vp, i32, ctypes.c_float,
                                                  vp, vp, sz, vp]),
        "ckv_critical_kv_attn": (ctypes.c_int, [sp, vp, vp, vp, vp, i32, ctypes.c_float,
                                                vp, vp, ctypes.c_int, vp, vp, vp, vp, vp,
                                                vp, vp, vp, sz, vp]),
        "ckv_critical_kv_attn_noalloc": (ctypes.c_int, [sp, vp, vp, vp, vp, i32,
                                                        ctypes.c_float, vp, vp, ctypes.c_int,
                                                        vp, vp, vp, vp, vp, vp, vp, vp]),
        "ckv_corrected_attn": (ctypes.c_int, [sp, vp, vp, vp, vp, i32, ctypes.c_float,
                                              vp, vp, ctypes.c_int, vp, vp, vp, vp, vp, vp,
                                              vp, vp, vp, vp, vp, sz, vp]),
        "ckv_chunk_landmarks": (ctypes.c_int, [sp, i32, vp, vp, vp, vp]),
        "ckv_select_chunks": (ctypes.c_int, [sp, i32, vp, vp, vp, i32, ctypes.c_float, vp, vp,
                                             vp, vp, vp, sz, vp]),
        "ckv_chunked_kv_attn": (ctypes.c_int, [sp, i32, vp, vp, vp, vp, i32, ctypes.c_float,
                                               vp, vp, ctypes.c_int, vp, vp, vp, vp, vp, vp,
                                               sz, vp]),
        "ckv_dual_token_attn": (ctypes.c_int, [sp, vp, vp, vp, vp, vp, vp, vp, i32,
                                               ctypes.c_float, vp, vp, vp, sz, vp]),
        "ckv_reconstruct_keys": (ctypes.c_int, [sp, i32, vp, vp, vp, vp, i32, vp, vp]),
        "ckv_corrected_attn_lowrank": (ctypes.c_int, [sp, vp, vp, vp, vp, i32, ctypes.c_float,
                                                      vp, vp, ctypes.c_int, i32, vp, vp, vp,
                                                      vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                                      vp, sz, vp]),
        "ckv_kernel_name": (ctypes.c_char_p, [ctypes.c_int]),
        "ckv_profile_begin": (ctypes.c_int, [ctypes.c_uint32]),
        "ckv_profile_begin_sampled": (ctypes.c_int, [ctypes.c_uint32, ctypes.c_uint32]),
        "ckv_profile_end": (ctypes.c_int, [ctypes.POINTER(KernelStats)]),
        "ckv_profile_end_n": (ctypes.c_int, [ctypes.POINTER(KernelStats), ctypes.c_int]),
        "ckv_rope_rows": (ctypes.c_int, [ctypes.POINTER(Rope), i32, vp, ctypes.POINTER(Rows),
                                         ctypes.POINTER(Rows), vp]),
        "ckv_rope_frequencies": (ctypes.c_int, [i32, ctypes.c_double,
                                                ctypes.POINTER(RopeScaling), vp,
                                                ctypes.POINTER(ctypes.c_float)]),
        "ckv_paged_write": (ctypes.c_int, [sp, ctypes.POINTER(PagedCache), i32, vp, vp, vp, vp,
                                           ctypes.c_int64, ctypes.POINTER(Rope),
                                           ctypes.POINTER(Rows), vp]),
        "ckv_paged_read": (ctypes.c_int, [sp, ctypes.POINTER(PagedCache), vp, vp, vp, i32, vp,
                                          vp, vp]),
        "ckv_paged_score_keys": (ctypes.c_int, [sp, ctypes.POINTER(PagedCache), vp, vp,
                                                ctypes.c_float, vp, vp]),
        "ckv_paged_decode_attn": (ctypes.c_int, [sp, ctypes.POINTER(PagedCache), i32, vp, vp,
                                                 ctypes.c_float, vp, vp, vp, sz, vp]),
        "ckv_paged_landmarks": (ctypes.c_int, [sp, ctypes.POINTER(PagedCache), i32, vp, vp, vp,
                                               vp]),
        "ckv_select_blocks": (ctypes.c_int, [sp, ctypes.POINTER(PagedCache), i32, i32, i32, vp,
                                             vp, vp, vp, vp, vp, sz, vp]),
        "ckv_paged_block_attn": (ctypes.c_int, [sp, ctypes.POINTER(PagedCache), i32, i32, i32,
                                                vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, sz,
                                                vp]),
        "ckv_blocks_workspace_bytes": (ctypes.c_int, [sp, i32, i32, i32, ctypes.POINTER(sz)]),
        "ckv_probe_read_rows": (ctypes.c_int, [sp, vp, vp, vp, i32, ctypes.c_int, vp, sz, vp]),
        "ckv_probe_sink_words": (sz, [sp, i32, ctypes.c_int]),
        "ckv_set_debug": (ctypes.c_int, [ctypes.c_int]),
        "ckv_set_one_launch_same_step": (ctypes.c_int, [ctypes.c_int]),
        "ckv_pipeline_create": (ctypes.c_int, [ctypes.POINTER(vp)]),
        "ckv_pipeline_destroy": (ctypes.c_int, [vp]),
        "ckv_pipeline_set_gather_width": (ctypes.c_int, [vp, ctypes.c_int]),
        "ckv_pipeline_set_checks": (ctypes.c_int, [vp, ctypes.c_uint]),
        "ckv_pipeline_prime": (ctypes.c_int, [vp, sp, i32, ctypes.POINTER(Layer), ctypes.c_int,
                                              ctypes.c_int, ctypes.POINTER(vp),
                                              ctypes.POINTER(vp), vp]),
        "ckv_decode_step": (ctypes.c_int, [vp, sp, ctypes.c_int, ctypes.POINTER(Layer), vp,
                                           i32, ctypes.c_float, ctypes.c_int,
                                           ctypes.POINTER(vp), ctypes.POINTER(vp), vp, sz, vp,
                                           vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name, None)
        if f is None:  # entries are added under one version
            raise ImportError(f"{LIB_PATH} has no {name}, the binding expects it; rebuild it")
        f.restype = res
        f.argtypes = args
    return lib


_lib = _load()
if _lib.ckv_abi_version() != ABI_VERSION:
    raise ImportError(f"{LIB_PATH} has ABI {_lib.ckv_abi_version()}, the binding expects "
                      f"{ABI_VERSION}; rebuild it")


def abi_version() -> int:
    return _lib.ckv_abi_version()


def status_str(status: int) -> str:
    return _lib.ckv_status_str(status).decode()


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise CkvError(fn, status, _lib.ckv_last_error_detail().decode())


def shape_for(batch: int, num_q_heads: int, num_kv_heads: int, max_ctx: int,
              head_dim: int = 128, key_row_stride: Optional[int] = None,
              kv_row_stride: Optional[int] = None) -> Shape:
    return Shape(batch, num_q_heads, num_kv_heads, head_dim, max_ctx, 0,
                 head_dim if key_row_stride is None else key_row_stride,
                 head_dim if kv_row_stride is None else kv_row_stride)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def workspace_bytes(shape: Shape, k: int, entry: int) -> int:
    n = ctypes.c_size_t(0)
    _check("ckv_workspace_bytes",
           _lib.ckv_workspace_bytes(ctypes.byref(shape), k, entry, ctypes.byref(n)))
    return n.value


def workspace(shape: Shape, k: int, entry: int, device="cuda") -> torch.Tensor:
    """A device byte tensor large enough for `entry` (torch allocations are
    256-byte aligned)."""
    return torch.empty(max(workspace_bytes(shape, k, entry), 1), dtype=torch.uint8,
                       device=device)


def score_keys(shape: Shape, q, k_score, ctx_lens, scale: float, scores,
               stream=None) -> None:
    _check("ckv_score_keys", _lib.ckv_score_keys(
        ctypes.byref(shape), _ptr(q), _ptr(k_score), _ptr(ctx_lens), scale,
        _ptr(scores), _stream(stream)))


def select_topk(shape: Shape, scores, ctx_lens, k: int, idx, n_sel, ws,
                stream=None) -> None:
    _check("ckv_select_topk", _lib.ckv_select_topk(
        ctypes.byref(shape), _ptr(scores), _ptr(ctx_lens), k, _ptr(idx), _ptr(n_sel),
        _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)))


def gather_kv(shape: Shape, k_src, v_src, src_kind: int, idx, n_sel, k: int,
              k_dst, v_dst, stream=None) -> None:
    _check("ckv_gather_kv", _lib.ckv_gather_kv(
        ctypes.byref(shape), _ptr(k_src), _ptr(v_src), src_kind, _ptr(idx), _ptr(n_sel),
        k, _ptr(k_dst), _ptr(v_dst), _stream(stream)))


def sparse_decode_attn(shape: Shape, q_att, k_buf, v_buf, n_sel, k: int,
                       scale: float, out, ws, stream=None) -> None:
    _check("ckv_sparse_decode_attn", _lib.ckv_sparse_decode_attn(
        ctypes.byref(shape), _ptr(q_att), _ptr(k_buf), _ptr(v_buf), _ptr(n_sel), k, scale,
        _ptr(out), _ptr(ws), ws.numel() if ws is not None else 0, _stream(stream)))


def critical_kv_attn(shape: Shape, q_att, q_sel, k_score, ctx_lens, k: int,
                     scale: float, k_src, v_src, src_kind: int, k_buf, v_buf,
                     n_sel_in, idx_out, n_sel_out, out, ws, stream=None,
                     idx_in=None) -> None:
    """Same-step (k_buf and idx_in None), pipelined over an assembled buffer
    (k_buf), or pipelined over the rows idx_in read in place."""
    _check("ckv_critical_kv_attn", _lib.ckv_critical_kv_attn(
        ctypes.byref(shape), _ptr(q_att), _ptr(q_sel), _ptr(k_score), _ptr(ctx_lens), k,
        scale, _ptr(k_src), _ptr(v_src), src_kind, _ptr(idx_in), _ptr(k_buf), _ptr(v_buf),
        _ptr(n_sel_in), _ptr(idx_out), _ptr(n_sel_out), _ptr(out), _ptr(ws),
        ws.numel() if ws is not None else 0, _stream(stream)))


NOALLOC_SCRATCH_BYTES = 64 << 20  # CKV_NOALLOC_SCRATCH_BYTES


def critical_kv_attn_noalloc(shape: Shape, q_att, q_sel, k_score, ctx_lens, k: int,
                             scale: float, k_src, v_src, src_kind: int, k_buf, v_buf,
                             n_sel_in, idx_out, n_sel_out, out, stream=None,
                             idx_in=None) -> None:
    """critical_kv_attn with the library's fixed per-device scratch instead of
    a workspace (the call allocates nothing)."""
    _check("ckv_critical_kv_attn_noalloc", _lib.ckv_critical_kv_attn_noalloc(
        ctypes.byref(shape), _ptr(q_att), _ptr(q_sel), _ptr(k_score), _ptr(ctx_lens), k,
        scale, _ptr(k_src), _ptr(v_src), src_kind, _ptr(idx_in), _ptr(k_buf), _ptr(v_buf),
        _ptr(n_sel_in), _ptr(idx_out), _ptr(n_sel_out), _ptr(out), _stream(stream)))


def corrected_attn(shape: Shape, q_att, q_sel, k_score, ctx_lens, k: int, scale: float,
                   k_src, v_src, src_kind: int, idx_pred, n_pred, k_buf, v_buf, idx_true,
                   n_true, hits, idx_next, n_next, out, ws, stream=None) -> None:
    _check("ckv_corrected_attn", _lib.ckv_corrected_attn(
        ctypes.byref(shape), _ptr(q_att), _ptr(q_sel), _ptr(k_score), _ptr(ctx_lens), k,
        scale, _ptr(k_src), _ptr(v_src), src_kind, _ptr(idx_pred), _ptr(n_pred),
        _ptr(k_buf), _ptr(v_buf), _ptr(idx_true), _ptr(n_true), _ptr(hits), _ptr(idx_next),
        _ptr(n_next), _ptr(out), _ptr(ws), ws.numel() if ws is not None else 0,
        _stream(stream)))


def corrected_attn_lowrank(shape: Shape, q_att, q_sel, k_score, ctx_lens, k: int,
                           scale: float, k_src, v_src, src_kind: int, rank: int, u_fac, w_fac,
                           idx_pred, n_pred, k_buf, v_buf, idx_true, n_true, hits, idx_next,
                           n_next, out, ws, stream=None) -> None:
    _check("ckv_corrected_attn_lowrank", _lib.ckv_corrected_attn_lowrank(
        ctypes.byref(shape), _ptr(q_att), _ptr(q_sel), _ptr(k_score), _ptr(ctx_lens), k,
        scale, _ptr(k_src), _ptr(v_src), src_kind, rank, _ptr(u_fac), _ptr(w_fac),
        _ptr(idx_pred), _ptr(n_pred), _ptr(k_buf), _ptr(v_buf), _ptr(idx_true), _ptr(n_true),
        _ptr(hits), _ptr(idx_next), _ptr(n_next), _ptr(out), _ptr(ws),
        ws.numel() if ws is not None else 0, _stream(stream)))


def reconstruct_keys(shape: Shape, rank: int, u_fac, w_fac, idx, n_sel, k: int, k_dst,
                     stream=None) -> None:
    _check("ckv_reconstruct_keys", _lib.ckv_reconstruct_keys(
        ctypes.byref(shape), rank, _ptr(u_fac), _ptr(w_fac), _ptr(idx), _ptr(n_sel), k,
        _ptr(k_dst), _stream(stream)))


def dual_token_attn(shape: Shape, q_cur, q_spec, k_buf, v_buf, n_sel, k_local, v_local,
                    k: int, scale: float, out_cur, out_spec, ws, stream=None) -> None:
    _check("ckv_dual_token_attn", _lib.ckv_dual_token_attn(
        ctypes.byref(shape), _ptr(q_cur), _ptr(q_spec), _ptr(k_buf), _ptr(v_buf), _ptr(n_sel),
        _ptr(k_local), _ptr(v_local), k, scale, _ptr(out_cur), _ptr(out_spec), _ptr(ws),
        ws.numel() if ws is not None else 0, _stream(stream)))


def chunk_landmarks(shape: Shape, chunk: int, keys, ctx_lens, landmarks,
                    stream=None) -> None:
    _check("ckv_chunk_landmarks", _lib.ckv_chunk_landmarks(
        ctypes.byref(shape), chunk, _ptr(keys), _ptr(ctx_lens), _ptr(landmarks),
        _stream(stream)))


def select_chunks(shape: Shape, chunk: int, q_sel, landmarks, ctx_lens, k: int,
                  scale: float, chunk_idx, n_chunks, rows, n_rows, ws, stream=None) -> None:
    _check("ckv_select_chunks", _lib.ckv_select_chunks(
        ctypes.byref(shape), chunk, _ptr(q_sel), _ptr(landmarks), _ptr(ctx_lens), k, scale,
        _ptr(chunk_idx), _ptr(n_chunks), _ptr(rows), _ptr(n_rows), _ptr(ws),
        ws.numel() if ws is not None else 0, _stream(stream)))


def chunked_kv_attn(shape: Shape, chunk: int, q_att, q_sel, landmarks, ctx_lens, k: int,
                    scale: float, k_src, v_src, src_kind: int, chunk_idx, n_chunks, rows,
                    n_rows, out, ws, stream=None) -> None:
    _check("ckv_chunked_kv_attn", _lib.ckv_chunked_kv_attn(
        ctypes.byref(shape), chunk, _ptr(q_att), _ptr(q_sel), _ptr(landmarks),
        _ptr(ctx_lens), k, scale, _ptr(k_src), _ptr(v_src), src_kind, _ptr(chunk_idx),
        _ptr(n_chunks), _ptr(rows), _ptr(n_rows), _ptr(out), _ptr(ws),
        ws.numel() if ws is not None else 0, _stream(stream)))


# ---- rotary positions and the paged cache -------------------------------------------
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_BF16, ROPE_F32 = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BANDS, ROPE_RAMP = 0, 1, 2, 3, 4
CACHE_BF16, CACHE_E4M3, CACHE_E2M1 = 0, 1, 2


# The current stream's handle without a Stream object around it (2.6 us of an
# 8 us call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(fn, dev: int, stream, *args) -> None:
    """Calls an entry with its last argument, the stream (None: the current one
    of device dev), with dev current."""
    if dev < 0:
        raise ValueError("the tensors have to be on a GPU")
    handle = _raw_stream(dev) if stream is None else _stream(stream)
    if dev == _current_device():
        status = fn(*args, handle)
    else:
        with torch.cuda.device(dev):
            status = fn(*args, handle)
    if status:
        _check(fn.__name__, status)


def _dense(name: str, t: torch.Tensor, dtype, n: int, dev: int) -> None:
    """What kernels read and write has to be there: dense, of its type, long
    enough, on the device of the call."""
    if t.dtype != dtype or not t.is_contiguous() or t.numel() < n or t.get_device() != dev:
        raise ValueError(f"{name}: a dense {dtype} tensor of {n} elements on device {dev}, not "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")


def rope_frequencies(rot_dim: int, base: float, kind: int = ROPE_PLAIN, factor: float = 1.0,
                     orig_ctx: int = 0, low: float = 0.0, high: float = 0.0):
    """``ckv_rope_frequencies``: (float64 CPU tensor of rot_dim / 2 radians per
    position, the factor for the rotated elements)."""
    out = torch.empty(max(rot_dim // 2, 1), dtype=torch.float64)
    s = RopeScaling(kind, orig_ctx, factor, low, high)
    scale = ctypes.c_float(1.0)
    _check("ckv_rope_frequencies", _lib.ckv_rope_frequencies(
        rot_dim, base, ctypes.byref(s), out.data_ptr(), ctypes.byref(scale)))
    return out, scale.value


def rope_for(inv_freq: torch.Tensor, head_dim: int = 128, rot_dim: Optional[int] = None,
             layout: int = ROPE_HALF, dtype: int = ROPE_BF16, inverse: bool = False,
             scale: float = 1.0) -> Rope:
    """The rotation handle over a device tensor of float64 frequencies (kept
    alive by the handle)."""
    rot = 2 * inv_freq.numel() if rot_dim is None else rot_dim
    if inv_freq.dtype != torch.float64 or not inv_freq.is_contiguous() or \
            2 * inv_freq.numel() < rot:
        raise ValueError(f"inv_freq: {rot // 2} dense float64 frequencies")
    r = Rope(inv_freq.data_ptr(), head_dim, rot, layout, dtype, int(inverse), scale)
    r.keep, r.dev = inv_freq, inv_freq.get_device()
    return r


def rows_for(src: torch.Tensor, dst: Optional[torch.Tensor] = None) -> Rows:
    """Head rows [tokens][heads][d] of one tensor (any token and head strides)
    into those of another of the same shape, or in place."""
    dst = src if dst is None else dst
    if src.dim() != 3 or src.shape != dst.shape or src.dtype != dst.dtype or \
            src.device != dst.device or \
            src.stride(2) != 1 or dst.stride(2) != 1:
        raise ValueError(f"rows: [tokens][heads][d] with adjacent elements, the same twice, not "
                         f"{tuple(src.shape)} and {tuple(dst.shape)}")
    r = Rows(src.data_ptr(), dst.data_ptr(), src.stride(0), src.stride(1), dst.stride(0),
             dst.stride(1), src.shape[1], 0)
    r.keep = (src, dst)
    r.holds = (src.shape[0], src.shape[2], _ROPE_TYPES.get(src.dtype), src.get_device())
    return r


_ROPE_TYPES = {torch.bfloat16: ROPE_BF16, torch.float32: ROPE_F32}


def _rows_ok(name: str, rows: Rows, rope: Rope, n: int, dev: int) -> None:
    holds = getattr(rows, "holds", None)  # None: filled in by hand
    if holds is not None and (holds[0] < n or holds[1] != rope.head_dim or
                              holds[2] != rope.type or holds[3] != dev):
        t = rows.keep[0]
        raise ValueError(f"{name}: {n} tokens of rows of {rope.head_dim} elements of the rope's "
                         f"type on device {dev}, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _rope_ok(rope: Rope, dev: int) -> None:
    if getattr(rope, "dev", dev) != dev:
        raise ValueError(f"the rope's frequencies are on {rope.keep.device}, not on device {dev}")


def rope_rows(rope: Rope, positions: torch.Tensor, q: Rows, k: Optional[Rows] = None,
              stream=None) -> None:
    """Rotates the head rows of q (and k) by their tokens' positions."""
    n, dev = positions.numel(), positions.get_device()
    _dense("positions", positions, torch.int32, n, dev)
    _rope_ok(rope, dev)
    _rows_ok("q", q, rope, n, dev)
    if k is not None:
        _rows_ok("k", k, rope, n, dev)
    _call(_lib.ckv_rope_rows, dev, stream, rope, n, positions.data_ptr(), q, k)


_E2M1 = getattr(torch, "float4_e2m1fn_x2", torch.uint8)  # bytes of two codes


def paged_cache_for(k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor,
                    k_exps: Optional[torch.Tensor] = None,
                    v_exps: Optional[torch.Tensor] = None) -> PagedCache:
    """The handle of a paged cache: pages as [pages][Hkv][page_size][d] views
    of one pair of strides (bf16, uint8 / float8_e4m3fn codes with uint8
    exponents [pages][Hkv][page_size], or uint8 / float4_e2m1fn_x2 bytes of two
    e2m1 codes, 64 a row, with uint8 exponents [pages][Hkv][page_size][4]),
    page_table [B][pages per request].  The handle keeps the tensors alive."""
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or \
            k_pages.stride() != v_pages.stride() or k_pages.dtype != v_pages.dtype or \
            k_pages.stride(3) != 1 or k_pages.shape[3] not in (64, 128):
        raise ValueError("k_pages, v_pages: [pages][Hkv][page_size][128] (64 bytes of two codes), "
                         "alike, rows dense")
    four = k_pages.shape[3] == 64
    kind = CACHE_E2M1 if four else CACHE_BF16 if k_pages.element_size() == 2 else CACHE_E4M3
    if k_pages.dtype not in ((torch.uint8, _E2M1) if four else
                             (torch.bfloat16, torch.uint8, torch.float8_e4m3fn)):
        raise ValueError(f"pages of {k_pages.dtype} {tuple(k_pages.shape)}")
    want = (*k_pages.shape[:3], 4) if four else k_pages.shape[:3]
    for e in (k_exps, v_exps):
        if (e is not None) != (kind != CACHE_BF16) or (e is not None and (
                e.dtype != torch.uint8 or e.shape != want or not e.is_contiguous())):
            raise ValueError("k_exps, v_exps: dense uint8 [pages][Hkv][page_size] of e4m3 pages, "
                             "[pages][Hkv][page_size][4] of e2m1 pages, none of bf16 pages")
    if page_table.dim() != 2 or page_table.dtype != torch.int32 or page_table.stride(1) != 1:
        raise ValueError("page_table: int32 [B][pages]")
    c = PagedCache(k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_exps), _ptr(v_exps),
                   page_table.data_ptr(), *((2 if four else 1) * _stride(k_pages, i) for i in range(3)), kind,
                   k_pages.shape[2], k_pages.shape[0],
                   page_table.shape[1] if page_table.shape[0] == 1 else page_table.stride(0))
    c.keep = (k_pages, v_pages, page_table, k_exps, v_exps)
    tensors = [x for x in c.keep if x is not None]
    if any(x.device != k_pages.device for x in tensors):
        raise ValueError("a cache's tensors on different devices")
    c.holds = (k_pages.shape[1], page_table.shape[0], page_table.shape[1] * k_pages.shape[2],
               k_pages.get_device())
    return c


def _stride(t: torch.Tensor, i: int) -> int:
    """A dimension's stride; of one that holds a single entry any will do."""
    return t.stride(i) if t.shape[i] > 1 else max(t.stride(i), t.shape[3])


def _cache_ok(shape: Shape, cache: PagedCache, dev: int) -> None:
    holds = getattr(cache, "holds", None)  # None: filled in by hand
    if holds is not None and (holds[0] != shape.num_kv_heads or holds[1] < shape.batch or
                              holds[2] < shape.max_ctx or holds[3] != dev):
        raise ValueError(f"a cache of {holds[0]} heads, {holds[1]} requests and {holds[2]} "
                         f"positions on device {holds[3]} for a shape of {shape.num_kv_heads}, "
                         f"{shape.batch} and {shape.max_ctx} on {dev}")


def paged_write(shape: Shape, cache: PagedCache, requests, positions: torch.Tensor,
                k: torch.Tensor, v: torch.Tensor, rope: Optional[Rope] = None,
                q: Optional[Rows] = None, stream=None) -> None:
    """Writes k, v [tokens][Hkv][128] into their pages (requests None: token t
    is request t's); with rope, keys (and the rows of q) are rotated."""
    n, dev = positions.numel(), positions.get_device()
    _cache_ok(shape, cache, dev)
    _dense("positions", positions, torch.int32, n, dev)
    if requests is not None:
        _dense("requests", requests, torch.int32, n, dev)
    heads = shape.num_kv_heads
    want, ks, vs = (n, heads, 128), k.stride(), v.stride()
    # (of a dimension that holds a single entry any stride will do)
    if k.shape != want or v.shape != want or ks[2] != 1 or vs[2] != 1 or \
            (heads > 1 and (ks[1] != 128 or vs[1] != 128)) or \
            (n > 1 and ks[0] != vs[0]) or k.dtype != torch.bfloat16 or \
            v.dtype != torch.bfloat16 or k.get_device() != dev or v.get_device() != dev:
        raise ValueError(f"k, v: bf16 {want} with dense heads and one token stride on device "
                         f"{dev}, not {k.dtype} {tuple(k.shape)} {ks} and {v.dtype} "
                         f"{tuple(v.shape)} {vs} on {k.device}")
    if rope is not None:
        _rope_ok(rope, dev)
        if q is not None:
            _rows_ok("q", q, rope, n, dev)
    stride = ks[0] if n > 1 else 128 * heads
    _call(_lib.ckv_paged_write, dev, stream, shape, cache, n, _ptr(requests),
          positions.data_ptr(), k.data_ptr(), v.data_ptr(), stride, rope, q)


def paged_read(shape: Shape, cache: PagedCache, ctx_lens: torch.Tensor, idx, n_sel, k: int,
               k_dst: torch.Tensor, v_dst: torch.Tensor, stream=None) -> None:
    """Rows idx of the pages (idx None: positions 0 .. k - 1) into k_dst, v_dst
    [B][Hkv][k][128] bf16."""
    dev, units = ctx_lens.get_device(), shape.batch * shape.num_kv_heads
    _cache_ok(shape, cache, dev)
    _dense("ctx_lens", ctx_lens, torch.int32, shape.batch, dev)
    if idx is not None:
        _dense("idx", idx, torch.int32, units * k, dev)
    if n_sel is not None:
        _dense("n_sel", n_sel, torch.int32, units, dev)
    _dense("k_dst", k_dst, torch.bfloat16, units * k * 128, dev)
    _dense("v_dst", v_dst, torch.bfloat16, units * k * 128, dev)
    _call(_lib.ckv_paged_read, dev, stream, shape, cache, ctx_lens.data_ptr(), _ptr(idx),
          _ptr(n_sel), k, k_dst.data_ptr(), v_dst.data_ptr())


def paged_score_keys(shape: Shape, cache: PagedCache, q: torch.Tensor, ctx_lens: torch.Tensor,
                     scale: float, scores: torch.Tensor, stream=None) -> None:
    dev = ctx_lens.get_device()
    _cache_ok(shape, cache, dev)
    _dense("ctx_lens", ctx_lens, torch.int32, shape.batch, dev)
    _dense("q", q, torch.bfloat16, shape.batch * shape.num_q_heads * 128, dev)
    _dense("scores", scores, torch.float32, shape.batch * shape.num_kv_heads * shape.max_ctx, dev)
    _call(_lib.ckv_paged_score_keys, dev, stream, shape, cache, q.data_ptr(),
          ctx_lens.data_ptr(), scale, scores.data_ptr())


def paged_decode_attn(shape: Shape, cache: PagedCache, num_tokens: int, q: torch.Tensor,
                      ctx_lens: torch.Tensor, scale: float, out: torch.Tensor, lse, ws,
                      stream=None) -> None:
    """Attention of the last num_tokens tokens (q [B][T][Hq][128]) over the
    paged cache into out (fp32, like q) and, unless None, lse [B][T][Hq]."""
    dev, rows = ctx_lens.get_device(), shape.batch * num_tokens * shape.num_q_heads
    _cache_ok(shape, cache, dev)
    _dense("ctx_lens", ctx_lens, torch.int32, shape.batch, dev)
    _dense("q", q, torch.bfloat16, rows * 128, dev)
    _dense("out", out, torch.float32, rows * 128, dev)
    if lse is not None:
        _dense("lse", lse, torch.float32, rows, dev)
    if ws is not None:
        _dense("ws", ws, torch.uint8, 0, dev)
    _call(_lib.ckv_paged_decode_attn, dev, stream, shape, cache, num_tokens, q.data_ptr(),
          ctx_lens.data_ptr(), scale, out.data_ptr(), _ptr(lse), _ptr(ws),
          ws.numel() if ws is not None else 0)


# ---- attention over selected blocks -----------------------------------------------------
def blocks_workspace_bytes(shape: Shape, block: int, k: int, num_tokens: int) -> int:
    out = ctypes.c_size_t(0)
    _check("ckv_blocks_workspace_bytes", _lib.ckv_blocks_workspace_bytes(
        ctypes.byref(shape), block, k, num_tokens, ctypes.byref(out)))
    return int(out.value)


def blocks_workspace(shape: Shape, block: int, k: int, num_tokens: int,
                     device="cuda") -> torch.Tensor:
    """A workspace for ``select_blocks`` and ``paged_block_attn`` of these sizes."""
    return torch.empty(max(256, blocks_workspace_bytes(shape, block, k, num_tokens)),
                       dtype=torch.uint8, device=device)


def paged_landmarks(shape: Shape, cache: PagedCache, block: int, ctx_lens: torch.Tensor,
                    landmarks: torch.Tensor, first: Optional[torch.Tensor] = None,
                    stream=None) -> None:
    """Mean keys of the cache's blocks into landmarks [B][Hkv][ceil(max_ctx /
    block)][128] bf16, from position first[b]'s block on (None: all)."""
    dev = ctx_lens.get_device()
    _cache_ok(shape, cache, dev)
    _dense("ctx_lens", ctx_lens, torch.int32, shape.batch, dev)
    if first is not None:
        _dense("first", first, torch.int32, shape.batch, dev)
    _dense("landmarks", landmarks, torch.bfloat16, _marks(shape, block), dev)
    _call(_lib.ckv_paged_landmarks, dev, stream, shape, cache, block, ctx_lens.data_ptr(),
          _ptr(first), landmarks.data_ptr())


def _marks(shape: Shape, block: int) -> int:
    return shape.batch * shape.num_kv_heads * -(-shape.max_ctx // max(block, 1)) * 128


def _tokens_ok(shape: Shape, cache: PagedCache, requests, positions: torch.Tensor,
               q: torch.Tensor) -> Tuple[int, int]:
    n, dev = positions.numel(), positions.get_device()
    _cache_ok(shape, cache, dev)
    _dense("positions", positions, torch.int32, n, dev)
    if requests is not None:
        _dense("requests", requests, torch.int32, n, dev)
    _dense("q", q, torch.bfloat16, n * shape.num_q_heads * 128, dev)
    return n, dev


def select_blocks(shape: Shape, cache: PagedCache, block: int, k: int, requests,
                  positions: torch.Tensor, q: torch.Tensor, landmarks: torch.Tensor,
                  idx: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """Each query token's blocks for each KV head into idx [tokens][Hkv][k]: its
    own and the k - 1 best earlier ones by their landmarks (requests None: token t
    is request t's; q [tokens][Hq][128])."""
    n, dev = _tokens_ok(shape, cache, requests, positions, q)
    _dense("landmarks", landmarks, torch.bfloat16, _marks(shape, block), dev)
    _dense("idx", idx, torch.int32, n * shape.num_kv_heads * k, dev)
    _dense("ws", ws, torch.uint8, 0, dev)
    _call(_lib.ckv_select_blocks, dev, stream, shape, cache, block, k, n, _ptr(requests),
          positions.data_ptr(), q.data_ptr(), landmarks.data_ptr(), idx.data_ptr(),
          ws.data_ptr(), ws.numel())


def paged_block_attn(shape: Shape, cache: PagedCache, block: int, k: int, requests,
                     positions: torch.Tensor, q: torch.Tensor, idx: torch.Tensor, scale: float,
                     out: torch.Tensor, lse: Optional[torch.Tensor], ws: torch.Tensor,
                     stream=None) -> None:
    """Attention of each query token over the blocks idx [tokens][Hkv][k] up to
    its own position, into out [tokens][Hq][128] fp32 and, unless None, lse."""
    n, dev = _tokens_ok(shape, cache, requests, positions, q)
    _dense("idx", idx, torch.int32, n * shape.num_kv_heads * k, dev)
    _dense("out", out, torch.float32, n * shape.num_q_heads * 128, dev)
    if lse is not None:
        _dense("lse", lse, torch.float32, n * shape.num_q_heads, dev)
    _dense("ws", ws, torch.uint8, 0, dev)
    _call(_lib.ckv_paged_block_attn, dev, stream, shape, cache, block, k, n, _ptr(requests),
          positions.data_ptr(), q.data_ptr(), idx.data_ptr(), scale, out.data_ptr(), _ptr(lse),
          ws.data_ptr(), ws.numel())


KERNEL_IDS = {"zero": 0, "score": 1, "hist": 2, "filter": 3, "finish": 4, "attn": 5,
              "combine": 6, "dual": 7, "gather": 8, "miss": 9, "landmarks": 10,
              "expand": 11, "reconstruct": 12, "select_attn": 13, "probe": 14,
              "critical": 15, "rope": 16, "paged_write": 17, "paged_read": 18,
              "paged_score": 19, "paged_attn": 20, "paged_merge": 21, "block_marks": 22,
              "block_score": 23, "block_select": 24, "block_attn": 25, "block_merge": 26,
              "block_many": 27}


def profile_begin(kernels=None, every: int = 1) -> None:
    """Start stamping library kernels with dispatch start/end events: all of
    them, or only the named kernel classes; with every > 1 only launches 0,
    every, 2*every, ... of each class."""
    mask = (1 << KERNEL_COUNT) - 1
    if kernels is not None:
        mask = 0
        for name in kernels:
            mask |= 1 << KERNEL_IDS[name]
    _check("ckv_profile_begin_sampled", _lib.ckv_profile_begin_sampled(mask, every))


def profile_end() -> dict:
    """Stop recording; {kernel name: (launches, total_ms, max_ms)} for every
    kernel class that ran (waits for the recorded kernels)."""
    arr = (KernelStats * KERNEL_COUNT)()
    _check("ckv_profile_end_n", _lib.ckv_profile_end_n(arr, KERNEL_COUNT))
    return {_lib.ckv_kernel_name(i).decode(): (arr[i].launches, arr[i].total_ms, arr[i].max_ms)
            for i in range(KERNEL_COUNT) if arr[i].launches}


def set_debug(on: bool) -> None:
    """Debug mode (process-wide): entries check their device-side inputs
    (context lengths, input counts and index sets) on the device and every
    launch synchronises; a violation raises CkvError (CKV_EINVAL)."""
    _check("ckv_set_debug", _lib.ckv_set_debug(1 if on else 0))


ONE_LAUNCH_OFF, ONE_LAUNCH_ROW_HALVES, ONE_LAUNCH_HEAD_HALVES = 0, 1, 2


def set_one_launch_same_step(on) -> None:
    """Whether same-step calls run as one launch where that form applies
    (process-wide).  True / ONE_LAUNCH_ROW_HALVES (the default): one launch
    whose two workgroups per unit attend over half the rows each and merge in
    the launch.  False / ONE_LAUNCH_OFF: the scoring launch, then the
    selection and attention launch, attending the same way (the same bits).
    ONE_LAUNCH_HEAD_HALVES: two workgroups per unit attending over the whole
    set with half the heads each, in one launch where that applies; the same
    index sets, outputs within fp32 rounding of the other forms."""
    _check("ckv_set_one_launch_same_step", _lib.ckv_set_one_launch_same_step(int(on)))


def probe_sink_words(shape: Shape, k: int, mode: int) -> int:
    """uint32 words of sink that probe_read_rows needs (0: shape, k or mode
    invalid)."""
    return int(_lib.ckv_probe_sink_words(ctypes.byref(shape), k, mode))


def probe_read_rows(shape: Shape, k_rows, v_rows, idx, k: int, mode: int, sink,
                    stream=None) -> None:
    """Read-rate probe (measurement only): reads the rows idx selects with the
    access pattern of one attention launch (PROBE_*) and no arithmetic; sink
    is a device tensor of at least probe_sink_words() int32/uint32 words."""
    _check("ckv_probe_read_rows", _lib.ckv_probe_read_rows(
        ctypes.byref(shape), _ptr(k_rows), _ptr(v_rows), _ptr(idx), k, mode, _ptr(sink),
        sink.numel() if sink is not None else 0, _stream(stream)))


def layer_array(layers) -> "ctypes.Array":
    """dicts with the ckv_layer field names (tensors, ints or None) -> the
    ckv_layer array the decode loop takes; an array is returned as it is, so
    a loop can build its per-parity arrays once."""
    if isinstance(layers, ctypes.Array):
        return layers
    arr = (Layer * len(layers))()
    for i, d in enumerate(layers):
        for name, typ in Layer._fields_:
            if typ is ctypes.c_int32:
                setattr(arr[i], name, int(d.get(name) or 0))
            else:
                setattr(arr[i], name, _ptr(d.get(name)))
    return arr


class Pipeline:
    """The decode loop of ``ckv_decode_step`` (owns its events): two buffers
    refilled on a copy stream, or, with ``k_buf`` and ``v_buf`` None, rows
    read in place from a cache in device memory."""

    def __init__(self):
        h = ctypes.c_void_p()
        _check("ckv_pipeline_create", _lib.ckv_pipeline_create(ctypes.byref(h)))
        self._h = h

    def close(self) -> None:
        if self._h:
            _lib.ckv_pipeline_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    CHECK_NO_FILL_WAIT, CHECK_NO_RELEASE_WAIT, CHECK_POISON, CHECK_NO_DEFER = 1, 2, 4, 8

    def set_checks(self, flags: int) -> None:
        """Tests of the event protocol only: skip the fill or release waits,
        or poison released buffers; or run every selection in its own layer's
        call (CHECK_NO_DEFER; see ckv_pipeline_set_checks)."""
        _check("ckv_pipeline_set_checks", _lib.ckv_pipeline_set_checks(self._h, flags))

    def set_gather_width(self, workgroups: int) -> None:
        _check("ckv_pipeline_set_gather_width",
               _lib.ckv_pipeline_set_gather_width(self._h, workgroups))

    @staticmethod
    def _bufs(k_buf, v_buf):
        """ctypes arrays of the two buffers; (None, None) for the in-place loop."""
        if k_buf is None and v_buf is None:
            return None, None
        kb = (ctypes.c_void_p * 2)(_ptr(k_buf[0]), _ptr(k_buf[1]))
        vb = (ctypes.c_void_p * 2)(_ptr(v_buf[0]), _ptr(v_buf[1]))
        return kb, vb

    def prime(self, shape: Shape, k: int, layers, src_kind: int, k_buf, v_buf,
              copy_stream) -> None:
        arr = layer_array(layers)
        kb, vb = self._bufs(k_buf, v_buf)
        _check("ckv_pipeline_prime", _lib.ckv_pipeline_prime(
            self._h, ctypes.byref(shape), k, arr, len(layers), src_kind, kb, vb,
            _stream(copy_stream)))

    def step(self, shape: Shape, layers, ctx_lens, k: int, scale: float, src_kind: int,
             k_buf, v_buf, ws, compute_stream, copy_stream) -> None:
        """One decode step over ``layers`` (dicts or a ``layer_array``)."""
        arr = layer_array(layers)
        kb, vb = self._bufs(k_buf, v_buf)
        _check("ckv_decode_step", _lib.ckv_decode_step(
            self._h, ctypes.byref(shape), len(layers), arr, _ptr(ctx_lens), k, scale,
            src_kind, kb, vb, _ptr(ws), ws.numel(), _stream(compute_stream),
            _stream(copy_stream)))
