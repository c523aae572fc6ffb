"""ctypes binding of libpdattn (include/pdattn.h): argument marshalling only.

Every step of the decode path runs in the library's CUDA kernels.  torch is used for device
memory and streams.  There is no CPU fallback: if the library has not been built, importing
`lib()` raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libpdattn.so")

OK = 0
INVALID_ARG = -1
UNSUPPORTED = -2
WORKSPACE_TOO_SMALL = -3
MISALIGNED = -4
NOT_BOUND = -5
CUDA_ERROR = -6
BAD_PAGE_INDEX = -7
DEVICE_TIMEOUT = -8
OUT_OF_PAGES = -9
BAD_SEQUENCE = -10

EXPORTS = [
    "pdattn_workspace_size", "pdattn_workspace_init", "pdattn_decode_ex", "pdattn_bind", "pdattn_decode",
    "pdattn_decode_host_fp8", "pdattn_decode_grouped_fp8",
    "pdattn_host_staging_size", "pdattn_decode_host", "pdattn_plan_host", "pdattn_check",
    "pdattn_last_launch_count", "pdattn_status_string", "pdattn_last_cuda_error", "pdattn_profile_events",
    "pdattn_gather_probe", "pdattn_stream_read_probe", "pdattn_wait_limit_probe", "pdattn_set_dynamic_spans",
    "pdattn_set_merge_mode", "pdattn_set_prefix_engine", "pdattn_set_host_zero_copy", "pdattn_set_short_piece_path",
    "pdattn_decode_static_scratch", "pdattn_append_kv",
    "pdattn_grouped_workspace_size", "pdattn_decode_grouped",
    "pdattn_multi_workspace_size", "pdattn_decode_multi", "pdattn_decode_fp8", "pdattn_append_kv_fp8", "pdattn_decode_fp8_multi",
    "pdattn_rope_append", "pdattn_rope_append_fp8", "pdattn_prefill_workspace_size", "pdattn_prefill",
    "pdattn_decode_scored", "pdattn_decode_scored_fp8",
    "pdattn_pages_workspace_size", "pdattn_pages_init", "pdattn_pages_reserve", "pdattn_pages_fork", "pdattn_pages_free",
    "pdattn_pages_compact", "pdattn_pages_copy",
    "pdattn_rope_append_at", "pdattn_rope_append_at_fp8", "pdattn_tree_workspace_size", "pdattn_decode_tree", "pdattn_decode_tree_fp8",
    "pdattn_tree_accept", "pdattn_pages_trim", "pdattn_summarize_append", "pdattn_summarize_pages", "pdattn_select_workspace_size",
    "pdattn_select_pages", "pdattn_decode_selected", "pdattn_decode_selected_fp8",
]


class PdattnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        L = lib()
        msg = L.pdattn_status_string(status).decode()
        if status == CUDA_ERROR:
            msg += ": " + L.pdattn_last_cuda_error().decode()
        super().__init__(f"{where}: {msg} ({status})")


class Args(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
        ("out", ctypes.c_void_p), ("block_table", ctypes.c_void_p), ("context_lens", ctypes.c_void_p),
        ("context_lens_host", ctypes.c_void_p),
        ("num_seqs", ctypes.c_int), ("num_q_heads", ctypes.c_int), ("num_kv_heads", ctypes.c_int),
        ("head_dim", ctypes.c_int), ("block_size", ctypes.c_int),
        ("max_blocks_per_seq", ctypes.c_int), ("num_blocks", ctypes.c_int),
        ("kv_block_stride", ctypes.c_int64), ("kv_head_stride", ctypes.c_int64), ("kv_token_stride", ctypes.c_int64),
        ("scale", ctypes.c_float),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
    ]


class RopeArgs(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("q_out", ctypes.c_void_p), ("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p),
        ("q_token_stride", ctypes.c_int64), ("k_token_stride", ctypes.c_int64), ("v_token_stride", ctypes.c_int64),
        ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
        ("context_lens", ctypes.c_void_p), ("cu_tokens", ctypes.c_void_p), ("inv_freq", ctypes.c_void_p),
        ("magnitude", ctypes.c_float), ("rotary_dim", ctypes.c_int), ("interleaved", ctypes.c_int),
        ("num_tokens", ctypes.c_int), ("num_seqs", ctypes.c_int), ("num_q_heads", ctypes.c_int),
        ("num_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("block_size", ctypes.c_int),
        ("max_blocks_per_seq", ctypes.c_int), ("num_blocks", ctypes.c_int),
        ("kv_block_stride", ctypes.c_int64), ("kv_head_stride", ctypes.c_int64), ("kv_token_stride", ctypes.c_int64),
        ("workspace", ctypes.c_void_p),
    ]


class ScoreArgs(ctypes.Structure):
    _fields_ = [("logit_cap", ctypes.c_float), ("bias_slopes", ctypes.c_void_p), ("window", ctypes.c_int),
                ("key_begin", ctypes.c_void_p), ("prefix_lens", ctypes.c_void_p), ("key_begin_host", ctypes.c_void_p)]


class SummaryArgs(ctypes.Structure):
    _fields_ = [("k_cache", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("codes", ctypes.c_void_p),
                ("exponents", ctypes.c_void_p), ("num_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("block_size", ctypes.c_int), ("num_blocks", ctypes.c_int), ("element_bytes", ctypes.c_int),
                ("kv_block_stride", ctypes.c_int64), ("kv_head_stride", ctypes.c_int64), ("kv_token_stride", ctypes.c_int64),
                ("workspace", ctypes.c_void_p)]


class SelectArgs(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("codes", ctypes.c_void_p), ("exponents", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p), ("context_lens", ctypes.c_void_p), ("selected", ctypes.c_void_p),
                ("num_seqs", ctypes.c_int), ("num_q_heads", ctypes.c_int), ("num_kv_heads", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("block_size", ctypes.c_int), ("max_blocks_per_seq", ctypes.c_int),
                ("num_blocks", ctypes.c_int), ("num_selected", ctypes.c_int), ("num_first", ctypes.c_int),
                ("num_recent", ctypes.c_int), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class PoolArgs(ctypes.Structure):
    _fields_ = [("ref_counts", ctypes.c_void_p), ("free_list", ctypes.c_void_p), ("free_count", ctypes.c_void_p),
                ("num_blocks", ctypes.c_int)]


class Plan(ctypes.Structure):
    _fields_ = [("n_static", ctypes.c_int), ("n_dynamic", ctypes.c_int), ("total_tiles", ctypes.c_int)]


_lib = None


def lib():
    """The loaded C-ABI library.  Raises if it has not been built (see build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2607_09207_b200.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        L.pdattn_workspace_size.argtypes = [i32] * 6 + [ctypes.POINTER(sz), ctypes.POINTER(sz)]
        L.pdattn_workspace_init.argtypes = [vp, sz, vp]
        L.pdattn_decode_ex.argtypes = [ctypes.POINTER(Args), vp]
        L.pdattn_bind.argtypes = [i32, i32, vp, sz, vp]
        L.pdattn_decode.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, f32, vp, vp]
        L.pdattn_host_staging_size.argtypes = [i32, i32, i32, i32, ctypes.POINTER(sz)]
        L.pdattn_decode_host.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, f32,
                                         vp, sz, vp, sz, vp]
        L.pdattn_plan_host.argtypes = [vp, i32, i32, i32, i32, i32, vp, ctypes.POINTER(Plan)]
        L.pdattn_set_dynamic_spans.argtypes = [i32]
        L.pdattn_set_merge_mode.argtypes = [i32]
        L.pdattn_set_prefix_engine.argtypes = [i32]
        L.pdattn_set_short_piece_path.argtypes = [i32]
        L.pdattn_set_host_zero_copy.argtypes = [i32]
        L.pdattn_decode_static_scratch.argtypes = [ctypes.POINTER(Args), vp, vp]
        L.pdattn_grouped_workspace_size.argtypes = [i32, i32, i32, i32, i32, ctypes.POINTER(sz)]
        L.pdattn_decode_grouped.argtypes = [ctypes.POINTER(Args), i32, vp, vp, vp]
        L.pdattn_decode_grouped_fp8.argtypes = [ctypes.POINTER(Args), i32, vp, vp, vp, vp, vp]
        L.pdattn_decode_host_fp8.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, f32,
                                             vp, sz, vp, sz, vp]
        L.pdattn_multi_workspace_size.argtypes = [i32, i32, i32, i32, i32, i32, ctypes.POINTER(sz)]
        L.pdattn_decode_multi.argtypes = [ctypes.POINTER(Args), i32, vp]
        L.pdattn_decode_fp8.argtypes = [ctypes.POINTER(Args), vp, vp, vp]
        L.pdattn_decode_fp8_multi.argtypes = [ctypes.POINTER(Args), i32, vp, vp, vp]
        L.pdattn_append_kv_fp8.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp]
        L.pdattn_append_kv.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i64, i64, i64, vp, vp]
        L.pdattn_check.argtypes = [vp, vp]
        L.pdattn_rope_append.argtypes = [ctypes.POINTER(RopeArgs), vp]
        L.pdattn_rope_append_fp8.argtypes = [ctypes.POINTER(RopeArgs), vp, vp, vp]
        L.pdattn_decode_scored.argtypes = [ctypes.POINTER(Args), ctypes.POINTER(ScoreArgs), vp]
        L.pdattn_decode_scored_fp8.argtypes = [ctypes.POINTER(Args), ctypes.POINTER(ScoreArgs), vp, vp, vp]
        L.pdattn_prefill_workspace_size.argtypes = [i32] * 6 + [ctypes.POINTER(sz)]
        L.pdattn_prefill.argtypes = [ctypes.POINTER(Args), vp, i32, ctypes.POINTER(ScoreArgs), vp]
        pool = ctypes.POINTER(PoolArgs)
        L.pdattn_pages_workspace_size.argtypes = [i32, i32, ctypes.POINTER(sz)]
        L.pdattn_pages_init.argtypes = [pool, vp]
        L.pdattn_pages_reserve.argtypes = [pool, vp, vp, vp, i32, i32, i32, vp, sz, vp]
        L.pdattn_pages_fork.argtypes = [pool, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, sz, vp]
        L.pdattn_pages_free.argtypes = [pool, vp, vp, vp, i32, i32, i32, i32, vp, sz, vp]
        L.pdattn_pages_compact.argtypes = [pool, vp, vp, i32, i32, i32, vp, vp, i32, vp, sz, vp]
        L.pdattn_pages_copy.argtypes = [vp] * 4 + [i32] * 6 + [i64] * 3 + [vp, vp]
        L.pdattn_rope_append_at.argtypes = [ctypes.POINTER(RopeArgs), vp, vp]
        L.pdattn_rope_append_at_fp8.argtypes = [ctypes.POINTER(RopeArgs), vp, vp, vp, vp]
        L.pdattn_tree_workspace_size.argtypes = [i32] * 5 + [ctypes.POINTER(sz)]
        L.pdattn_decode_tree.argtypes = [ctypes.POINTER(Args), vp, i32, vp, i32, vp]
        L.pdattn_decode_tree_fp8.argtypes = [ctypes.POINTER(Args), vp, i32, vp, i32, vp, vp, vp]
        L.pdattn_tree_accept.argtypes = [vp] * 7 + [i32] * 8 + [i64] * 3 + [vp, vp]
        L.pdattn_pages_trim.argtypes = [pool, vp, vp, vp, i32, i32, i32, vp, sz, vp]
        L.pdattn_summarize_append.argtypes = [ctypes.POINTER(SummaryArgs), vp, vp, vp, i32, i32, i32, vp]
        L.pdattn_summarize_pages.argtypes = [ctypes.POINTER(SummaryArgs), vp, i32, vp]
        L.pdattn_select_workspace_size.argtypes = [i32] * 3 + [ctypes.POINTER(sz)]
        L.pdattn_select_pages.argtypes = [ctypes.POINTER(SelectArgs), vp]
        L.pdattn_decode_selected.argtypes = [ctypes.POINTER(Args), vp, i32, vp]
        L.pdattn_decode_selected_fp8.argtypes = [ctypes.POINTER(Args), vp, i32, vp, vp, vp]
        L.pdattn_profile_events.argtypes = [vp, vp]
        L.pdattn_gather_probe.argtypes = [ctypes.POINTER(Args), vp]
        L.pdattn_stream_read_probe.argtypes = [vp, sz, vp, vp]
        L.pdattn_wait_limit_probe.argtypes = [vp, i32, vp]
        L.pdattn_last_launch_count.argtypes = []
        L.pdattn_status_string.argtypes = [i32]
        L.pdattn_status_string.restype = ctypes.c_char_p
        L.pdattn_last_cuda_error.argtypes = []
        L.pdattn_last_cuda_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _stream_ptr(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream)


def workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size=16, max_context_len=0) -> int:
    dev, pin = ctypes.c_size_t(0), ctypes.c_size_t(0)
    st = lib().pdattn_workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size, max_context_len,
                                     ctypes.byref(dev), ctypes.byref(pin))
    if st != OK:
        raise PdattnError(st, "pdattn_workspace_size")
    return dev.value


def alloc_workspace(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size=16, device="cuda", stream=None):
    """torch-owned workspace, error word cleared."""
    n = workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    st = lib().pdattn_workspace_init(ws.data_ptr(), n, _stream_ptr(stream))
    if st != OK:
        raise PdattnError(st, "pdattn_workspace_init")
    return ws


def decode_ex(q, k_cache, v_cache, block_table, context_lens, scale, out, workspace,
              context_lens_host: Optional[np.ndarray] = None, num_blocks: Optional[int] = None,
              stream=None, check: bool = True, probe: bool = False) -> int:
    """pdattn_decode_ex.  k_cache / v_cache: bf16 tensors indexed [page, kv_head, slot, dim] with any
    strides whose last dimension is contiguous.  Returns the status (raises unless check=False)."""
    S, Hq, d = q.shape
    NB, Hkv, bs, _ = k_cache.shape
    a = Args()
    a.q, a.k_cache, a.v_cache, a.out = q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), out.data_ptr()
    a.block_table, a.context_lens = block_table.data_ptr(), context_lens.data_ptr()
    keep = None
    if context_lens_host is not None:
        keep = np.ascontiguousarray(context_lens_host, dtype=np.int32)
        a.context_lens_host = keep.ctypes.data
    else:
        a.context_lens_host = None
    a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size = S, Hq, Hkv, d, bs
    a.max_blocks_per_seq = block_table.shape[1] if block_table.dim() == 2 else 0
    a.num_blocks = NB if num_blocks is None else num_blocks
    a.kv_block_stride, a.kv_head_stride, a.kv_token_stride = k_cache.stride(0), k_cache.stride(1), k_cache.stride(2)
    a.scale = float(scale)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    fn = lib().pdattn_gather_probe if probe else lib().pdattn_decode_ex
    st = fn(ctypes.byref(a), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_gather_probe" if probe else "pdattn_decode_ex")
    return st


def decode_static_scratch(q, k_cache, v_cache, block_table, context_lens, scale, out,
                          context_lens_host: Optional[np.ndarray] = None, status_out: Optional[torch.Tensor] = None,
                          stream=None, check: bool = True) -> int:
    """pdattn_decode_static_scratch: the decode step on the library's built-in scratch array, for callers
    that can neither provide a workspace nor let the library allocate one.  status_out: optional int32
    device tensor of one element that receives this call's error bits."""
    S, Hq, d = q.shape
    NB, Hkv, bs, _ = k_cache.shape
    a = Args()
    a.q, a.k_cache, a.v_cache, a.out = q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), out.data_ptr()
    a.block_table, a.context_lens = block_table.data_ptr(), context_lens.data_ptr()
    keep = None
    if context_lens_host is not None:
        keep = np.ascontiguousarray(context_lens_host, dtype=np.int32)
        a.context_lens_host = keep.ctypes.data
    a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size = S, Hq, Hkv, d, bs
    a.max_blocks_per_seq = block_table.shape[1] if block_table.dim() == 2 else 0
    a.num_blocks = NB
    a.kv_block_stride, a.kv_head_stride, a.kv_token_stride = k_cache.stride(0), k_cache.stride(1), k_cache.stride(2)
    a.scale = float(scale)
    st = lib().pdattn_decode_static_scratch(ctypes.byref(a), status_out.data_ptr() if status_out is not None else None,
                                            _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_decode_static_scratch")
    return st


def grouped_workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size=16) -> int:
    n = ctypes.c_size_t(0)
    st = lib().pdattn_grouped_workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size, ctypes.byref(n))
    if st != OK:
        raise PdattnError(st, "pdattn_grouped_workspace_size")
    return n.value


def alloc_grouped_workspace(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size=16, device="cuda", stream=None):
    n = grouped_workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    st = lib().pdattn_workspace_init(ws.data_ptr(), n, _stream_ptr(stream))
    if st != OK:
        raise PdattnError(st, "pdattn_workspace_init")
    return ws


def decode_grouped(q, k_cache, v_cache, block_table, context_lens, scale, out, workspace, context_lens_host,
                   group_size, prefix_tiles, prefix_tiles_host, stream=None, check: bool = True) -> int:
    """pdattn_decode_grouped: sequences come in groups of `group_size` whose first prefix_tiles[g] * 64 tokens
    are the same physical pages (GRPO samples of one prompt); those tiles are read once per group."""
    S, Hq, d = q.shape
    NB, Hkv, bs, _ = k_cache.shape
    a = Args()
    a.q, a.k_cache, a.v_cache, a.out = q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), out.data_ptr()
    a.block_table, a.context_lens = block_table.data_ptr(), context_lens.data_ptr()
    lens = np.ascontiguousarray(context_lens_host, dtype=np.int32)
    a.context_lens_host = lens.ctypes.data
    a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size = S, Hq, Hkv, d, bs
    a.max_blocks_per_seq = block_table.shape[1]
    a.num_blocks = NB
    a.kv_block_stride, a.kv_head_stride, a.kv_token_stride = k_cache.stride(0), k_cache.stride(1), k_cache.stride(2)
    a.scale = float(scale)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    pth = np.ascontiguousarray(prefix_tiles_host, dtype=np.int32)
    st = lib().pdattn_decode_grouped(ctypes.byref(a), int(group_size), prefix_tiles.data_ptr(), pth.ctypes.data,
                                     _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_decode_grouped")
    return st


def multi_workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size, num_query_tokens) -> int:
    n = ctypes.c_size_t(0)
    st = lib().pdattn_multi_workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size,
                                           num_query_tokens, ctypes.byref(n))
    if st != OK:
        raise PdattnError(st, "pdattn_multi_workspace_size")
    return n.value


def alloc_multi_workspace(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size, num_query_tokens,
                          device="cuda", stream=None):
    n = multi_workspace_size(num_seqs, num_q_heads, num_kv_heads, head_dim, block_size, num_query_tokens)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    st = lib().pdattn_workspace_init(ws.data_ptr(), n, _stream_ptr(stream))
    if st != OK:
        raise PdattnError(st, "pdattn_workspace_init")
    return ws


def decode_multi(q, k_cache, v_cache, block_table, context_lens, scale, out, workspace, context_lens_host=None,
                 stream=None, check: bool = True) -> int:
    """pdattn_decode_multi: q and out are [num_seqs, T, num_q_heads, head_dim]; the last T tokens of every
    sequence are new and each attends to the keys up to its own position."""
    S, T, Hq, d = q.shape
    NB, Hkv, bs, _ = k_cache.shape
    a = Args()
    a.q, a.k_cache, a.v_cache, a.out = q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), out.data_ptr()
    a.block_table, a.context_lens = block_table.data_ptr(), context_lens.data_ptr()
    lens = None
    if context_lens_host is not None:
        lens = np.ascontiguousarray(context_lens_host, dtype=np.int32)
        a.context_lens_host = lens.ctypes.data
    a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size = S, Hq, Hkv, d, bs
    a.max_blocks_per_seq = block_table.shape[1]
    a.num_blocks = NB
    a.kv_block_stride, a.kv_head_stride, a.kv_token_stride = k_cache.stride(0), k_cache.stride(1), k_cache.stride(2)
    a.scale = float(scale)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    st = lib().pdattn_decode_multi(ctypes.byref(a), int(T), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_decode_multi")
    return st


def decode_fp8(q, k8, v8, k_scale, v_scale, block_table, context_lens, scale, out, workspace,
               context_lens_host=None, stream=None, check: bool = True) -> int:
    """pdattn_decode_fp8: k8 uint8 [pages, Hkv, block_size, d], v8 uint8 [pages, Hkv, d, block_size] (e4m3 codes),
    k_scale / v_scale fp32 [Hkv] on the device."""
    T = q.shape[1] if q.dim() == 4 else 0          # [S, T, Hq, d]: several new tokens per sequence
    S, Hq, d = q.shape[0], q.shape[-2], q.shape[-1]
    NB, Hkv, bs, _ = k8.shape
    assert k8.dtype == torch.uint8 and v8.dtype == torch.uint8 and tuple(v8.shape) == (NB, Hkv, d, bs)
    assert k8.is_contiguous() and v8.is_contiguous() and k_scale.dtype == torch.float32 and v_scale.dtype == torch.float32
    a = Args()
    a.q, a.k_cache, a.v_cache, a.out = q.data_ptr(), k8.data_ptr(), v8.data_ptr(), out.data_ptr()
    a.block_table, a.context_lens = block_table.data_ptr(), context_lens.data_ptr()
    lens = None
    if context_lens_host is not None:
        lens = np.ascontiguousarray(context_lens_host, dtype=np.int32)
        a.context_lens_host = lens.ctypes.data
    a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size = S, Hq, Hkv, d, bs
    a.max_blocks_per_seq = block_table.shape[1]
    a.num_blocks = NB
    a.kv_block_stride, a.kv_head_stride, a.kv_token_stride = Hkv * bs * d, bs * d, d
    a.scale = float(scale)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    if T:
        st = lib().pdattn_decode_fp8_multi(ctypes.byref(a), T, k_scale.data_ptr(), v_scale.data_ptr(), _stream_ptr(stream))
    else:
        st = lib().pdattn_decode_fp8(ctypes.byref(a), k_scale.data_ptr(), v_scale.data_ptr(), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_decode_fp8")
    return st


def decode_grouped_fp8(q, k8, v8, k_scale, v_scale, block_table, context_lens, scale, out, workspace,
                       context_lens_host, group_size, prefix_tiles, prefix_tiles_host, stream=None,
                       check: bool = True) -> int:
    """pdattn_decode_grouped_fp8: decode_grouped over the e4m3 code pools of decode_fp8."""
    S, Hq, d = q.shape
    NB, Hkv, bs, _ = k8.shape
    assert k8.dtype == torch.uint8 and v8.dtype == torch.uint8 and tuple(v8.shape) == (NB, Hkv, d, bs)
    assert k8.is_contiguous() and v8.is_contiguous()
    a = Args()
    a.q, a.k_cache, a.v_cache, a.out = q.data_ptr(), k8.data_ptr(), v8.data_ptr(), out.data_ptr()
    a.block_table, a.context_lens = block_table.data_ptr(), context_lens.data_ptr()
    lens = np.ascontiguousarray(context_lens_host, dtype=np.int32)
    a.context_lens_host = lens.ctypes.data
    a.num_seqs, a.num_q_heads, a.num_kv_heads, a.head_dim, a.block_size = S, Hq, Hkv, d, bs
    a.max_blocks_per_seq = block_table.shape[1]
    a.num_blocks = NB
    a.kv_block_stride, a.kv_head_stride, a.kv_token_stride = Hkv * bs * d, bs * d, d
    a.scale = float(scale)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    pth = np.ascontiguousarray(prefix_tiles_host, dtype=np.int32)
    st = lib().pdattn_decode_grouped_fp8(ctypes.byref(a), int(group_size), prefix_tiles.data_ptr(), pth.ctypes.data,
                                         k_scale.data_ptr(), v_scale.data_ptr(), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_decode_grouped_fp8")
    return st


def decode_host_fp8(q_host, block_table_host, context_lens_host, out_host, k8, v8, k_scale, v_scale, scale, staging,
                    workspace, stream=None, check: bool = True) -> int:
    """pdattn_decode_host_fp8: q / block_table / context_lens / out are HOST tensors (pinned), code pools and scales
    on the device."""
    S, Hq, d = q_host.shape
    NB, Hkv, bs, _ = k8.shape
    st = lib().pdattn_decode_host_fp8(q_host.data_ptr(), block_table_host.data_ptr(), context_lens_host.data_ptr(),
                                      out_host.data_ptr(), k8.data_ptr(), v8.data_ptr(), k_scale.data_ptr(),
                                      v_scale.data_ptr(), S, Hq, Hkv, d, bs, block_table_host.shape[1], NB, float(scale),
                                      staging.data_ptr(), staging.numel(), workspace.data_ptr(), workspace.numel(),
                                      _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_decode_host_fp8")
    return st


def append_kv_fp8(k_new, v_new, k8, v8, k_scale, v_scale, block_table, context_lens, workspace=None, stream=None,
                  check: bool = True) -> int:
    """pdattn_append_kv_fp8: quantise the new K/V rows into the fp8 cache and advance context_lens (device, in place)."""
    S, Hkv, d = k_new.shape
    NB, _, bs, _ = k8.shape
    st = lib().pdattn_append_kv_fp8(k_new.data_ptr(), v_new.data_ptr(), k8.data_ptr(), v8.data_ptr(), k_scale.data_ptr(),
                                    v_scale.data_ptr(), block_table.data_ptr(), context_lens.data_ptr(), S, Hkv, d, bs,
                                    block_table.shape[1], NB, workspace.data_ptr() if workspace is not None else None,
                                    _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_append_kv_fp8")
    return st


def append_kv(k_new, v_new, k_cache, v_cache, block_table, context_lens, workspace=None, stream=None,
              check: bool = True) -> int:
    """pdattn_append_kv: write this step's K/V rows ([S, Hkv, d]) into the paged caches and advance
    context_lens (device tensor, in place)."""
    S, Hkv, d = k_new.shape
    NB, _, bs, _ = k_cache.shape
    st = lib().pdattn_append_kv(k_new.data_ptr(), v_new.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                block_table.data_ptr(), context_lens.data_ptr(), S, Hkv, d, bs, block_table.shape[1],
                                NB, k_cache.stride(0), k_cache.stride(1), k_cache.stride(2),
                                workspace.data_ptr() if workspace is not None else None, _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_append_kv")
    return st


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _expect(where: str, dtype, *tensors):
    """dtype and device checks of the tensors a call takes (None is passed over): the library sees plain pointers."""
    here = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and (t.dtype is not dtype or t.get_device() != here):
            if t.dtype is not dtype:
                raise TypeError(f"{where}: a tensor of {dtype} is wanted, got {t.dtype}")
            raise ValueError(f"{where}: a tensor lives on {t.device}, the current device is cuda:{here}")


def _expect_dense(where: str, dtype, *tensors):
    """_expect, and no gaps between the elements."""
    here = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and (t.dtype is not dtype or t.get_device() != here or not t.is_contiguous()):
            _expect(where, dtype, t)
            raise ValueError(f"{where}: a dense tensor is wanted, got strides {t.stride()} for shape {tuple(t.shape)}")


def _expect_workspace(where: str, workspace):
    """A dense tensor of bytes on the current device, one that can hold the error word at least."""
    _expect_dense(where, torch.uint8, workspace)
    if workspace.numel() < 4:
        raise ValueError(f"{where}: a workspace of {workspace.numel()} bytes")


def _expect_device(where: str, device: int):
    here = torch._C._cuda_getDevice()
    if device != here:
        raise ValueError(f"{where}: tensors on cuda:{device}, the current device is cuda:{here}")


def _expect_caches(where: str, k_cache, v_cache):
    """bf16 caches [page, kv_head, slot, dim] that can share one set of strides."""
    _expect(where, torch.bfloat16, k_cache, v_cache)
    if k_cache.shape != v_cache.shape or k_cache.stride() != v_cache.stride() or k_cache.stride(3) != 1:
        raise ValueError(f"{where}: k_cache and v_cache need the same shape and strides, head_dim contiguous")


def _expect_codes(where: str, k8, v8, k_scale, v_scale):
    """The code pools of decode_fp8 and their scales."""
    _expect_dense(where, torch.uint8, k8, v8)
    _expect_dense(where, torch.float32, k_scale, v_scale)
    NB, Hkv, bs, d = k8.shape
    if v8.shape != (NB, Hkv, d, bs) or k_scale.numel() != Hkv or v_scale.numel() != Hkv:
        raise ValueError(f"{where}: code pools {tuple(k8.shape)} and {tuple(v8.shape)} with {k_scale.numel()} and "
                         f"{v_scale.numel()} scales do not belong together")


def _token_stride(where, t, shape) -> int:
    """Elements between two tokens of t [N, heads, d], whose heads lie densely."""
    N, H, d = shape
    st = t.stride()
    if t.shape != shape or (N and (st[2] != 1 or (H > 1 and st[1] != d))):
        raise ValueError(f"{where}: {N} rows of {H} dense heads of {d} are wanted, got shape {tuple(t.shape)}, strides {st}")
    return st[0] if N > 1 else H * d


def _rope_args(where, q, k_new, v_new, q_out, k_cache, v_cache, kv_strides, block_table, context_lens, inv_freq, cu_tokens,
               rotary_dim, interleaved, magnitude, workspace) -> RopeArgs:
    shape = k_new.shape
    N, Hkv, d = shape
    NB, heads, bs, dim = k_cache.shape
    _expect(where, torch.bfloat16, q, k_new, v_new)
    _expect_dense(where, torch.bfloat16, q_out)
    _expect_dense(where, torch.int32, block_table, context_lens, cu_tokens)
    _expect_dense(where, torch.float32, inv_freq)
    if workspace is not None:
        _expect_workspace(where, workspace)
    S, MB = block_table.shape
    rotary = d if rotary_dim is None else int(rotary_dim)
    if (heads != Hkv or dim != d or context_lens.numel() != S or inv_freq.numel() * 2 != rotary
            or (cu_tokens is not None and cu_tokens.numel() != S + 1)):
        raise ValueError(f"{where}: shapes do not belong together")
    Hq, q_stride = 0, 0
    if q is not None:
        Hq = q.shape[1]
        q_stride = _token_stride(where, q, (N, Hq, d))
        if q_out is None or q_out.shape != (N, Hq, d):
            raise ValueError(f"{where}: q_out has the shape of q")
    return RopeArgs(_ptr(q), _ptr(q_out) if Hq else None, k_new.data_ptr(), v_new.data_ptr(), q_stride,
                    _token_stride(where, k_new, shape), _token_stride(where, v_new, shape), k_cache.data_ptr(), v_cache.data_ptr(),
                    block_table.data_ptr(), context_lens.data_ptr(), _ptr(cu_tokens), inv_freq.data_ptr(), magnitude, rotary,
                    1 if interleaved else 0, N, S, Hq, Hkv, d, bs, MB, NB, *kv_strides, _ptr(workspace))


def _positions(where, positions, num_tokens):
    _expect_dense(where, torch.int32, positions)
    if positions.numel() != num_tokens:
        raise ValueError(f"{where}: {positions.numel()} positions for {num_tokens} tokens")
    return positions.data_ptr()


def rope_append(q, k_new, v_new, q_out, k_cache, v_cache, block_table, context_lens, inv_freq, *, cu_tokens=None,
                rotary_dim=None, interleaved: bool = False, magnitude: float = 1.0, workspace=None, stream=None,
                check: bool = True, positions=None) -> int:
    """pdattn_rope_append: rotate q ([N, Hq, d], rows of any token stride; None: only k and v) into q_out and k_new into
    the paged cache beside v_new ([N, Hkv, d]).  context_lens counts the new tokens; cu_tokens [S + 1] (None: one new
    token per sequence).  positions (int32 [N], pdattn_rope_append_at): those of the rotation, for tokens of a tree."""
    where = "pdattn_rope_append"
    _expect_caches(where, k_cache, v_cache)
    a = _rope_args(where, q, k_new, v_new, q_out, k_cache, v_cache, k_cache.stride()[:3], block_table, context_lens, inv_freq,
                   cu_tokens, rotary_dim, interleaved, magnitude, workspace)
    if positions is None:
        st = lib().pdattn_rope_append(ctypes.byref(a), _stream_ptr(stream))
    else:
        where = "pdattn_rope_append_at"
        st = lib().pdattn_rope_append_at(ctypes.byref(a), _positions(where, positions, a.num_tokens), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def rope_append_fp8(q, k_new, v_new, q_out, k8, v8, k_scale, v_scale, block_table, context_lens, inv_freq, *,
                    cu_tokens=None, rotary_dim=None, interleaved: bool = False, magnitude: float = 1.0, workspace=None,
                    stream=None, check: bool = True, positions=None) -> int:
    """pdattn_rope_append_fp8: rope_append into the e4m3 code pools of decode_fp8."""
    where = "pdattn_rope_append_fp8"
    _expect_codes(where, k8, v8, k_scale, v_scale)
    a = _rope_args(where, q, k_new, v_new, q_out, k8, v8, (0, 0, 0), block_table, context_lens, inv_freq, cu_tokens, rotary_dim,
                   interleaved, magnitude, workspace)
    if positions is None:
        st = lib().pdattn_rope_append_fp8(ctypes.byref(a), k_scale.data_ptr(), v_scale.data_ptr(), _stream_ptr(stream))
    else:
        where = "pdattn_rope_append_at_fp8"
        st = lib().pdattn_rope_append_at_fp8(ctypes.byref(a), _positions(where, positions, a.num_tokens), k_scale.data_ptr(),
                                             v_scale.data_ptr(), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


class Score:
    """Modified scores and masks (pdattn_score_args): logit_cap, bias_slopes (fp32 [Hq]), window, key_begin (int32, one per
    query token), prefix_lens (int32 [S]); key_begin_host: the host copy a decode call with host lengths needs."""

    def __init__(self, logit_cap: float = 0.0, bias_slopes=None, window: int = 0, key_begin=None, prefix_lens=None,
                 key_begin_host: Optional[np.ndarray] = None):
        _expect_dense("Score", torch.float32, bias_slopes)
        _expect_dense("Score", torch.int32, key_begin, prefix_lens)
        host = None if key_begin_host is None else np.ascontiguousarray(key_begin_host, dtype=np.int32)
        self.keep = (bias_slopes, key_begin, prefix_lens, host)
        self.device = next((t.get_device() for t in self.keep[:3] if t is not None), None)
        self.args = ScoreArgs(float(logit_cap), _ptr(bias_slopes), int(window), _ptr(key_begin), _ptr(prefix_lens),
                              None if host is None else host.ctypes.data)

    def fits(self, where: str, num_q_heads: int, num_tokens: int, num_seqs: int):
        slopes, begin, prefix, host = self.keep
        if self.device is not None:
            _expect_device(where, self.device)
        if slopes is not None and slopes.numel() != num_q_heads:
            raise ValueError(f"{where}: bias_slopes has {slopes.numel()} entries for {num_q_heads} query heads")
        if begin is not None and begin.numel() != num_tokens:
            raise ValueError(f"{where}: key_begin has {begin.numel()} entries for {num_tokens} query tokens")
        if host is not None and host.size != num_tokens:
            raise ValueError(f"{where}: key_begin_host has {host.size} entries for {num_tokens} query tokens")
        if prefix is not None and prefix.numel() != num_seqs:
            raise ValueError(f"{where}: prefix_lens has {prefix.numel()} entries for {num_seqs} sequences")


def _step_args(where, q, k_cache, v_cache, kv_strides, block_table, context_lens, scale, out, workspace,
               context_lens_host=None) -> Args:
    """The argument block of a call over bf16 or code caches whose q and out are [rows, Hq, d]."""
    _expect_dense(where, torch.bfloat16, q, out)
    _expect_dense(where, torch.int32, block_table, context_lens)
    _expect_workspace(where, workspace)
    shape = q.shape
    _, Hq, d = shape
    NB, Hkv, bs, dim = k_cache.shape
    S, MB = block_table.shape
    if dim != d or out.shape != shape or context_lens.numel() != S:
        raise ValueError(f"{where}: shapes do not belong together")
    host = None
    if context_lens_host is not None:
        host = np.ascontiguousarray(context_lens_host, dtype=np.int32)
        if host.size != S:
            raise ValueError(f"{where}: context_lens_host has {host.size} entries for {S} sequences")
    a = Args(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), out.data_ptr(), block_table.data_ptr(),
             context_lens.data_ptr(), None if host is None else host.ctypes.data, S, Hq, Hkv, d, bs, MB, NB, *kv_strides, scale,
             workspace.data_ptr(), workspace.numel())
    a.keep = host                                  # lives as long as the block
    return a


def prefill_workspace_size(num_seqs, num_tokens, num_q_heads, num_kv_heads, head_dim, block_size=16) -> int:
    n = ctypes.c_size_t(0)
    st = lib().pdattn_prefill_workspace_size(num_seqs, num_tokens, num_q_heads, num_kv_heads, head_dim, block_size,
                                             ctypes.byref(n))
    if st != OK:
        raise PdattnError(st, "pdattn_prefill_workspace_size")
    return n.value


def alloc_prefill_workspace(num_seqs, num_tokens, num_q_heads, num_kv_heads, head_dim, block_size=16, device="cuda",
                            stream=None):
    n = prefill_workspace_size(num_seqs, num_tokens, num_q_heads, num_kv_heads, head_dim, block_size)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    st = lib().pdattn_workspace_init(ws.data_ptr(), n, _stream_ptr(stream))
    if st != OK:
        raise PdattnError(st, "pdattn_workspace_init")
    return ws


def prefill(q, k_cache, v_cache, block_table, context_lens, cu_tokens, scale, out, workspace, *,
            score: Optional[Score] = None, stream=None, check: bool = True) -> int:
    """pdattn_prefill: q and out [N, Hq, d]; the tokens cu_tokens[s] .. cu_tokens[s + 1] are the last ones of sequence s's
    context_lens[s] (their K and V are in the caches); each attends by the rules of `score` (None: plain causal)."""
    where = "pdattn_prefill"
    _expect_caches(where, k_cache, v_cache)
    _expect_dense(where, torch.int32, cu_tokens)
    a = _step_args(where, q, k_cache, v_cache, k_cache.stride()[:3], block_table, context_lens, scale, out, workspace)
    if cu_tokens.numel() != a.num_seqs + 1:
        raise ValueError(f"{where}: cu_tokens has {cu_tokens.numel()} entries for {a.num_seqs} sequences")
    if score is not None:
        score.fits(where, a.num_q_heads, q.shape[0], a.num_seqs)
    st = lib().pdattn_prefill(ctypes.byref(a), cu_tokens.data_ptr(), q.shape[0],
                              ctypes.byref(score.args) if score is not None else None, _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def decode_scored(q, k_cache, v_cache, block_table, context_lens, scale, out, workspace, score: Score,
                  context_lens_host: Optional[np.ndarray] = None, stream=None, check: bool = True) -> int:
    """pdattn_decode_scored: decode_ex with the modified scores and masks of `score`."""
    where = "pdattn_decode_scored"
    _expect_caches(where, k_cache, v_cache)
    a = _step_args(where, q, k_cache, v_cache, k_cache.stride()[:3], block_table, context_lens, scale, out, workspace,
                   context_lens_host)
    return _scored(where, lib().pdattn_decode_scored, q, a, score, (), stream, check)


def decode_scored_fp8(q, k8, v8, k_scale, v_scale, block_table, context_lens, scale, out, workspace, score: Score,
                      context_lens_host: Optional[np.ndarray] = None, stream=None, check: bool = True) -> int:
    """pdattn_decode_scored_fp8: decode_scored over the e4m3 code pools of decode_fp8."""
    where = "pdattn_decode_scored_fp8"
    _expect_codes(where, k8, v8, k_scale, v_scale)
    a = _step_args(where, q, k8, v8, (0, 0, 0), block_table, context_lens, scale, out, workspace, context_lens_host)
    return _scored(where, lib().pdattn_decode_scored_fp8, q, a, score, (k_scale.data_ptr(), v_scale.data_ptr()), stream, check)


def _scored(where, call, q, a: Args, score: Score, scales, stream, check) -> int:
    if q.shape[0] != a.num_seqs:
        raise ValueError(f"{where}: {q.shape[0]} query rows for {a.num_seqs} sequences")
    score.fits(where, a.num_q_heads, a.num_seqs, a.num_seqs)
    st = call(ctypes.byref(a), ctypes.byref(score.args), *scales, _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def tree_workspace_size(num_q_heads, num_kv_heads, head_dim, block_size=16, max_tree_tokens=64) -> int:
    n = ctypes.c_size_t(0)
    st = lib().pdattn_tree_workspace_size(num_q_heads, num_kv_heads, head_dim, block_size, max_tree_tokens, ctypes.byref(n))
    if st != OK:
        raise PdattnError(st, "pdattn_tree_workspace_size")
    return n.value


def _alloc(n, device, stream):
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    st = lib().pdattn_workspace_init(ws.data_ptr(), n, _stream_ptr(stream))
    if st != OK:
        raise PdattnError(st, "pdattn_workspace_init")
    return ws


def alloc_tree_workspace(num_q_heads, num_kv_heads, head_dim, block_size=16, max_tree_tokens=64, device="cuda", stream=None):
    return _alloc(tree_workspace_size(num_q_heads, num_kv_heads, head_dim, block_size, max_tree_tokens), device, stream)


def _tree(where, call, q, a: Args, cu_tokens, tree_mask, max_tree_tokens, scales, stream, check) -> int:
    _expect_dense(where, torch.int32, cu_tokens)
    if tree_mask.dtype not in (torch.int64, torch.uint64):
        raise TypeError(f"{where}: tree_mask holds 64 bits per token, got {tree_mask.dtype}")
    _expect_dense(where, tree_mask.dtype, tree_mask)
    if cu_tokens.numel() != a.num_seqs + 1:
        raise ValueError(f"{where}: cu_tokens has {cu_tokens.numel()} entries for {a.num_seqs} sequences")
    if tree_mask.numel() != q.shape[0]:
        raise ValueError(f"{where}: tree_mask has {tree_mask.numel()} entries for {q.shape[0]} tokens")
    st = call(ctypes.byref(a), cu_tokens.data_ptr(), q.shape[0], tree_mask.data_ptr(), max_tree_tokens, *scales, _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def decode_tree(q, k_cache, v_cache, block_table, context_lens, cu_tokens, tree_mask, scale, out, workspace, *,
                max_tree_tokens: int = 64, stream=None, check: bool = True) -> int:
    """pdattn_decode_tree: q and out [N, Hq, d]; the drafted tokens cu_tokens[s] .. cu_tokens[s + 1] are the last ones of sequence s's
    context_lens[s], and token j of them sees token i of the tree where bit i of its tree_mask (int64 or uint64 [N]) is set.  Give the
    batch's max_tree_tokens where it is known: small trees take longer in the form for 64 (256 of 8 tokens 270 us in place of 238)."""
    where = "pdattn_decode_tree"
    _expect_caches(where, k_cache, v_cache)
    a = _step_args(where, q, k_cache, v_cache, k_cache.stride()[:3], block_table, context_lens, scale, out, workspace)
    return _tree(where, lib().pdattn_decode_tree, q, a, cu_tokens, tree_mask, max_tree_tokens, (), stream, check)


def decode_tree_fp8(q, k8, v8, k_scale, v_scale, block_table, context_lens, cu_tokens, tree_mask, scale, out, workspace, *,
                    max_tree_tokens: int = 64, stream=None, check: bool = True) -> int:
    """pdattn_decode_tree_fp8: decode_tree over the e4m3 code pools of decode_fp8."""
    where = "pdattn_decode_tree_fp8"
    _expect_codes(where, k8, v8, k_scale, v_scale)
    a = _step_args(where, q, k8, v8, (0, 0, 0), block_table, context_lens, scale, out, workspace)
    return _tree(where, lib().pdattn_decode_tree_fp8, q, a, cu_tokens, tree_mask, max_tree_tokens,
                 (k_scale.data_ptr(), v_scale.data_ptr()), stream, check)


def _expect_pools(where, k_cache, v_cache):
    """bf16 caches, or the code pools of decode_fp8."""
    if k_cache.dtype == torch.uint8:
        _expect_dense(where, torch.uint8, k_cache, v_cache)
        NB, Hkv, bs, d = k_cache.shape
        if tuple(v_cache.shape) != (NB, Hkv, d, bs):
            raise ValueError(f"{where}: code pools {tuple(k_cache.shape)} and {tuple(v_cache.shape)} do not belong together")
    else:
        _expect_caches(where, k_cache, v_cache)


def tree_accept(k_cache, v_cache, block_table, context_lens, cu_tokens, accepted, accepted_counts, workspace=None, stream=None,
                check: bool = True) -> int:
    """pdattn_tree_accept: K and V of the tree's tokens accepted[s, :accepted_counts[s]] (int32 [S, M], [S]) move to the front of the tree's
    slots, in bf16 caches or the uint8 code pools of decode_fp8; the lengths stay.  Pages are summarised after this and pages_trim, by
    summarize_append with the accepted counts."""
    where = "pdattn_tree_accept"
    _expect_dense(where, torch.int32, block_table, context_lens, cu_tokens, accepted, accepted_counts)
    _expect_pools(where, k_cache, v_cache)
    if workspace is not None:
        _expect_workspace(where, workspace)
    S, MB = block_table.shape
    if context_lens.numel() != S or cu_tokens.numel() != S + 1 or accepted.dim() != 2 or accepted.shape[0] != S or accepted_counts.numel() != S:
        raise ValueError(f"{where}: shapes do not belong together")
    NB, Hkv, bs, d = k_cache.shape
    st = lib().pdattn_tree_accept(k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(), context_lens.data_ptr(),
                                  cu_tokens.data_ptr(), accepted.data_ptr(), accepted_counts.data_ptr(), accepted.shape[1], S, Hkv, d,
                                  bs, MB, NB, k_cache.element_size(), *k_cache.stride()[:3], _ptr(workspace), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


class PageSummary:
    """Summaries of a pool's pages (pdattn_summary_args): codes int8 [pages, Hkv, 2, d] (minima, maxima), exponents int8 [pages, Hkv]."""

    def __init__(self, codes, exponents):
        _expect_dense("PageSummary", torch.int8, codes, exponents)
        self.shape = shape = codes.shape
        if len(shape) != 4 or shape[2] != 2 or exponents.shape != shape[:2]:
            raise ValueError(f"PageSummary: codes {tuple(shape)} and exponents {tuple(exponents.shape)} do not belong together")
        self.codes, self.exponents = codes, exponents
        self.device = codes.get_device()

    @classmethod
    def create(cls, num_blocks: int, num_kv_heads: int, head_dim: int, device="cuda") -> "PageSummary":
        return cls(torch.zeros(num_blocks, num_kv_heads, 2, head_dim, dtype=torch.int8, device=device),
                   torch.zeros(num_blocks, num_kv_heads, dtype=torch.int8, device=device))


def _summary_args(where, k_cache, summary: PageSummary, k_scale, workspace) -> SummaryArgs:
    NB, Hkv, bs, d = k_cache.shape
    strides = k_cache.stride()
    codes = k_cache.dtype is torch.uint8
    if codes:
        _expect_dense(where, torch.uint8, k_cache)
        if k_scale is None or k_scale.numel() != Hkv:
            raise ValueError(f"{where}: a pool of codes comes with one k_scale per KV head")
        _expect_dense(where, torch.float32, k_scale)
    else:
        _expect(where, torch.bfloat16, k_cache)
        if strides[3] != 1:
            raise ValueError(f"{where}: head_dim has to be contiguous")
        if k_scale is not None:
            raise ValueError(f"{where}: k_scale belongs to a pool of codes")
    if workspace is not None:
        _expect_workspace(where, workspace)
    _expect_device(where, summary.device)
    if summary.shape != (NB, Hkv, 2, d):
        raise ValueError(f"{where}: a cache {tuple(k_cache.shape)} with summaries {tuple(summary.shape)}")
    return SummaryArgs(k_cache.data_ptr(), _ptr(k_scale), summary.codes.data_ptr(), summary.exponents.data_ptr(), Hkv, d, bs, NB,
                       1 if codes else 2, strides[0], strides[1], strides[2], _ptr(workspace))


def summarize_append(k_cache, summary: PageSummary, block_table, context_lens, cu_tokens=None, num_tokens: Optional[int] = None, k_scale=None,
                     workspace=None, stream=None, check: bool = True) -> int:
    """pdattn_summarize_append: summaries of the pages that the last cu_tokens[s + 1] - cu_tokens[s] tokens of every sequence filled (None:
    one token each).  num_tokens, needed with cu_tokens: cu_tokens[S], or more.  Not for drafted tokens (see tree_accept)."""
    where = "pdattn_summarize_append"
    _expect_dense(where, torch.int32, block_table, context_lens, cu_tokens)
    a = _summary_args(where, k_cache, summary, k_scale, workspace)
    S, MB = block_table.shape
    if context_lens.numel() != S or (cu_tokens is not None and cu_tokens.numel() != S + 1):
        raise ValueError(f"{where}: shapes do not belong together")
    if cu_tokens is None:
        num_tokens = S
    elif num_tokens is None:
        raise ValueError(f"{where}: num_tokens is needed with cu_tokens")
    st = lib().pdattn_summarize_append(ctypes.byref(a), block_table.data_ptr(), context_lens.data_ptr(), _ptr(cu_tokens), num_tokens, S, MB,
                                       _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def summarize_pages(k_cache, summary: PageSummary, pages, k_scale=None, workspace=None, stream=None, check: bool = True) -> int:
    """pdattn_summarize_pages: summaries of the pages of a list (int32; entries below 0 are passed over)."""
    where = "pdattn_summarize_pages"
    _expect_dense(where, torch.int32, pages)
    a = _summary_args(where, k_cache, summary, k_scale, workspace)
    st = lib().pdattn_summarize_pages(ctypes.byref(a), pages.data_ptr(), pages.numel(), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def select_workspace_size(num_seqs, num_kv_heads, max_blocks_per_seq) -> int:
    n = ctypes.c_size_t(0)
    st = lib().pdattn_select_workspace_size(num_seqs, num_kv_heads, max_blocks_per_seq, ctypes.byref(n))
    if st != OK:
        raise PdattnError(st, "pdattn_select_workspace_size")
    return n.value


def alloc_select_workspace(num_seqs, num_kv_heads, max_blocks_per_seq, device="cuda", stream=None):
    return _alloc(select_workspace_size(num_seqs, num_kv_heads, max_blocks_per_seq), device, stream)


def select_pages(q, summary: PageSummary, block_table, context_lens, selected, block_size: int, workspace, *, num_first: int = 1,
                 num_recent: int = 1, stream=None, check: bool = True) -> int:
    """pdattn_select_pages: selected (int32 [S, Hkv, K]) receives, per sequence and KV head, the pages the token q [S, Hq, d] is to see: the
    first num_first, the last num_recent and the best of the others by their summaries, ascending, -1 past the last."""
    where = "pdattn_select_pages"
    _expect_dense(where, torch.bfloat16, q)
    _expect_dense(where, torch.int32, block_table, context_lens, selected)
    _expect_workspace(where, workspace)
    _expect_device(where, summary.device)
    S, Hq, d = q.shape
    NB, Hkv, _, dim = summary.shape
    rows, MB = block_table.shape
    lists = selected.shape
    if rows != S or context_lens.numel() != S or len(lists) != 3 or lists[0] != S or lists[1] != Hkv or dim != d:
        raise ValueError(f"{where}: shapes do not belong together")
    a = SelectArgs(q.data_ptr(), summary.codes.data_ptr(), summary.exponents.data_ptr(), block_table.data_ptr(), context_lens.data_ptr(),
                   selected.data_ptr(), S, Hq, Hkv, d, block_size, MB, NB, lists[2], num_first, num_recent, workspace.data_ptr(),
                   workspace.numel())
    st = lib().pdattn_select_pages(ctypes.byref(a), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def _selected(where, call, q, a: Args, selected, scales, stream, check) -> int:
    _expect_dense(where, torch.int32, selected)
    if q.shape[0] != a.num_seqs or selected.dim() != 3 or tuple(selected.shape[:2]) != (a.num_seqs, a.num_kv_heads):
        raise ValueError(f"{where}: q {tuple(q.shape)} and selected {tuple(selected.shape)} for {a.num_seqs} sequences of {a.num_kv_heads} KV heads")
    st = call(ctypes.byref(a), selected.data_ptr(), selected.shape[2], *scales, _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def decode_selected(q, k_cache, v_cache, block_table, context_lens, selected, scale, out, workspace,
                    context_lens_host: Optional[np.ndarray] = None, stream=None, check: bool = True) -> int:
    """pdattn_decode_selected: decode_ex over the chosen pages of every sequence and KV head (selected int32 [S, Hkv, K])."""
    where = "pdattn_decode_selected"
    _expect_caches(where, k_cache, v_cache)
    a = _step_args(where, q, k_cache, v_cache, k_cache.stride()[:3], block_table, context_lens, scale, out, workspace,
                   context_lens_host)
    return _selected(where, lib().pdattn_decode_selected, q, a, selected, (), stream, check)


def decode_selected_fp8(q, k8, v8, k_scale, v_scale, block_table, context_lens, selected, scale, out, workspace,
                        context_lens_host: Optional[np.ndarray] = None, stream=None, check: bool = True) -> int:
    """pdattn_decode_selected_fp8: decode_selected over the e4m3 code pools of decode_fp8."""
    where = "pdattn_decode_selected_fp8"
    _expect_codes(where, k8, v8, k_scale, v_scale)
    a = _step_args(where, q, k8, v8, (0, 0, 0), block_table, context_lens, scale, out, workspace, context_lens_host)
    return _selected(where, lib().pdattn_decode_selected_fp8, q, a, selected, (k_scale.data_ptr(), v_scale.data_ptr()), stream, check)


class PagePool:
    """The books of a page pool (pdattn_page_pool): int32 device tensors ref_counts [num_blocks], free_list [num_blocks],
    free_count [1]."""

    def __init__(self, ref_counts, free_list, free_count):
        _expect_dense("PagePool", torch.int32, ref_counts, free_list, free_count)
        if free_list.numel() != ref_counts.numel() or free_count.numel() != 1:
            raise ValueError("PagePool: ref_counts and free_list have one entry per page, free_count has one")
        self.ref_counts, self.free_list, self.free_count = ref_counts, free_list, free_count
        self.num_blocks = ref_counts.numel()
        self.device = ref_counts.get_device()
        self.args = PoolArgs(ref_counts.data_ptr(), free_list.data_ptr(), free_count.data_ptr(), self.num_blocks)

    @classmethod
    def create(cls, num_blocks: int, device="cuda", stream=None) -> "PagePool":
        """A pool whose pages are all free."""
        pool = cls(*(torch.empty(n, dtype=torch.int32, device=device) for n in (num_blocks, num_blocks, 1)))
        st = lib().pdattn_pages_init(ctypes.byref(pool.args), _stream_ptr(stream))
        if st != OK:
            raise PdattnError(st, "pdattn_pages_init")
        return pool


def pages_workspace_size(num_blocks: int, num_seqs: int) -> int:
    n = ctypes.c_size_t(0)
    st = lib().pdattn_pages_workspace_size(num_blocks, num_seqs, ctypes.byref(n))
    if st != OK:
        raise PdattnError(st, "pdattn_pages_workspace_size")
    return n.value


def alloc_pages_workspace(num_blocks: int, num_seqs: int, device="cuda", stream=None):
    n = pages_workspace_size(num_blocks, num_seqs)
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    st = lib().pdattn_workspace_init(ws.data_ptr(), n, _stream_ptr(stream))
    if st != OK:
        raise PdattnError(st, "pdattn_workspace_init")
    return ws


def _pages_check(where, pool, workspace, block_table, context_lens, *lists):
    _expect_dense(where, torch.int32, block_table, context_lens, *lists)
    _expect_workspace(where, workspace)
    _expect_device(where, pool.device)
    if block_table.dim() != 2 or context_lens.numel() != block_table.shape[0]:
        raise ValueError(f"{where}: block_table [S, MB] and context_lens [S] do not belong together")


def pages_reserve(pool: PagePool, block_table, context_lens, new_tokens, block_size: int, workspace, stream=None,
                  check: bool = True) -> int:
    """pdattn_pages_reserve: pages for new_tokens[s] further tokens of every sequence; context_lens advances (in place)."""
    where = "pdattn_pages_reserve"
    _pages_check(where, pool, workspace, block_table, context_lens, new_tokens)
    S, MB = block_table.shape
    if new_tokens.numel() != S:
        raise ValueError(f"{where}: new_tokens has one entry per row")
    st = lib().pdattn_pages_reserve(ctypes.byref(pool.args), block_table.data_ptr(), context_lens.data_ptr(),
                                    new_tokens.data_ptr(), S, MB, block_size, workspace.data_ptr(), workspace.numel(),
                                    _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def pages_fork(pool: PagePool, block_table, context_lens, parents, children, copy_src, copy_dst, block_size: int,
               workspace, stream=None, check: bool = True) -> int:
    """pdattn_pages_fork: the empty rows children[i] become copies of the rows parents[i]; the partial pages to copy are
    written to (copy_src, copy_dst)."""
    where = "pdattn_pages_fork"
    _pages_check(where, pool, workspace, block_table, context_lens, parents, children, copy_src, copy_dst)
    n = parents.numel()
    if children.numel() != n or copy_src.numel() < n or copy_dst.numel() < n:
        raise ValueError(f"{where}: {n} parents, {children.numel()} children, room for {copy_src.numel()} and {copy_dst.numel()} copies")
    S, MB = block_table.shape
    st = lib().pdattn_pages_fork(ctypes.byref(pool.args), block_table.data_ptr(), context_lens.data_ptr(), parents.data_ptr(),
                                 children.data_ptr(), n, S, MB, block_size, copy_src.data_ptr(), copy_dst.data_ptr(),
                                 workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def pages_free(pool: PagePool, block_table, context_lens, seqs, block_size: int, workspace, stream=None,
               check: bool = True) -> int:
    """pdattn_pages_free: rows seqs give their pages back and become empty."""
    where = "pdattn_pages_free"
    _pages_check(where, pool, workspace, block_table, context_lens, seqs)
    S, MB = block_table.shape
    st = lib().pdattn_pages_free(ctypes.byref(pool.args), block_table.data_ptr(), context_lens.data_ptr(), seqs.data_ptr(),
                                 seqs.numel(), S, MB, block_size, workspace.data_ptr(), workspace.numel(),
                                 _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def pages_trim(pool: PagePool, block_table, context_lens, new_lens, block_size: int, workspace, stream=None,
               check: bool = True) -> int:
    """pdattn_pages_trim: row s is shortened to new_lens[s] tokens; the pages behind them go back."""
    where = "pdattn_pages_trim"
    _pages_check(where, pool, workspace, block_table, context_lens, new_lens)
    S, MB = block_table.shape
    if new_lens.numel() != S:
        raise ValueError(f"{where}: new_lens has one entry per row")
    st = lib().pdattn_pages_trim(ctypes.byref(pool.args), block_table.data_ptr(), context_lens.data_ptr(), new_lens.data_ptr(), S, MB,
                                 block_size, workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def pages_compact(pool: PagePool, block_table, context_lens, copy_src, copy_dst, block_size: int, workspace, stream=None,
                  check: bool = True) -> int:
    """pdattn_pages_compact: renumber the referenced pages densely; the moves are written to (copy_src, copy_dst)."""
    where = "pdattn_pages_compact"
    _pages_check(where, pool, workspace, block_table, context_lens, copy_src, copy_dst)
    if copy_src.numel() != copy_dst.numel():
        raise ValueError(f"{where}: copy_src and copy_dst have the same length")
    S, MB = block_table.shape
    st = lib().pdattn_pages_compact(ctypes.byref(pool.args), block_table.data_ptr(), context_lens.data_ptr(), S, MB, block_size,
                                    copy_src.data_ptr(), copy_dst.data_ptr(), copy_src.numel(), workspace.data_ptr(),
                                    workspace.numel(), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def pages_copy(k_cache, v_cache, copy_src, copy_dst, workspace=None, stream=None, check: bool = True) -> int:
    """pdattn_pages_copy: page copy_src[i] to page copy_dst[i] in both caches ([page, kv_head, slot, dim] bf16, or the
    uint8 code pools of decode_fp8)."""
    where = "pdattn_pages_copy"
    _expect_dense(where, torch.int32, copy_src, copy_dst)
    if workspace is not None:
        _expect_workspace(where, workspace)
    if copy_src.numel() != copy_dst.numel():
        raise ValueError(f"{where}: copy_src and copy_dst have the same length")
    NB, Hkv, bs, d = k_cache.shape
    if k_cache.dtype == torch.uint8:
        _expect_dense(where, torch.uint8, k_cache, v_cache)
        if tuple(v_cache.shape) != (NB, Hkv, d, bs):
            raise ValueError(f"{where}: code pools {tuple(k_cache.shape)} and {tuple(v_cache.shape)} do not belong together")
    else:
        _expect_caches(where, k_cache, v_cache)
    st = lib().pdattn_pages_copy(k_cache.data_ptr(), v_cache.data_ptr(), copy_src.data_ptr(), copy_dst.data_ptr(),
                                 copy_src.numel(), Hkv, d, bs, NB, k_cache.element_size(), *k_cache.stride()[:3],
                                 _ptr(workspace), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, where)
    return st


def stream_read_probe(src: torch.Tensor, sink: torch.Tensor, stream=None):
    st = lib().pdattn_stream_read_probe(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(),
                                        _stream_ptr(stream))
    if st != OK:
        raise PdattnError(st, "pdattn_stream_read_probe")


def bind(max_blocks_per_seq, num_blocks, workspace, context_lens_host: Optional[np.ndarray] = None):
    """pdattn_bind.  The caller keeps `workspace` and `context_lens_host` alive while bound."""
    hp = context_lens_host.ctypes.data if context_lens_host is not None else None
    st = lib().pdattn_bind(max_blocks_per_seq, num_blocks, workspace.data_ptr(), workspace.numel(), hp)
    if st != OK:
        raise PdattnError(st, "pdattn_bind")


def decode(q, k_cache, v_cache, block_table, context_lens, num_seqs, num_q_heads, num_kv_heads, head_dim,
           block_size, scale, out, stream=None, check: bool = True) -> int:
    """pdattn_decode (13-argument form, dense [NB, Hkv, bs, d] caches, uses the thread's binding)."""
    st = lib().pdattn_decode(q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(),
                             context_lens.data_ptr(), num_seqs, num_q_heads, num_kv_heads, head_dim, block_size,
                             float(scale), out.data_ptr(), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_decode")
    return st


def host_staging_size(num_seqs, num_q_heads, head_dim, max_blocks_per_seq) -> int:
    n = ctypes.c_size_t(0)
    st = lib().pdattn_host_staging_size(num_seqs, num_q_heads, head_dim, max_blocks_per_seq, ctypes.byref(n))
    if st != OK:
        raise PdattnError(st, "pdattn_host_staging_size")
    return n.value


def decode_host(q_host, block_table_host, context_lens_host, out_host, k_cache, v_cache, scale, staging, workspace,
                stream=None, check: bool = True) -> int:
    """pdattn_decode_host: q / block_table / context_lens / out are HOST tensors (pinned), caches on device."""
    S, Hq, d = q_host.shape
    NB, Hkv, bs, _ = k_cache.shape
    st = lib().pdattn_decode_host(q_host.data_ptr(), block_table_host.data_ptr(), context_lens_host.data_ptr(),
                                  out_host.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), S, Hq, Hkv, d, bs,
                                  block_table_host.shape[1], NB, float(scale), staging.data_ptr(), staging.numel(),
                                  workspace.data_ptr(), workspace.numel(), _stream_ptr(stream))
    if check and st != OK:
        raise PdattnError(st, "pdattn_decode_host")
    return st


class HostStep:
    """pdattn_decode_host for a decode loop that reuses its buffers: the engine rewrites q_host, block_table_host
    and context_lens_host in place every step and reads out_host after synchronising the stream.  The arguments
    are marshalled once, so a step is a single foreign call (argument marshalling only; same entry point, same
    results as decode_host)."""

    def __init__(self, q_host, block_table_host, context_lens_host, out_host, k_cache, v_cache, scale, staging,
                 workspace, stream=None):
        S, Hq, d = q_host.shape
        NB, Hkv, bs, _ = k_cache.shape
        self._keep = (q_host, block_table_host, context_lens_host, out_host, k_cache, v_cache, staging, workspace)
        vp, ci = ctypes.c_void_p, ctypes.c_int
        self._args = (vp(q_host.data_ptr()), vp(block_table_host.data_ptr()), vp(context_lens_host.data_ptr()),
                      vp(out_host.data_ptr()), vp(k_cache.data_ptr()), vp(v_cache.data_ptr()), ci(S), ci(Hq), ci(Hkv),
                      ci(d), ci(bs), ci(block_table_host.shape[1]), ci(NB), ctypes.c_float(float(scale)),
                      vp(staging.data_ptr()), ctypes.c_size_t(staging.numel()), vp(workspace.data_ptr()),
                      ctypes.c_size_t(workspace.numel()), vp(_stream_ptr(stream)))
        self._fn = lib().pdattn_decode_host

    def __call__(self, check: bool = True) -> int:
        st = self._fn(*self._args)
        if check and st != OK:
            raise PdattnError(st, "pdattn_decode_host")
        return st


def set_dynamic_spans(per_cta: int):
    st = lib().pdattn_set_dynamic_spans(per_cta)
    if st != OK:
        raise PdattnError(st, "pdattn_set_dynamic_spans")


def set_merge_mode(mode: int):
    """-1: default (1 for batches of long sequences with host lengths, else 2); 0: barrier merge + combine kernel; 1: chained merge + final merge of cut units inside the
    decode kernel; 2: chained merge + combine kernel."""
    st = lib().pdattn_set_merge_mode(mode)
    if st != OK:
        raise PdattnError(st, "pdattn_set_merge_mode")


def set_short_piece_path(mode: int):
    """-1: the short-piece kernel instantiation for batches below 1.5 tiles per unit on average (default); 0: never; 1: whenever
    it applies (chained merge, bf16 cache, at most 8 query rows per KV head, host lengths)."""
    st = lib().pdattn_set_short_piece_path(mode)
    if st != OK:
        raise PdattnError(st, "pdattn_set_short_piece_path")


def set_prefix_engine(engine: int):
    """-1: default (tcgen05); 0: warp-level MMAs; 1: tcgen05 with tensor-memory accumulators."""
    st = lib().pdattn_set_prefix_engine(engine)
    if st != OK:
        raise PdattnError(st, "pdattn_set_prefix_engine")


def set_host_zero_copy(mode: int):
    """-1 / 1: decode_host uses pinned, mapped q and out in place; 0: always through the staging copies."""
    st = lib().pdattn_set_host_zero_copy(mode)
    if st != OK:
        raise PdattnError(st, "pdattn_set_host_zero_copy")


def wait_limit_probe(workspace, limit_us: int, stream=None) -> int:
    """One warp waits limit_us microseconds on a barrier nothing arrives on, then raises the timeout bit."""
    return lib().pdattn_wait_limit_probe(workspace.data_ptr(), int(limit_us), _stream_ptr(stream))


def plan_host(context_lens_host, num_kv_heads, n_ctas, dynamic_per_cta=0, max_spans=None):
    """pdattn_plan_host -> (spans[n_spans + 1, 4], Plan).  Row i is (unit, tile, flat, 0); span i holds
    spans[i + 1, 2] - spans[i, 2] tiles.  Needs no GPU."""
    lens = np.ascontiguousarray(context_lens_host, dtype=np.int32)
    if max_spans is None:
        max_spans = n_ctas * 9
    spans = np.zeros((max_spans + 1, 4), dtype=np.int32)
    plan = Plan()
    st = lib().pdattn_plan_host(lens.ctypes.data if lens.size else None, lens.size, num_kv_heads, n_ctas,
                                dynamic_per_cta, max_spans, spans.ctypes.data, ctypes.byref(plan))
    if st != OK:
        raise PdattnError(st, "pdattn_plan_host")
    return spans[: plan.n_static + plan.n_dynamic + 1].copy(), plan


def check(workspace, stream=None) -> int:
    """pdattn_check: synchronises, returns OK / BAD_PAGE_INDEX / DEVICE_TIMEOUT and clears the word."""
    return lib().pdattn_check(workspace.data_ptr(), _stream_ptr(stream))


def last_launch_count() -> int:
    return lib().pdattn_last_launch_count()


def decode_workload(w, out=None, workspace=None, use_host_lens: bool = True, stream=None):
    """Convenience for tests and the benchmark: run one step on a workloads.Workload living on the GPU."""
    if out is None:
        out = torch.empty_like(w.q)
    if workspace is None:
        workspace = alloc_workspace(w.num_seqs, w.num_q_heads, w.num_kv_heads, w.head_dim, w.block_size,
                                    device=w.q.device)
    decode_ex(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, w.scale, out, workspace,
              context_lens_host=w.context_lens_host if use_host_lens else None, stream=stream)
    return out
