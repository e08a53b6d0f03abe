"""Thin ctypes binding of libfastkv_b200.so: argument marshalling only.

Function names mirror the C ABI (include/fastkv.h).  Tensors are torch CUDA tensors used purely
as device memory; every step of the path runs inside the library's kernels.  There is no CPU or
PyTorch fallback: if the library is missing or fails to load, importing the symbols raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

from . import build as _build

FASTKV_OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_DEVICE_TIMEOUT, ERR_DEVICE_INDEX = range(1, 7)
POOL_AVG, POOL_MAX = 0, 1
GROUP_THEN_POOL, POOL_THEN_GROUP = 0, 1
Q_FULL, Q_WINDOW = 0, 1
CACHE_BF16, CACHE_E4M3 = 0, 1
ROT_HALVES, ROT_ADJACENT = 0, 1

EXPORTS = ["fastkv_workspace_bytes", "fastkv_score", "fastkv_select_kv", "fastkv_select_tsp", "fastkv_select",
           "fastkv_compact", "fastkv_decode_attn_workspace_bytes", "fastkv_decode_attn", "fastkv_prefill_workspace_bytes",
           "fastkv_prefill_attention", "fastkv_paged_append", "fastkv_paged_attn_workspace_bytes", "fastkv_paged_attn",
           "fastkv_prefix_attn_workspace_bytes", "fastkv_prefix_attn",
           "fastkv_paged_weights", "fastkv_paged_evict_workspace_bytes", "fastkv_paged_evict",
           "fastkv_device_status", "fastkv_layer_host_arena_bytes",
           "fastkv_layer_host", "fastkv_score_static", "fastkv_score_static_status", "fastkv_debug_set",
           "fastkv_debug_kernel_time",
           "fastkv_status_string", "fastkv_last_error", "fastkv_kernel_launches"]
_INT_RETURNING = [n for n in EXPORTS if n not in ("fastkv_status_string", "fastkv_last_error",
                                                  "fastkv_kernel_launches")]


class FastKVError(RuntimeError):
    def __init__(self, status: int, where: str):
        lib = _load()
        text = lib.fastkv_status_string(status).decode()
        detail = lib.fastkv_last_error().decode()
        super().__init__("%s: %s (%d)%s" % (where, text, status, ": " + detail if detail else ""))
        self.status = status


class Shape(ctypes.Structure):
    """fastkv_shape"""
    _fields_ = [("batch", ctypes.c_int32), ("total_len", ctypes.c_int32), ("max_len", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("hidden_dim", ctypes.c_int32), ("window", ctypes.c_int32), ("pool_kernel", ctypes.c_int32),
                ("pool_mode", ctypes.c_int32), ("agg_order", ctypes.c_int32), ("force_window", ctypes.c_int32),
                ("q_layout", ctypes.c_int32), ("softmax_scale", ctypes.c_float),
                ("cu_seqlens", ctypes.c_void_p),
                ("q_stride_tok", ctypes.c_int64), ("q_stride_head", ctypes.c_int64),
                ("k_stride_tok", ctypes.c_int64), ("k_stride_head", ctypes.c_int64),
                ("v_stride_tok", ctypes.c_int64), ("v_stride_head", ctypes.c_int64),
                ("hidden_stride_tok", ctypes.c_int64)]


class Budget(ctypes.Structure):
    """fastkv_budget"""
    _fields_ = [("k", ctypes.c_int32), ("total", ctypes.c_int32), ("cu_k", ctypes.c_void_p)]


class PagedCache(ctypes.Structure):
    """fastkv_paged_cache"""
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("format", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p), ("k_scales", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("block_table", ctypes.c_void_p)]
    _device = _index = None             # where its tensors are (make_paged_cache)


class NewRows(ctypes.Structure):
    """fastkv_new_rows"""
    _fields_ = [("total", ctypes.c_int32), ("max_new", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("rot_pairs", ctypes.c_int32), ("total_src", ctypes.c_int32),
                ("cu_new", ctypes.c_void_p), ("cu_src", ctypes.c_void_p),
                ("q_stride_tok", ctypes.c_int64), ("q_stride_head", ctypes.c_int64),
                ("k_stride_tok", ctypes.c_int64), ("k_stride_head", ctypes.c_int64),
                ("v_stride_tok", ctypes.c_int64), ("v_stride_head", ctypes.c_int64)]


class Query(ctypes.Structure):
    """fastkv_query"""
    _fields_ = [("n_q_heads", ctypes.c_int32), ("q_len", ctypes.c_int32), ("max_len", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("total_len", ctypes.c_int64)]


class Prefix(ctypes.Structure):
    """fastkv_prefix"""
    _fields_ = [("n_prefixes", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("max_len", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("cu_seqs", ctypes.c_void_p)]
    _device = None                      # where its tensors are (make_prefix)


class Eviction(ctypes.Structure):
    """fastkv_eviction"""
    _fields_ = [("keep", ctypes.c_int32), ("limit", ctypes.c_int32), ("window", ctypes.c_int32), ("max_len", ctypes.c_int32)]


_lib = None


def _load():
    global _lib
    if _lib is None:
        path = _build.LIB_PATH
        if not os.path.exists(path):
            raise RuntimeError("libfastkv_b200.so is not built; run `python -m paper_2502_01068_b200.build` "
                               "(there is no fallback path)")
        lib = ctypes.CDLL(path)
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        ps, pb = ctypes.POINTER(Shape), ctypes.POINTER(Budget)
        lib.fastkv_workspace_bytes.argtypes = [ps, ctypes.POINTER(sz)]
        lib.fastkv_score.argtypes = [ps, vp, vp, vp, vp, vp, sz, vp]
        lib.fastkv_select_kv.argtypes = [ps, vp, pb, vp, vp, sz, vp]
        lib.fastkv_select_tsp.argtypes = [ps, vp, pb, vp, vp, sz, vp]
        lib.fastkv_select.argtypes = [ps, vp, pb, vp, vp, pb, vp, vp, sz, vp]
        lib.fastkv_compact.argtypes = [ps, vp, pb, vp, pb, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.fastkv_device_status.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
        lib.fastkv_layer_host_arena_bytes.argtypes = [ps, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(sz)]
        lib.fastkv_layer_host.argtypes = [ps, ctypes.c_int32, ctypes.c_int32] + [vp] * 12 + [sz, vp]
        lib.fastkv_status_string.argtypes = [ctypes.c_int]
        lib.fastkv_status_string.restype = ctypes.c_char_p
        lib.fastkv_last_error.restype = ctypes.c_char_p
        lib.fastkv_kernel_launches.restype = ctypes.c_int64
        lib.fastkv_score_static.argtypes = [ps, vp, vp, vp, vp, vp]
        lib.fastkv_decode_attn_workspace_bytes.argtypes = [ps, ctypes.POINTER(sz)]
        lib.fastkv_decode_attn.argtypes = [ps, vp, vp, vp, pb, vp, vp, vp, sz, vp]
        lib.fastkv_prefill_workspace_bytes.argtypes = [ps, ctypes.POINTER(sz)]
        lib.fastkv_prefill_attention.argtypes = [ps, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        pc, pn, pq = ctypes.POINTER(PagedCache), ctypes.POINTER(NewRows), ctypes.POINTER(Query)
        lib.fastkv_paged_append.argtypes = [pc, pn] + [vp] * 10 + [sz, vp]
        lib.fastkv_paged_attn_workspace_bytes.argtypes = [pc, pq, ctypes.POINTER(sz)]
        lib.fastkv_paged_attn.argtypes = [pc, pq, vp, vp, vp, vp, vp, sz, vp]
        px = ctypes.POINTER(Prefix)
        lib.fastkv_prefix_attn_workspace_bytes.argtypes = [pc, px, pq, ctypes.POINTER(sz)]
        lib.fastkv_prefix_attn.argtypes = [pc, px, pq, vp, vp, vp, vp, vp, sz, vp]
        pv = ctypes.POINTER(Eviction)
        lib.fastkv_paged_weights.argtypes = [pc, pq, vp, vp, vp, ctypes.c_float, vp, ctypes.c_int64, vp, sz, vp]
        lib.fastkv_paged_evict_workspace_bytes.argtypes = [pc, pv, ctypes.POINTER(sz)]
        lib.fastkv_paged_evict.argtypes = [pc, pv, vp, vp, vp, ctypes.c_int64, vp, vp, vp, vp, sz, vp]
        lib.fastkv_score_static_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
        lib.fastkv_debug_set.argtypes = [ctypes.c_char_p, ctypes.c_int64]
        lib.fastkv_debug_kernel_time.argtypes = [ctypes.c_int32, ctypes.POINTER(ctypes.c_double),
                                                 ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_char_p)]
        for fn in _INT_RETURNING:
            getattr(lib, fn).restype = ctypes.c_int
        _lib = lib
    return _lib


def library_path() -> str:
    return _build.LIB_PATH


def _p(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        return t.data_ptr()
    return t.ctypes.data          # numpy array (host entry points)


def _stream(stream) -> Optional[int]:
    if stream is None:
        # the current stream's handle without building a Stream object (3.2 us of a call's 10 on the host)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) or None
    return stream.cuda_stream or None


def _check(rc: int, where: str) -> None:
    if rc != FASTKV_OK:
        raise FastKVError(rc, where)


def make_shape(*, total_len: int, n_q_heads: int, n_kv_heads: int, head_dim: int, hidden_dim: int = 0,
               window: int = 8, pool_kernel: int = 7, pool_mode: int = POOL_AVG,
               agg_order: int = GROUP_THEN_POOL, force_window: bool = True, q_layout: int = Q_WINDOW,
               softmax_scale: float = 0.0, batch: int = 1, max_len: Optional[int] = None,
               cu_seqlens=None, q_stride_tok: Optional[int] = None, q_stride_head: Optional[int] = None,
               k_stride_tok: Optional[int] = None, k_stride_head: Optional[int] = None,
               v_stride_tok: Optional[int] = None, v_stride_head: Optional[int] = None,
               hidden_stride_tok: Optional[int] = None) -> Shape:
    """Fill a fastkv_shape; strides default to dense [tokens, heads, head_dim] tensors."""
    s = Shape()
    s.batch, s.total_len, s.max_len = batch, total_len, total_len if max_len is None else max_len
    s.n_q_heads, s.n_kv_heads, s.head_dim, s.hidden_dim = n_q_heads, n_kv_heads, head_dim, hidden_dim
    s.window, s.pool_kernel, s.pool_mode, s.agg_order = window, pool_kernel, pool_mode, agg_order
    s.force_window, s.q_layout, s.softmax_scale = int(force_window), q_layout, softmax_scale
    s.cu_seqlens = _p(cu_seqlens)
    s._keep_alive = cu_seqlens          # the struct only holds the address: the tensor must outlive it
    s.q_stride_head = head_dim if q_stride_head is None else q_stride_head
    s.q_stride_tok = n_q_heads * head_dim if q_stride_tok is None else q_stride_tok
    s.k_stride_head = head_dim if k_stride_head is None else k_stride_head
    s.k_stride_tok = n_kv_heads * head_dim if k_stride_tok is None else k_stride_tok
    s.v_stride_head = head_dim if v_stride_head is None else v_stride_head
    s.v_stride_tok = n_kv_heads * head_dim if v_stride_tok is None else v_stride_tok
    s.hidden_stride_tok = hidden_dim if hidden_stride_tok is None else hidden_stride_tok
    return s


def make_budget(k: int = 0, *, batch: int = 1, cu_k=None, total: Optional[int] = None) -> Budget:
    b = Budget()
    b.k = k
    b.cu_k = _p(cu_k)
    b._keep_alive = cu_k                # the struct only holds the address: the tensor must outlive it
    b.total = (k * batch) if total is None else total
    return b


def fastkv_workspace_bytes(shape: Shape) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().fastkv_workspace_bytes(ctypes.byref(shape), ctypes.byref(n)), "fastkv_workspace_bytes")
    return int(n.value)


def fastkv_score(shape: Shape, q, k, scores_kv, scores_tsp, workspace, stream=None) -> None:
    _check(_load().fastkv_score(ctypes.byref(shape), _p(q), _p(k), _p(scores_kv), _p(scores_tsp), _p(workspace),
                                workspace.numel() * workspace.element_size(), _stream(stream)), "fastkv_score")


def fastkv_select_kv(shape: Shape, scores_kv, budget: Budget, idx_kv, workspace, stream=None) -> None:
    _check(_load().fastkv_select_kv(ctypes.byref(shape), _p(scores_kv), ctypes.byref(budget), _p(idx_kv),
                                    _p(workspace), workspace.numel() * workspace.element_size(),
                                    _stream(stream)), "fastkv_select_kv")


def fastkv_select_tsp(shape: Shape, scores_tsp, budget: Budget, idx_tsp, workspace, stream=None) -> None:
    _check(_load().fastkv_select_tsp(ctypes.byref(shape), _p(scores_tsp), ctypes.byref(budget), _p(idx_tsp),
                                     _p(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(stream)), "fastkv_select_tsp")


def fastkv_select(shape: Shape, scores_kv, kv: Budget, idx_kv, scores_tsp, tsp: Budget, idx_tsp, workspace,
                  stream=None) -> None:
    _check(_load().fastkv_select(ctypes.byref(shape), _p(scores_kv), ctypes.byref(kv), _p(idx_kv), _p(scores_tsp),
                                 ctypes.byref(tsp), _p(idx_tsp), _p(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)), "fastkv_select")


def fastkv_compact(shape: Shape, idx_kv, kv: Optional[Budget], idx_tsp, tsp: Optional[Budget], k, v, hidden,
                   pos_ids, k_out, v_out, hidden_out, pos_out, workspace, stream=None) -> None:
    _check(_load().fastkv_compact(ctypes.byref(shape), _p(idx_kv), ctypes.byref(kv) if kv else None,
                                  _p(idx_tsp), ctypes.byref(tsp) if tsp else None, _p(k), _p(v), _p(hidden),
                                  _p(pos_ids), _p(k_out), _p(v_out), _p(hidden_out), _p(pos_out),
                                  _p(workspace), workspace.numel() * workspace.element_size(),
                                  _stream(stream)), "fastkv_compact")


def fastkv_decode_attn_workspace_bytes(shape: Shape) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().fastkv_decode_attn_workspace_bytes(ctypes.byref(shape), ctypes.byref(n)),
           "fastkv_decode_attn_workspace_bytes")
    return int(n.value)


def fastkv_decode_attn(shape: Shape, q, k_cache, v_cache, kv: Budget, out, lse, workspace, stream=None) -> None:
    _check(_load().fastkv_decode_attn(ctypes.byref(shape), _p(q), _p(k_cache), _p(v_cache), ctypes.byref(kv), _p(out),
                                      _p(lse), _p(workspace), workspace.numel() * workspace.element_size(),
                                      _stream(stream)), "fastkv_decode_attn")


def fastkv_prefill_workspace_bytes(shape: Shape) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().fastkv_prefill_workspace_bytes(ctypes.byref(shape), ctypes.byref(n)), "fastkv_prefill_workspace_bytes")
    return int(n.value)


def fastkv_prefill_attention(shape: Shape, q, k, v, out, scores_kv, scores_tsp, workspace, stream=None) -> None:
    _check(_load().fastkv_prefill_attention(ctypes.byref(shape), _p(q), _p(k), _p(v), _p(out), _p(scores_kv),
                                            _p(scores_tsp), _p(workspace), workspace.numel() * workspace.element_size(),
                                            _stream(stream)), "fastkv_prefill_attention")


def _page_format(pages: torch.Tensor) -> int:
    if pages.dtype in (torch.bfloat16, torch.int16):
        return CACHE_BF16
    if pages.dtype in (torch.float8_e4m3fn, torch.uint8):
        return CACHE_E4M3
    raise TypeError("pages are bf16 (bfloat16, int16) or 8-bit (float8_e4m3fn, uint8), not %s" % pages.dtype)


def make_paged_cache(k_pages, v_pages, block_table, k_scales=None, v_scales=None) -> PagedCache:
    """Fill a fastkv_paged_cache from its tensors: pools [n_pages, n_kv_heads, page_size, head_dim], block_table int32
    [batch, max_pages], and for 8-bit pages the scales, fp32 [n_pages, n_kv_heads].  All dense, on one device."""
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype:
        raise ValueError("k_pages and v_pages are [n_pages, n_kv_heads, page_size, head_dim], alike")
    if block_table.dim() != 2 or block_table.dtype != torch.int32:
        raise ValueError("block_table is int32 [batch, max_pages]")
    fmt = _page_format(k_pages)
    for s in (k_scales, v_scales):
        if (s is not None) != (fmt == CACHE_E4M3):
            raise ValueError("k_scales and v_scales go with 8-bit pages and only with them")
        if s is not None and (s.dtype != torch.float32 or s.shape != k_pages.shape[:2]):
            raise ValueError("scales are float32 [n_pages, n_kv_heads]")
    parts = [x for x in (k_pages, v_pages, block_table, k_scales, v_scales) if x is not None]
    if any(not x.is_contiguous() for x in parts) or any(x.device != k_pages.device for x in parts):
        raise ValueError("the cache's tensors must be dense and on one device")
    c = PagedCache()
    c.batch, c.max_pages = block_table.shape
    c.n_pages, c.n_kv_heads, c.page_size, c.head_dim = k_pages.shape
    c.format = fmt
    c.k_pages, c.v_pages, c.block_table = _p(k_pages), _p(v_pages), _p(block_table)
    c.k_scales, c.v_scales = _p(k_scales), _p(v_scales)
    c._keep_alive = parts               # the struct only holds addresses: the tensors must outlive it
    c._device = k_pages.device
    c._index = k_pages.device.index
    return c


def make_new_rows(*, batch: int, total: int, n_kv_heads: int, head_dim: int, max_new: Optional[int] = None, cu_new=None,
                  n_q_heads: int = 0, rot_dim: int = 0, rot_pairs: int = ROT_HALVES, total_src: int = 0, cu_src=None,
                  q_stride_tok: Optional[int] = None, q_stride_head: Optional[int] = None,
                  k_stride_tok: Optional[int] = None, k_stride_head: Optional[int] = None,
                  v_stride_tok: Optional[int] = None, v_stride_head: Optional[int] = None) -> NewRows:
    """Fill a fastkv_new_rows; strides default to dense [rows, heads, head_dim] tensors, max_new to an even share (the whole
    call when cu_new is given)."""
    r = NewRows()
    r.total = total
    r.max_new = max_new if max_new is not None else (total if cu_new is not None else total // batch)
    r.n_q_heads, r.rot_dim, r.rot_pairs, r.total_src = n_q_heads, rot_dim, rot_pairs, total_src
    r.cu_new, r.cu_src = _p(cu_new), _p(cu_src)
    r._keep_alive = (cu_new, cu_src)    # the struct only holds addresses: the tensors must outlive it
    r.q_stride_head = head_dim if q_stride_head is None else q_stride_head
    r.q_stride_tok = n_q_heads * head_dim if q_stride_tok is None else q_stride_tok
    r.k_stride_head = head_dim if k_stride_head is None else k_stride_head
    r.k_stride_tok = n_kv_heads * head_dim if k_stride_tok is None else k_stride_tok
    r.v_stride_head = head_dim if v_stride_head is None else v_stride_head
    r.v_stride_tok = n_kv_heads * head_dim if v_stride_tok is None else v_stride_tok
    return r


def make_query(*, n_q_heads: int, max_len: int, q_len: int = 1, total_len: int = 0, softmax_scale: float = 0.0) -> Query:
    """Fill a fastkv_query."""
    q = Query()
    q.n_q_heads, q.q_len, q.max_len, q.softmax_scale, q.total_len = n_q_heads, q_len, max_len, softmax_scale, total_len
    return q


def _here(cache: PagedCache) -> int:
    """The current device, on which the library launches: a cache that lives on another one is refused."""
    dev = torch._C._cuda_getDevice()
    if cache._index != dev:
        raise ValueError("the cache is on %s, the current device is cuda:%d" % (cache._device, dev))
    return dev


# The two calls of a decode step marshal their arguments in line: on the host a call costs as much as its kernels take for
# small batches.
def fastkv_paged_append(cache: PagedCache, rows: NewRows, lens, q, k, v, pos, inv_freq, idx, q_out, new_lens, workspace,
                        stream=None) -> None:
    """Append rows to the paged cache (new tokens, rotated by their positions, or the rows that idx names); see the header."""
    dev = _here(cache)
    rc = (_lib or _load()).fastkv_paged_append(
        cache, rows, None if lens is None else lens.data_ptr(), None if q is None else q.data_ptr(),
        None if k is None else k.data_ptr(), None if v is None else v.data_ptr(), None if pos is None else pos.data_ptr(),
        None if inv_freq is None else inv_freq.data_ptr(), None if idx is None else idx.data_ptr(),
        None if q_out is None else q_out.data_ptr(), None if new_lens is None else new_lens.data_ptr(), workspace.data_ptr(),
        workspace.nbytes, torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    if rc != FASTKV_OK:
        raise FastKVError(rc, "fastkv_paged_append")


def fastkv_paged_attn_workspace_bytes(cache: PagedCache, query: Query) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().fastkv_paged_attn_workspace_bytes(ctypes.byref(cache), ctypes.byref(query), ctypes.byref(n)),
           "fastkv_paged_attn_workspace_bytes")
    return int(n.value)


def fastkv_paged_attn(cache: PagedCache, query: Query, lens, q, out, lse, workspace, stream=None) -> None:
    """Attention of query.q_len new tokens per sequence over the paged cache; see the header."""
    dev = _here(cache)
    rc = (_lib or _load()).fastkv_paged_attn(
        cache, query, None if lens is None else lens.data_ptr(), None if q is None else q.data_ptr(),
        None if out is None else out.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes,
        torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    if rc != FASTKV_OK:
        raise FastKVError(rc, "fastkv_paged_attn")


def make_prefix(table, lens, *, max_len: int, cu_seqs=None) -> Prefix:
    """Fill a fastkv_prefix: table int32 [n_prefixes, max_pages], lens int32 [n_prefixes], cu_seqs int32 [n_prefixes + 1] (not needed
    with one prefix that all sequences share).  All dense, on the cache's device."""
    if table.dim() != 2 or table.dtype != torch.int32:
        raise ValueError("table is int32 [n_prefixes, max_pages]")
    n = table.shape[0]
    for x, size, name in ((lens, n, "lens"), (cu_seqs, n + 1, "cu_seqs")):
        if x is not None and (x.dtype != torch.int32 or x.dim() != 1 or x.shape[0] != size):
            raise ValueError("%s is int32 [%d]" % (name, size))
    parts = [x for x in (table, lens, cu_seqs) if x is not None]
    if any(not x.is_contiguous() or x.device != table.device for x in parts):
        raise ValueError("the prefix's tensors must be dense and on one device")
    p = Prefix()
    p.n_prefixes, p.max_pages = table.shape
    p.max_len, p.table, p.lens, p.cu_seqs = max_len, _p(table), _p(lens), _p(cu_seqs)
    p._keep_alive = parts               # the struct only holds addresses: the tensors must outlive it
    p._device = table.device
    return p


def fastkv_prefix_attn_workspace_bytes(cache: PagedCache, prefix: Prefix, query: Query) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().fastkv_prefix_attn_workspace_bytes(ctypes.byref(cache), ctypes.byref(prefix), ctypes.byref(query), ctypes.byref(n)),
           "fastkv_prefix_attn_workspace_bytes")
    return int(n.value)


def fastkv_prefix_attn(cache: PagedCache, prefix: Prefix, query: Query, lens, q, out, lse, workspace, stream=None) -> None:
    """Attention of query.q_len new tokens per sequence over shared prefixes and the sequences' own entries; see the header."""
    dev = _here(cache)
    if prefix._device != cache._device:
        raise ValueError("the prefix is on %s, the cache on %s" % (prefix._device, cache._device))
    rc = (_lib or _load()).fastkv_prefix_attn(
        cache, prefix, query, None if lens is None else lens.data_ptr(), None if q is None else q.data_ptr(),
        None if out is None else out.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes,
        torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    if rc != FASTKV_OK:
        raise FastKVError(rc, "fastkv_prefix_attn")


def _entry_rows(cache: PagedCache, x, dtype, name: str):
    """Weights or ids: dense [batch, n_kv_heads, stride], on the cache's device."""
    if x.dim() != 3 or x.shape[0] != cache.batch or x.shape[1] != cache.n_kv_heads or x.dtype != dtype:
        raise ValueError("%s: %s [batch, n_kv_heads, stride]" % (name, dtype))
    if not x.is_contiguous() or x.device != cache._device:
        raise ValueError("%s must be dense and on the cache's device" % name)


def fastkv_paged_weights(cache: PagedCache, query: Query, lens, q, lse, decay: float, weights, workspace, stream=None) -> None:
    """Add the attention weight that query.q_len new tokens per sequence give each entry to decay * weights; see the header."""
    dev = _here(cache)
    _entry_rows(cache, weights, torch.float32, "weights")
    rc = (_lib or _load()).fastkv_paged_weights(
        cache, query, None if lens is None else lens.data_ptr(), None if q is None else q.data_ptr(),
        None if lse is None else lse.data_ptr(), decay, weights.data_ptr(), weights.shape[2], workspace.data_ptr(), workspace.nbytes,
        torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    if rc != FASTKV_OK:
        raise FastKVError(rc, "fastkv_paged_weights")


def make_eviction(*, keep: int, max_len: int, limit: Optional[int] = None, window: int = 8) -> Eviction:
    """Fill a fastkv_eviction; limit defaults to keep."""
    v = Eviction()
    v.keep, v.limit, v.window, v.max_len = keep, keep if limit is None else limit, window, max_len
    return v


def fastkv_paged_evict_workspace_bytes(cache: PagedCache, eviction: Eviction) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().fastkv_paged_evict_workspace_bytes(ctypes.byref(cache), ctypes.byref(eviction), ctypes.byref(n)),
           "fastkv_paged_evict_workspace_bytes")
    return int(n.value)


def fastkv_paged_evict(cache: PagedCache, eviction: Eviction, lens, weights, ids, new_weights, new_ids, new_lens, workspace,
                       stream=None) -> None:
    """Cut sequences of more than eviction.limit entries to eviction.keep, by weight, in place; see the header."""
    dev = _here(cache)
    _entry_rows(cache, weights, torch.float32, "weights")
    for x, dtype, name in ((new_weights, torch.float32, "new_weights"), (ids, torch.int32, "ids"), (new_ids, torch.int32, "new_ids")):
        if x is not None:
            _entry_rows(cache, x, dtype, name)
            if x.shape != weights.shape:
                raise ValueError("%s is shaped like weights" % name)
    rc = (_lib or _load()).fastkv_paged_evict(
        cache, eviction, None if lens is None else lens.data_ptr(), weights.data_ptr(), None if ids is None else ids.data_ptr(),
        weights.shape[2], None if new_weights is None else new_weights.data_ptr(), None if new_ids is None else new_ids.data_ptr(),
        None if new_lens is None else new_lens.data_ptr(), workspace.data_ptr(), workspace.nbytes,
        torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    if rc != FASTKV_OK:
        raise FastKVError(rc, "fastkv_paged_evict")


def fastkv_device_status(workspace, stream=None):
    status, site = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(_load().fastkv_device_status(_p(workspace), _stream(stream), ctypes.byref(status),
                                        ctypes.byref(site)), "fastkv_device_status")
    return int(status.value), int(site.value)


def fastkv_layer_host_arena_bytes(shape: Shape, k_kv: int, k_tsp: int) -> int:
    n = ctypes.c_size_t(0)
    _check(_load().fastkv_layer_host_arena_bytes(ctypes.byref(shape), k_kv, k_tsp, ctypes.byref(n)),
           "fastkv_layer_host_arena_bytes")
    return int(n.value)


def fastkv_layer_host(shape: Shape, k_kv: int, k_tsp: int, q, k, v, hidden, pos_ids, idx_kv, idx_tsp, k_out,
                      v_out, hidden_out, pos_out, arena, stream=None) -> None:
    """Host-buffer layer step: q..pos_out are host tensors/arrays, `arena` is a device tensor."""
    _check(_load().fastkv_layer_host(ctypes.byref(shape), k_kv, k_tsp, _p(q), _p(k), _p(v), _p(hidden),
                                     _p(pos_ids), _p(idx_kv), _p(idx_tsp), _p(k_out), _p(v_out),
                                     _p(hidden_out), _p(pos_out), _p(arena),
                                     arena.numel() * arena.element_size(), _stream(stream)),
           "fastkv_layer_host")


def fastkv_score_static(shape: Shape, q, k, scores_kv, scores_tsp, stream=None) -> None:
    """fastkv_score without a workspace argument: the scratch is a fixed 16 MiB array inside the
    library, for callers that cannot allocate device memory.  Shapes that need more raise
    FastKVError(ERR_WORKSPACE).  Calls on one device share the array: do not overlap them.
    fastkv_score_static_status() reads the device status word the call left behind."""
    _check(_load().fastkv_score_static(ctypes.byref(shape), _p(q), _p(k), _p(scores_kv), _p(scores_tsp),
                                       _stream(stream)), "fastkv_score_static")


def fastkv_score_static_status(stream=None):
    """(status, site) left by the last fastkv_score_static call on the current device."""
    status, site = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(_load().fastkv_score_static_status(_stream(stream), ctypes.byref(status), ctypes.byref(site)),
           "fastkv_score_static_status")
    return int(status.value), int(site.value)


def fastkv_debug_set(key: str, value: int) -> None:
    """Test and tuning hooks of the library (process-wide); see include/fastkv.h for the keys."""
    _check(_load().fastkv_debug_set(key.encode(), int(value)), "fastkv_debug_set")


def fastkv_debug_kernel_time(kernel: int):
    """(name, total milliseconds, launches) recorded for one kernel class while the "time_kernels" hook was on."""
    ms, n, name = ctypes.c_double(0.0), ctypes.c_int64(0), ctypes.c_char_p()
    _check(_load().fastkv_debug_kernel_time(kernel, ctypes.byref(ms), ctypes.byref(n), ctypes.byref(name)),
           "fastkv_debug_kernel_time")
    return name.value.decode(), float(ms.value), int(n.value)


def fastkv_status_string(status: int) -> str:
    return _load().fastkv_status_string(status).decode()


def fastkv_last_error() -> str:
    return _load().fastkv_last_error().decode()


def fastkv_kernel_launches() -> int:
    return int(_load().fastkv_kernel_launches())
