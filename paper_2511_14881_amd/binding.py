"""Thin Python face of the C-ABI library (``include/silvertorch.h``): the same entry points,
argument marshalling only.  PyTorch supplies device memory and the stream; every step of the
retrieval path runs inside the library's HIP kernels.  There is no fallback: if the shared
library has not been built, the first call raises."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "csrc", "libsilvertorch.so")
_lib = None

ST_OK, ST_EINVAL, ST_ENOMEM, ST_EHIP, ST_EWORKSPACE = 0, -1, -2, -3, -4

EXPORTS = [
    "st_last_error", "st_version", "st_bloom_build", "st_bloom_free", "st_bloom_trim", "st_bloom_bytes",
    "st_bloom_layout_bytes", "st_bloom_n_items", "st_bloom_export_signatures", "st_bloom_mask",
    "st_search_workspace_bytes", "st_search", "st_search_multitask", "st_score_pairs",
    "st_search_plan", "st_set_scoring_path", "st_timing_begin", "st_timing_end",
    "st_search_overflow_flags_offset", "st_bloom_mask_expr", "st_search_expr_workspace_bytes",
    "st_search_expr", "st_search_ivf_workspace_bytes", "st_search_ivf", "st_quantize_global", "st_value_model",
    "st_search_host_plan", "st_search_host_units", "st_stream_read", "st_search_static",
    "st_kv_append", "st_kv_read", "st_kv_attend_workspace_bytes", "st_kv_attend", "st_kv_select_workspace_bytes",
    "st_kv_select", "st_kv_evict", "st_kv_host_plan",
]

ST_OP_LEAF, ST_OP_AND, ST_OP_OR, ST_OP_NOT = 0, 1, 2, 3  # operations of a filter program


class StError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"silvertorch error {code}: {msg}")
        self.code = code


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        L = C.CDLL(LIB_PATH)
        p, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.st_last_error.restype = C.c_char_p
        L.st_last_error.argtypes = []
        L.st_version.restype = i32
        L.st_bloom_build.restype = C.c_int
        L.st_bloom_build.argtypes = [p, p, i64, i32, i32, p, C.POINTER(p)]
        L.st_bloom_free.restype = C.c_int
        L.st_bloom_free.argtypes = [p]
        L.st_bloom_trim.restype = C.c_int
        L.st_bloom_trim.argtypes = []
        L.st_bloom_bytes.restype = i64
        L.st_bloom_bytes.argtypes = [p]
        L.st_bloom_layout_bytes.restype = i64
        L.st_bloom_layout_bytes.argtypes = [i64, i32]
        L.st_bloom_n_items.restype = i64
        L.st_bloom_n_items.argtypes = [p]
        L.st_bloom_export_signatures.restype = C.c_int
        L.st_bloom_export_signatures.argtypes = [p, p, p]
        L.st_bloom_mask.restype = C.c_int
        L.st_bloom_mask.argtypes = [p, p, p, i32, p, p]
        L.st_search_workspace_bytes.restype = i64
        L.st_search_workspace_bytes.argtypes = [i64, i32, i32, i32, i32]
        L.st_search_overflow_flags_offset.restype = i64
        L.st_search_overflow_flags_offset.argtypes = [i64, i32, i32, i32, i32]
        L.st_search.restype = C.c_int
        L.st_search.argtypes = [p, p, p, i64, i32, p, p, i32, p, p, i32, p, p, p, p, i64, p]
        L.st_search_static.restype = C.c_int
        L.st_search_static.argtypes = [p, p, p, i64, i32, p, p, i32, p, p, i32, p, p, p, p]
        L.st_search_multitask.restype = C.c_int
        L.st_search_multitask.argtypes = [p, p, p, i64, i32, p, p, i32, i32, p, p, p, i32, p, p, p, p,
                                          i64, p]
        L.st_score_pairs.restype = C.c_int
        L.st_score_pairs.argtypes = [p, p, i32, p, p, p, p, i64, p, p, p]
        L.st_search_plan.restype = i32
        L.st_search_plan.argtypes = [i64, i32, i32, i32, p, i32, p]
        L.st_set_scoring_path.restype = i32
        L.st_set_scoring_path.argtypes = [i32]
        L.st_timing_begin.restype = C.c_int
        L.st_timing_begin.argtypes = [i32]
        L.st_timing_end.restype = C.c_int
        L.st_timing_end.argtypes = [p, p]
        L.st_bloom_mask_expr.restype = C.c_int
        L.st_bloom_mask_expr.argtypes = [p, p, p, p, i32, p, p]
        L.st_search_expr_workspace_bytes.restype = i64
        L.st_search_expr_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i64]
        L.st_search_expr.restype = C.c_int
        L.st_search_expr.argtypes = [p, p, p, i64, i32, p, p, i32, i32, p, p, p, p, i32, p, p, p, p, i64, p]
        L.st_search_ivf_workspace_bytes.restype = i64
        L.st_search_ivf_workspace_bytes.argtypes = [i64, i32, i32, i32, i32, i32, i64]
        L.st_search_ivf.restype = C.c_int
        L.st_search_ivf.argtypes = [p, p, p, i64, i32, p, p, p, i32, i32, p, p, i32, p, p, p, i32, p, p, p, p, p,
                                    i64, p]
        L.st_value_model.restype = C.c_int
        L.st_value_model.argtypes = [p, i64, i32, p, p, i32, p, p]
        L.st_search_host_plan.restype = C.c_int
        L.st_search_host_plan.argtypes = [i64, i32, i32, i32, i32, i32, i32, p, p, p]
        L.st_search_host_units.restype = C.c_int
        L.st_search_host_units.argtypes = [i64, i32, i32, i32, i32, i32, i32, i32, p, p, p]
        L.st_stream_read.restype = C.c_int
        L.st_stream_read.argtypes = [p, i64, p, i32, p]
        L.st_quantize_global.restype = C.c_int
        L.st_quantize_global.argtypes = [p, i64, i32, p, p, p, p, p]
        L.st_kv_append.restype = C.c_int
        L.st_kv_append.argtypes = [p, p, p, i64, p, i64, i32, p]
        L.st_kv_read.restype = C.c_int
        L.st_kv_read.argtypes = [p, p, i32, p, p, p, p]
        L.st_kv_attend_workspace_bytes.restype = i64
        L.st_kv_attend_workspace_bytes.argtypes = [p, p, i32, i32, i32]
        L.st_kv_attend.restype = C.c_int
        L.st_kv_attend.argtypes = [p, p, p, i64, i32, i32, C.c_float, i32, p, i32, p, i32, p, p, p, C.c_float, p, p, i64, p]
        L.st_kv_select_workspace_bytes.restype = i64
        L.st_kv_select_workspace_bytes.argtypes = [p, p, i32, i32]
        L.st_kv_select.restype = C.c_int
        L.st_kv_select.argtypes = [p, p, p, i64, i32, i32, i32, p, i32, i32, i32, i32, p, p, i64, p]
        L.st_kv_host_plan.restype = C.c_int
        L.st_kv_host_plan.argtypes = [p, p, i32, i32, i32, p]
        L.st_kv_evict.restype = C.c_int
        L.st_kv_evict.argtypes = [p, p, i32, i32, i32, i32, p, p, p, p, p, p]
        _lib = L
    return _lib


def last_error() -> str:
    return lib().st_last_error().decode()


def _check(rc: int) -> int:
    if rc < 0:
        raise StError(int(rc), last_error())
    return int(rc)


def _dptr(t: torch.Tensor | None):
    return None if t is None else C.c_void_p(t.data_ptr())


def _hptr(a: np.ndarray | None):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _stream(stream) -> C.c_void_p:
    s = stream if stream is not None else torch.cuda.current_stream()
    return C.c_void_p(s.cuda_stream)


def _on(stream, call, *args):
    """call(*args) on a stream that need not be the current one: what it allocates is that stream's, so that nothing of it is handed
    out before the work there is done, and its results are kept for the current stream too."""
    here = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        got = call(*args)
    for t in got if isinstance(got, tuple) else (got,):
        t.record_stream(here)
    return got


def _need(t: torch.Tensor, dtype, name: str):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{name} must be a contiguous CUDA tensor of {dtype}")


def _filters(filt_ids, filt_offsets, n: int):
    ids = np.ascontiguousarray(np.asarray(filt_ids, dtype=np.uint64))
    off = np.ascontiguousarray(np.asarray(filt_offsets, dtype=np.int64))
    if off.size != n + 1:
        raise ValueError("filt_offsets must have one more entry than there are filters")
    if off[-1] != ids.size:
        raise ValueError("filt_offsets[-1] must equal len(filt_ids)")
    return ids, off


class BloomIndex:
    """Owns an ``st_bloom*``."""

    def __init__(self, handle: int, n_items: int, m_bits: int, k_hashes: int):
        self.handle, self.n_items, self.m_bits, self.k_hashes = handle, n_items, m_bits, k_hashes

    @property
    def nbytes(self) -> int:
        return _check(lib().st_bloom_bytes(C.c_void_p(self.handle)))

    def free(self):
        if self.handle:
            _check(lib().st_bloom_free(C.c_void_p(self.handle)))
            self.handle = 0

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def st_bloom_build(feat_offsets, feat_ids, n_items: int, m_bits: int, k_hashes: int,
                   stream=None) -> BloomIndex:
    """feat_offsets int64 [N+1] and feat_ids (int64 bit patterns of uint64) as CUDA tensors or
    numpy arrays."""
    keep = []

    def ptr(x, np_dtype):
        if isinstance(x, torch.Tensor) and x.is_cuda:
            if x.dtype != torch.int64 or not x.is_contiguous():
                raise TypeError("feature tensors must be contiguous int64")
            keep.append(x)
            return _dptr(x)
        a = x.numpy() if isinstance(x, torch.Tensor) else np.asarray(x)
        if a.dtype not in (np.dtype(np.int64), np.dtype(np.uint64)):
            a = a.astype(np_dtype)
        a = np.ascontiguousarray(a).view(np_dtype)
        keep.append(a)
        return _hptr(a)

    out = C.c_void_p()
    _check(lib().st_bloom_build(ptr(feat_offsets, np.int64), ptr(feat_ids, np.uint64), n_items, m_bits,
                                k_hashes, _stream(stream), C.byref(out)))
    return BloomIndex(out.value, n_items, m_bits, k_hashes)


def st_bloom_trim() -> None:
    """Gives the memory that freed indexes left with the library back to the driver."""
    _check(lib().st_bloom_trim())


def st_bloom_layout_bytes(n_items: int, m_bits: int) -> int:
    return _check(lib().st_bloom_layout_bytes(n_items, m_bits))


def st_bloom_export_signatures(bloom: BloomIndex, stream=None) -> torch.Tensor:
    if stream is not None:
        return _on(stream, st_bloom_export_signatures, bloom)
    words = (bloom.m_bits + 63) // 64
    out = torch.empty((bloom.n_items, words), dtype=torch.int64, device="cuda")
    _check(lib().st_bloom_export_signatures(C.c_void_p(bloom.handle), _dptr(out), _stream(stream)))
    return out


def st_bloom_mask(bloom: BloomIndex, filt_ids, filt_offsets, stream=None) -> torch.Tensor:
    if stream is not None:
        return _on(stream, st_bloom_mask, bloom, filt_ids, filt_offsets)
    n_f = len(filt_offsets) - 1
    ids, off = _filters(filt_ids, filt_offsets, n_f)
    out = torch.zeros((n_f, (bloom.n_items + 63) // 64), dtype=torch.int64, device="cuda")
    _check(lib().st_bloom_mask(C.c_void_p(bloom.handle), _hptr(ids), _hptr(off), n_f, _dptr(out),
                               _stream(stream)))
    return out


def st_search_workspace_bytes(n_items: int, d: int, batch: int, n_tasks: int, K: int) -> int:
    return _check(lib().st_search_workspace_bytes(n_items, d, batch, n_tasks, K))


def st_search_overflow_flags_offset(n_items: int, d: int, batch: int, n_tasks: int, K: int) -> int:
    return _check(lib().st_search_overflow_flags_offset(n_items, d, batch, n_tasks, K))


def st_search_plan(n_items: int, batch: int, K: int, q_split: int = 1):
    levels = np.zeros((32, 3), dtype=np.int64)
    caps = np.zeros(2, dtype=np.int64)
    n = _check(lib().st_search_plan(n_items, batch, K, q_split, _hptr(levels), 32, _hptr(caps)))
    return levels[:n].copy(), int(caps[0]), int(caps[1])


def st_search_host_plan(n_items: int, d: int, batch: int, n_tasks: int, K: int, m_bits: int, k_hashes: int,
                        filt_ids, filt_offsets) -> dict:
    """The host part of a search alone (no GPU): a summary of the groups and the schedule."""
    ids, off = _filters(filt_ids, filt_offsets, batch)
    out = np.zeros(8, dtype=np.int32)
    _check(lib().st_search_host_plan(n_items, d, batch, n_tasks, K, m_bits, k_hashes, _hptr(ids), _hptr(off),
                                     _hptr(out)))
    keys = ("distinct_filters", "mfma_groups", "dot_groups", "q_split", "waves", "levels", "table_bytes", "seed_pass")
    return {k: int(v) for k, v in zip(keys, out)}


def st_search_host_units(n_items: int, d: int, batch: int, n_tasks: int, weighted: bool, K: int, m_bits: int, k_hashes: int,
                         filt_ids, filt_offsets) -> tuple[int, int]:
    """(passing pairs of the first level from which on the last one is scanned by units, -1: never; all its pairs)."""
    ids, off = _filters(filt_ids, filt_offsets, batch)
    out = np.zeros(2, dtype=np.int64)
    _check(lib().st_search_host_units(n_items, d, batch, n_tasks, int(weighted), K, m_bits, k_hashes, _hptr(ids), _hptr(off),
                                      _hptr(out)))
    return int(out[0]), int(out[1])


def st_set_scoring_path(path: int) -> int:
    return int(lib().st_set_scoring_path(path))


def st_timing_begin(max_launches: int) -> None:
    _check(lib().st_timing_begin(max_launches))


def st_timing_end():
    """{'scan'|'select'|'rescue'|'expr': (total_ms, launches)}"""
    ms = np.zeros(4, dtype=np.float64)
    n = np.zeros(4, dtype=np.int64)
    _check(lib().st_timing_end(_hptr(ms), _hptr(n)))
    return {k: (float(ms[i]), int(n[i])) for i, k in enumerate(("scan", "select", "rescue", "expr"))}


class SearchBuffers:
    """Workspace and outputs for repeated searches of one shape.  n_expr_entries: room for filter
    programs of that many entries per batch (st_search_expr); None for the plain searches."""

    def __init__(self, n_items: int, d: int, batch: int, n_tasks: int, K: int, n_expr_entries: int | None = None):
        if n_expr_entries is None:
            self.nbytes = st_search_workspace_bytes(n_items, d, batch, n_tasks, K)
        else:
            self.nbytes = _check(lib().st_search_expr_workspace_bytes(n_items, d, batch, n_tasks, K, n_expr_entries))
        self._ovf = (st_search_overflow_flags_offset(n_items, d, batch, n_tasks, K), batch)
        self.workspace = torch.empty(self.nbytes, dtype=torch.uint8, device="cuda")
        self.ids = torch.empty((batch, K), dtype=torch.int64, device="cuda")
        self.scores = torch.empty((batch, K), dtype=torch.float32, device="cuda")
        self.count = torch.empty(batch, dtype=torch.int32, device="cuda")

    def overflow_flags(self):
        """int32 [batch] view: 1 where the last search on these buffers had to recompute the query
        by the slow exact path (read after the stream has synchronised)."""
        off, batch = self._ovf
        return self.workspace[off:off + 4 * batch].view(torch.int32)


def st_search(bloom: BloomIndex, items, item_scale, queries, query_scale, filt_ids, filt_offsets,
              K: int, buffers: SearchBuffers | None = None, stream=None):
    if stream is not None and buffers is None:
        return _on(stream, st_search, bloom, items, item_scale, queries, query_scale, filt_ids, filt_offsets, K)
    _need(items, torch.int8, "items")
    _need(item_scale, torch.float32, "item_scale")
    _need(queries, torch.int8, "queries")
    _need(query_scale, torch.float32, "query_scale")
    n, d = items.shape
    B = queries.shape[0]
    if queries.dim() != 2 or queries.shape[1] != d or query_scale.numel() != B or item_scale.numel() != n:
        raise ValueError("shape mismatch")
    ids, off = _filters(filt_ids, filt_offsets, B)
    buf = buffers or SearchBuffers(n, d, B, 1, K)
    _check(lib().st_search(C.c_void_p(bloom.handle), _dptr(items), _dptr(item_scale), n, d, _dptr(queries),
                           _dptr(query_scale), B, _hptr(ids), _hptr(off), K, _dptr(buf.ids),
                           _dptr(buf.scores), _dptr(buf.count), _dptr(buf.workspace), buf.nbytes,
                           _stream(stream)))
    return buf.ids, buf.scores, buf.count


ST_STATIC_SCRATCH_BYTES = 80 << 20


def st_search_static(bloom: BloomIndex, items, item_scale, queries, query_scale, filt_ids, filt_offsets,
                     K: int, out=None, stream=None):
    """st_search on the library's own fixed workspace (no allocation inside the call).  out: the
    (ids, scores, count) tensors to fill; allocated here, outside the library, if not given."""
    if stream is not None and out is None:
        return _on(stream, st_search_static, bloom, items, item_scale, queries, query_scale, filt_ids, filt_offsets, K)
    _need(items, torch.int8, "items")
    _need(item_scale, torch.float32, "item_scale")
    _need(queries, torch.int8, "queries")
    _need(query_scale, torch.float32, "query_scale")
    n, d = items.shape
    B = queries.shape[0]
    if queries.dim() != 2 or queries.shape[1] != d or query_scale.numel() != B or item_scale.numel() != n:
        raise ValueError("shape mismatch")
    ids, off = _filters(filt_ids, filt_offsets, B)
    if out is None:
        out = (torch.empty((B, K), dtype=torch.int64, device="cuda"),
               torch.empty((B, K), dtype=torch.float32, device="cuda"),
               torch.empty(B, dtype=torch.int32, device="cuda"))
    _check(lib().st_search_static(C.c_void_p(bloom.handle), _dptr(items), _dptr(item_scale), n, d, _dptr(queries),
                                  _dptr(query_scale), B, _hptr(ids), _hptr(off), K, _dptr(out[0]), _dptr(out[1]),
                                  _dptr(out[2]), _stream(stream)))
    return out


def st_search_multitask(bloom: BloomIndex, items, item_scale, queries, query_scale, task_weight,
                        filt_ids, filt_offsets, K: int, buffers: SearchBuffers | None = None,
                        stream=None):
    if stream is not None and buffers is None:
        return _on(stream, st_search_multitask, bloom, items, item_scale, queries, query_scale, task_weight, filt_ids, filt_offsets, K)
    _need(items, torch.int8, "items")
    _need(item_scale, torch.float32, "item_scale")
    _need(queries, torch.int8, "queries")
    _need(query_scale, torch.float32, "query_scale")
    n, d = items.shape
    if queries.dim() != 3 or queries.shape[2] != d:
        raise ValueError("queries must be [B, T, d]")
    B, T = queries.shape[0], queries.shape[1]
    w = np.ascontiguousarray(np.asarray(task_weight, dtype=np.float32))
    if w.size != T or query_scale.numel() != B * T or item_scale.numel() != n:
        raise ValueError("shape mismatch")
    ids, off = _filters(filt_ids, filt_offsets, B)
    buf = buffers or SearchBuffers(n, d, B, T, K)
    _check(lib().st_search_multitask(C.c_void_p(bloom.handle), _dptr(items), _dptr(item_scale), n, d,
                                     _dptr(queries), _dptr(query_scale), B, T, _hptr(w), _hptr(ids),
                                     _hptr(off), K, _dptr(buf.ids), _dptr(buf.scores), _dptr(buf.count),
                                     _dptr(buf.workspace), buf.nbytes, _stream(stream)))
    return buf.ids, buf.scores, buf.count


def _programs(expr_ops, expr_ids, expr_offsets, n: int):
    ops = np.ascontiguousarray(np.asarray(expr_ops, dtype=np.int32))
    ids = np.asarray(expr_ids)
    if ids.dtype != np.dtype(np.uint64):
        ids = ids.astype(np.uint64)
    ids = np.ascontiguousarray(ids)
    off = np.ascontiguousarray(np.asarray(expr_offsets, dtype=np.int64))
    if off.size != n + 1 or ops.size != ids.size or (off.size and ops.size < off[-1]):
        raise ValueError("filter program arrays do not match their offsets")
    return ops, ids, off


def st_bloom_mask_expr(bloom: BloomIndex, expr_ops, expr_ids, expr_offsets, stream=None) -> torch.Tensor:
    if stream is not None:
        return _on(stream, st_bloom_mask_expr, bloom, expr_ops, expr_ids, expr_offsets)
    n_e = len(expr_offsets) - 1
    ops, ids, off = _programs(expr_ops, expr_ids, expr_offsets, n_e)
    out = torch.zeros((n_e, (bloom.n_items + 63) // 64), dtype=torch.int64, device="cuda")
    _check(lib().st_bloom_mask_expr(C.c_void_p(bloom.handle), _hptr(ops), _hptr(ids), _hptr(off), n_e,
                                    _dptr(out), _stream(stream)))
    return out


def st_search_expr_workspace_bytes(n_items: int, d: int, batch: int, n_tasks: int, K: int,
                                   n_expr_entries: int) -> int:
    return _check(lib().st_search_expr_workspace_bytes(n_items, d, batch, n_tasks, K, n_expr_entries))


def st_search_expr(bloom: BloomIndex, items, item_scale, queries, query_scale, expr_ops, expr_ids,
                   expr_offsets, K: int, task_weight=None, buffers: SearchBuffers | None = None, stream=None):
    """queries [B, d] (task_weight None) or [B, T, d] with T weights; query b's filter is program b."""
    if stream is not None and buffers is None:
        return _on(stream, st_search_expr, bloom, items, item_scale, queries, query_scale, expr_ops, expr_ids, expr_offsets, K,
                   task_weight)
    _need(items, torch.int8, "items")
    _need(item_scale, torch.float32, "item_scale")
    _need(queries, torch.int8, "queries")
    _need(query_scale, torch.float32, "query_scale")
    n, d = items.shape
    B = queries.shape[0]
    if task_weight is None:
        if queries.dim() != 2 or queries.shape[1] != d:
            raise ValueError("queries must be [B, d]")
        T, w = 1, None
    else:
        if queries.dim() != 3 or queries.shape[2] != d:
            raise ValueError("queries must be [B, T, d]")
        T = queries.shape[1]
        w = np.ascontiguousarray(np.asarray(task_weight, dtype=np.float32))
        if w.size != T:
            raise ValueError("shape mismatch")
    if query_scale.numel() != B * T or item_scale.numel() != n:
        raise ValueError("shape mismatch")
    ops, ids, off = _programs(expr_ops, expr_ids, expr_offsets, B)
    buf = buffers or SearchBuffers(n, d, B, T, K, n_expr_entries=int(off[-1]))
    _check(lib().st_search_expr(C.c_void_p(bloom.handle), _dptr(items), _dptr(item_scale), n, d, _dptr(queries),
                                _dptr(query_scale), B, T, None if w is None else _hptr(w), _hptr(ops),
                                _hptr(ids), _hptr(off), K, _dptr(buf.ids), _dptr(buf.scores), _dptr(buf.count),
                                _dptr(buf.workspace), buf.nbytes, _stream(stream)))
    return buf.ids, buf.scores, buf.count


def st_search_ivf_workspace_bytes(n_items: int, d: int, batch: int, K: int, n_clusters: int, n_probe: int,
                                  n_expr_entries: int) -> int:
    return _check(lib().st_search_ivf_workspace_bytes(n_items, d, batch, K, n_clusters, n_probe, n_expr_entries))


class IvfBuffers(SearchBuffers):
    """Workspace and outputs of st_search_ivf for one shape."""

    def __init__(self, n_items: int, d: int, batch: int, K: int, n_clusters: int, n_probe: int, n_expr_entries: int):
        super().__init__(n_items, d, batch, 1, K)
        self.nbytes = st_search_ivf_workspace_bytes(n_items, d, batch, K, n_clusters, n_probe, n_expr_entries)
        self.workspace = torch.empty(self.nbytes, dtype=torch.uint8, device="cuda")
        self.probes = torch.empty((batch, n_probe), dtype=torch.int32, device="cuda")


def st_search_ivf(bloom: BloomIndex, items, item_scale, centroids, centroid_scale, cluster_offsets, n_probe: int,
                  queries, query_scale, expr_ops, expr_ids, expr_offsets, K: int,
                  buffers: IvfBuffers | None = None, stream=None):
    """Returns (ids, scores, count, probes); cluster_offsets int64 [n_clusters + 1] on the device."""
    if stream is not None and buffers is None:
        return _on(stream, st_search_ivf, bloom, items, item_scale, centroids, centroid_scale, cluster_offsets, n_probe, queries,
                   query_scale, expr_ops, expr_ids, expr_offsets, K)
    _need(items, torch.int8, "items")
    _need(item_scale, torch.float32, "item_scale")
    _need(centroids, torch.int8, "centroids")
    _need(centroid_scale, torch.float32, "centroid_scale")
    _need(cluster_offsets, torch.int64, "cluster_offsets")
    _need(queries, torch.int8, "queries")
    _need(query_scale, torch.float32, "query_scale")
    n, d = items.shape
    n_c = centroids.shape[0]
    B = queries.shape[0]
    if (queries.dim() != 2 or queries.shape[1] != d or centroids.shape[1] != d or query_scale.numel() != B
            or item_scale.numel() != n or centroid_scale.numel() != n_c or cluster_offsets.numel() != n_c + 1):
        raise ValueError("shape mismatch")
    ops, ids, off = _programs(expr_ops, expr_ids, expr_offsets, B)
    buf = buffers or IvfBuffers(n, d, B, K, n_c, n_probe, int(off[-1]))
    _check(lib().st_search_ivf(C.c_void_p(bloom.handle), _dptr(items), _dptr(item_scale), n, d, _dptr(centroids),
                               _dptr(centroid_scale), _dptr(cluster_offsets), n_c, n_probe, _dptr(queries),
                               _dptr(query_scale), B, _hptr(ops), _hptr(ids), _hptr(off), K, _dptr(buf.ids),
                               _dptr(buf.scores), _dptr(buf.count), _dptr(buf.probes), _dptr(buf.workspace),
                               buf.nbytes, _stream(stream)))
    return buf.ids, buf.scores, buf.count, buf.probes


def st_stream_read(src: torch.Tensor, sink: torch.Tensor, workgroups: int, stream=None) -> None:
    """Bandwidth probe: reads all of src (any dtype, contiguous) once; sink int32/uint32 [workgroups]."""
    if not (src.is_cuda and src.is_contiguous() and sink.is_cuda and sink.numel() >= workgroups):
        raise TypeError("src must be a contiguous CUDA tensor and sink hold one word per workgroup")
    _check(lib().st_stream_read(_dptr(src), src.numel() * src.element_size(), _dptr(sink), workgroups, _stream(stream)))


def st_quantize_global(x, stream=None):
    """fp32 [N, d] CUDA tensor -> (int8 [N, d], row scales fp32 [N], minmax fp32 [2]) on the device."""
    if stream is not None:
        return _on(stream, st_quantize_global, x)
    _need(x, torch.float32, "x")
    if x.dim() != 2:
        raise ValueError("x must be [N, d]")
    n, d = x.shape
    q = torch.empty((n, d), dtype=torch.int8, device="cuda")
    rs = torch.empty(n, dtype=torch.float32, device="cuda")
    mm = torch.empty(2, dtype=torch.float32, device="cuda")
    scratch = torch.empty(2, dtype=torch.int32, device="cuda")
    _check(lib().st_quantize_global(_dptr(x), n, d, _dptr(q), _dptr(rs), _dptr(mm), _dptr(scratch), _stream(stream)))
    return q, rs, mm


def st_value_model(task_scores, ops, consts, out=None, stream=None):
    """task_scores fp32 [n, T] CUDA tensor; postfix formula (ops int32, consts fp32) -> fp32 [n]."""
    if stream is not None and out is None:
        return _on(stream, st_value_model, task_scores, ops, consts)
    _need(task_scores, torch.float32, "task_scores")
    if task_scores.dim() != 2:
        raise ValueError("task_scores must be [n, T]")
    n, T = task_scores.shape
    o = np.ascontiguousarray(np.asarray(ops, dtype=np.int32))
    c = np.ascontiguousarray(np.asarray(consts, dtype=np.float32))
    if o.size != c.size:
        raise ValueError("ops and consts differ in length")
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device="cuda")
    _check(lib().st_value_model(_dptr(task_scores), n, T, _hptr(o), _hptr(c), o.size, _dptr(out), _stream(stream)))
    return out


def st_score_pairs(items, item_scale, queries, query_scale, pair_item, pair_query, stream=None):
    if stream is not None:
        return _on(stream, st_score_pairs, items, item_scale, queries, query_scale, pair_item, pair_query)
    _need(items, torch.int8, "items")
    _need(queries, torch.int8, "queries")
    _need(pair_item, torch.int64, "pair_item")
    _need(pair_query, torch.int32, "pair_query")
    d = items.shape[1]
    q2 = queries.reshape(-1, d)
    n = pair_item.numel()
    dots = torch.empty(n, dtype=torch.int32, device="cuda")
    scores = torch.empty(n, dtype=torch.float32, device="cuda")
    _check(lib().st_score_pairs(_dptr(items), _dptr(item_scale), d, _dptr(q2), _dptr(query_scale.reshape(-1)),
                                _dptr(pair_item), _dptr(pair_query), n, _dptr(dots), _dptr(scores),
                                _stream(stream)))
    return dots, scores


# ------------------------------------------------------------------ cached histories

# The current stream as a number: torch.cuda.current_stream() builds an object first, which takes longer than a launch.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _kv_stream(stream):
    if stream is not None or _raw_stream is None or _raw_device is None:
        return _stream(stream)
    return _raw_stream(_raw_device())


ST_KV_BLOCK, ST_KV_MAX_BLOCKS, ST_KV_MAX_HEADS = 64, 16384, 1024
ST_BF16, ST_F16 = 0, 1
_KV_TYPES = {torch.bfloat16: ST_BF16, torch.float16: ST_F16}


class _KvCacheC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "bounds")] + [
        ("n_pages", C.c_int64), ("n_heads", C.c_int32), ("d", C.c_int32)]


class _KvBatchC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("tables", "lengths", "offsets")] + [
        (n, C.c_int32) for n in ("n_seq", "max_blocks", "n_tok", "max_tok", "max_len")]


class KvCache:
    """Pages of cached keys and values (``st_kv_cache``) on the tensors given: k int8 [pages, heads, 64, d],
    v int8 [pages, heads, d, 64] (in slot order), k_scale and v_scale fp32 [pages, heads], bounds int8 [pages, heads, 2, d]."""

    def __init__(self, k, v, k_scale, v_scale, bounds):
        for t, dtype, name in ((k, torch.int8, "k"), (v, torch.int8, "v"), (k_scale, torch.float32, "k_scale"),
                               (v_scale, torch.float32, "v_scale"), (bounds, torch.int8, "bounds")):
            _need(t, dtype, name)
        if k.dim() != 4:
            raise ValueError("k must be [pages, heads, 64, d]")
        n, h, b, d = k.shape
        if b != ST_KV_BLOCK or v.shape != (n, h, d, b) or k_scale.shape != (n, h) or v_scale.shape != (n, h) or bounds.shape != (n, h, 2, d):
            raise ValueError("shape mismatch")
        self.k, self.v, self.k_scale, self.v_scale, self.bounds = k, v, k_scale, v_scale, bounds
        self.n_pages, self.n_heads, self.d = n, h, d
        self._c = _KvCacheC(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), bounds.data_ptr(), n, h, d)
        self._p = C.cast(C.pointer(self._c), C.c_void_p)

    @classmethod
    def empty(cls, n_pages: int, n_heads: int, d: int, device="cuda") -> "KvCache":
        def new(shape, dtype):
            return torch.zeros(shape, dtype=dtype, device=device)
        return cls(new((n_pages, n_heads, ST_KV_BLOCK, d), torch.int8), new((n_pages, n_heads, d, ST_KV_BLOCK), torch.int8),
                   new((n_pages, n_heads), torch.float32), new((n_pages, n_heads), torch.float32),
                   new((n_pages, n_heads, 2, d), torch.int8))


class KvBatch:
    """The sequences of a call (``st_kv_batch``): tables int32 [n_seq, max_blocks], lengths int32 [n_seq] (the call's
    tokens included), n_tok tokens in all; offsets int32 [n_seq + 1] where sequences have different numbers of them, with
    max_tok a bound on one sequence's (n_tok if not given: a call of many sequences then takes work and workspace for n_seq * n_tok
    tokens, so give it where the counts are known).  max_len bounds the lengths (64 * max_blocks if not given)."""

    def __init__(self, tables, lengths, n_tok: int, offsets=None, max_tok: int | None = None, max_len: int | None = None):
        _need(tables, torch.int32, "tables")
        _need(lengths, torch.int32, "lengths")
        if tables.dim() != 2 or lengths.numel() != tables.shape[0]:
            raise ValueError("shape mismatch")
        n_seq, max_blocks = tables.shape
        if offsets is not None:
            _need(offsets, torch.int32, "offsets")
            if offsets.numel() != n_seq + 1:
                raise ValueError("offsets must have one more entry than there are sequences")
        if max_tok is None:
            max_tok = n_tok if offsets is not None else n_tok // max(n_seq, 1)
        if max_len is None:
            max_len = max_blocks * ST_KV_BLOCK
        self.tables, self.lengths, self.offsets = tables, lengths, offsets
        self.n_seq, self.max_blocks, self.n_tok, self.max_tok, self.max_len = n_seq, max_blocks, n_tok, max_tok, max_len
        self._c = _KvBatchC(tables.data_ptr(), lengths.data_ptr(), None if offsets is None else offsets.data_ptr(), n_seq,
                            max_blocks, n_tok, max_tok, max_len)
        self._p = C.cast(C.pointer(self._c), C.c_void_p)


def _kv_rows(t: torch.Tensor, n_tok: int, d: int, name: str):
    """Rows [n_tok, heads, d] of a 16-bit type, whole heads side by side; rows may be further apart."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in _KV_TYPES):
        raise TypeError(f"{name} must be a CUDA tensor of torch.bfloat16 or torch.float16")
    if t.dim() != 3 or t.shape[0] != n_tok or t.shape[2] != d:
        raise ValueError(f"{name} must be [{n_tok}, heads, {d}]")
    if t.stride(2) != 1 or (t.shape[1] > 1 and t.stride(1) != d):
        raise ValueError(f"the heads of a row of {name} must be contiguous")
    return t.stride(0) if n_tok > 1 else t.shape[1] * d, _KV_TYPES[t.dtype]


def _kv_mask(mask, n_tok: int):
    if mask is None:
        return None, 0
    _need(mask, torch.int64, "mask")
    if mask.dim() != 2 or mask.shape[0] != n_tok:
        raise ValueError("mask must be [n_tok, words]")
    return C.c_void_p(mask.data_ptr()), mask.shape[1]


def _kv_out(t, shape, dtype, name: str):
    _need(t, dtype, name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}")
    return t


class KvBuffers:
    """Workspace and outputs of repeated st_kv_attend and st_kv_select calls of one shape: queries like q; n_sel: room
    for that many selected blocks; mass: room for the blocks' weights."""

    def __init__(self, cache: KvCache, batch: KvBatch, q: torch.Tensor, n_sel: int = 0, mass: bool = False):
        n_q_heads = q.shape[1]
        self.nbytes = st_kv_attend_workspace_bytes(cache, batch, n_q_heads, n_sel, mass)
        self.out = torch.empty((batch.n_tok, n_q_heads, cache.d), dtype=q.dtype, device="cuda")
        self.blocks = self.mass = None
        if n_sel:
            self.nbytes = max(self.nbytes, st_kv_select_workspace_bytes(cache, batch, n_q_heads, n_sel))
            self.blocks = torch.empty((batch.n_tok, cache.n_heads, n_sel), dtype=torch.int32, device="cuda")
        if mass:
            self.mass = torch.empty((batch.n_seq, cache.n_heads, batch.max_blocks), dtype=torch.float32, device="cuda")
        self.workspace = torch.empty(self.nbytes, dtype=torch.uint8, device="cuda")


def st_kv_append(cache: KvCache, batch: KvBatch, k, v, stream=None) -> None:
    """Writes the batch's tokens (rows [n_tok, heads, d], bf16 or fp16) behind what the sequences held."""
    ks, dtype = _kv_rows(k, batch.n_tok, cache.d, "k")
    vs, v_dtype = _kv_rows(v, batch.n_tok, cache.d, "v")
    if dtype != v_dtype or k.shape[1] != cache.n_heads or v.shape[1] != cache.n_heads:
        raise ValueError("k and v must be of one type and have the cache's heads")
    _check(lib().st_kv_append(cache._p, batch._p, k.data_ptr(), ks, v.data_ptr(), vs, dtype, _kv_stream(stream)))


def st_kv_read(cache: KvCache, batch: KvBatch, n_blocks: int, stream=None):
    """The last n_blocks blocks of each sequence as fp32 (k, v [n_seq, n_blocks, heads, 64, d], bounds [.., 2, d])."""
    if stream is not None:
        return _on(stream, st_kv_read, cache, batch, n_blocks)
    shape = (batch.n_seq, n_blocks, cache.n_heads, ST_KV_BLOCK, cache.d)
    k = cache.k_scale.new_empty(shape)
    v = cache.k_scale.new_empty(shape)
    bounds = cache.k_scale.new_empty((*shape[:3], 2, cache.d))
    _check(lib().st_kv_read(cache._p, batch._p, n_blocks, k.data_ptr(), v.data_ptr(), bounds.data_ptr(), _kv_stream(stream)))
    return k, v, bounds


def st_kv_attend_workspace_bytes(cache: KvCache, batch: KvBatch, n_q_heads: int, n_sel: int = 0, mass: bool = False) -> int:
    return _check(lib().st_kv_attend_workspace_bytes(cache._p, batch._p, n_q_heads, n_sel, int(mass)))


def st_kv_attend(cache: KvCache, batch: KvBatch, q, scale: float | None = None, causal: bool = True, mask=None,
                 blocks=None, mass=None, decay: float = 1.0, mass_out=None, lse=None, out=None,
                 buffers: KvBuffers | None = None, stream=None) -> torch.Tensor:
    """Attention of q [n_tok, n_q_heads, d] over the cache; returns out, like q.  scale: 1 / sqrt(d) if not given.
    mask int64 [n_tok, words], a bit to a position; blocks int32 [n_tok, heads, n_sel] from st_kv_select.  The blocks'
    weights go to mass_out (or buffers.mass) where that or mass (the weights so far, times decay) is given; lse fp32
    [n_tok, n_q_heads] is filled where given."""
    if stream is not None:
        return _on(stream, st_kv_attend, cache, batch, q, scale, causal, mask, blocks, mass, decay, mass_out, lse, out, buffers)
    q_stride, dtype = _kv_rows(q, batch.n_tok, cache.d, "q")
    n_q_heads, n_sel = q.shape[1], 0
    mask_p, words = _kv_mask(mask, batch.n_tok)
    if blocks is not None:
        _need(blocks, torch.int32, "blocks")
        if blocks.dim() != 3 or blocks.shape[0] != batch.n_tok or blocks.shape[1] != cache.n_heads:
            raise ValueError("blocks must be [n_tok, heads, n_sel]")
        n_sel = blocks.shape[2]
    shape = (batch.n_seq, cache.n_heads, batch.max_blocks)
    if mass is not None:
        mass = _kv_out(mass, shape, torch.float32, "mass")
    with_mass = mass is not None or mass_out is not None
    if buffers is not None:
        out = buffers.out if out is None else out
        if with_mass and mass_out is None:
            mass_out = buffers.mass
        work, nbytes = buffers.workspace, buffers.nbytes
    else:
        nbytes = st_kv_attend_workspace_bytes(cache, batch, n_q_heads, n_sel, with_mass)
        work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    if out is None:
        out = q.new_empty((batch.n_tok, n_q_heads, cache.d))
    else:
        _kv_out(out, (batch.n_tok, n_q_heads, cache.d), q.dtype, "out")
    if with_mass:
        mass_out = torch.empty_like(mass) if mass_out is None else _kv_out(mass_out, shape, torch.float32, "mass_out")
    if lse is not None:
        lse = _kv_out(lse, (batch.n_tok, n_q_heads), torch.float32, "lse")
    _check(lib().st_kv_attend(cache._p, batch._p, q.data_ptr(), q_stride, dtype, n_q_heads,
                              cache.d ** -0.5 if scale is None else scale, int(causal), mask_p, words,
                              _dptr(blocks), n_sel, out.data_ptr(), _dptr(lse), _dptr(mass), decay, _dptr(mass_out),
                              work.data_ptr(), nbytes, _kv_stream(stream)))
    return out


def st_kv_select_workspace_bytes(cache: KvCache, batch: KvBatch, n_q_heads: int, n_sel: int) -> int:
    return _check(lib().st_kv_select_workspace_bytes(cache._p, batch._p, n_q_heads, n_sel))


def st_kv_select(cache: KvCache, batch: KvBatch, q, n_sel: int, causal: bool = True, mask=None, sink: int = 0,
                 recent: int = 0, out=None, buffers: KvBuffers | None = None, stream=None) -> torch.Tensor:
    """The n_sel blocks that each token and head of the cache reads: int32 [n_tok, heads, n_sel], ascending, -1 behind."""
    if stream is not None:
        return _on(stream, st_kv_select, cache, batch, q, n_sel, causal, mask, sink, recent, out, buffers)
    q_stride, dtype = _kv_rows(q, batch.n_tok, cache.d, "q")
    n_q_heads = q.shape[1]
    mask_p, words = _kv_mask(mask, batch.n_tok)
    if buffers is not None:
        out = buffers.blocks if out is None else out
        work, nbytes = buffers.workspace, buffers.nbytes
    else:
        nbytes = st_kv_select_workspace_bytes(cache, batch, n_q_heads, n_sel)
        work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    if out is None:
        out = batch.lengths.new_empty((batch.n_tok, cache.n_heads, n_sel))
    else:
        _kv_out(out, (batch.n_tok, cache.n_heads, n_sel), torch.int32, "out")
    _check(lib().st_kv_select(cache._p, batch._p, q.data_ptr(), q_stride, dtype, n_q_heads, int(causal), mask_p, words, n_sel,
                              sink, recent, out.data_ptr(), work.data_ptr(), nbytes, _kv_stream(stream)))
    return out


def st_kv_host_plan(cache: KvCache, batch: KvBatch, n_q_heads: int, n_sel: int = 0, mass: bool = False) -> dict:
    """How an attention and a selection of these sizes would run (no GPU work; see ``include/silvertorch.h``)."""
    out = np.zeros(10, dtype=np.int32)
    _check(lib().st_kv_host_plan(cache._p, batch._p, n_q_heads, n_sel, int(mass), _hptr(out)))
    keys = ("waves", "tiles", "chunk", "splits", "join_waves", "sum_lanes", "score_and_choose", "score_chunks", "score_rounds", "choose_keys")
    return {k: int(v) for k, v in zip(keys, out)}


def st_kv_evict(batch: KvBatch, mass, budget: int, sink: int = 0, recent: int = 1, out=None, stream=None):
    """Cuts each sequence to at most budget blocks by mass fp32 [n_seq, heads, max_blocks].  Returns (tables, lengths,
    mass, freed, n_freed); out: the tensors to fill, of which tables, lengths and mass may be the batch's own."""
    if stream is not None:
        return _on(stream, st_kv_evict, batch, mass, budget, sink, recent, out)
    _need(mass, torch.float32, "mass")
    if mass.dim() != 3 or mass.shape[0] != batch.n_seq or mass.shape[2] != batch.max_blocks:
        raise ValueError("mass must be [n_seq, heads, max_blocks]")
    if out is None:
        out = (torch.empty_like(batch.tables), torch.empty_like(batch.lengths), torch.empty_like(mass),
               torch.empty_like(batch.tables), torch.empty_like(batch.lengths))
    else:
        rows = (batch.n_seq, batch.max_blocks)
        for t, shape, dtype, name in zip(out, (rows, (batch.n_seq,), mass.shape, rows, (batch.n_seq,)),
                                         (torch.int32, torch.int32, torch.float32, torch.int32, torch.int32),
                                         ("tables", "lengths", "mass", "freed", "n_freed"), strict=True):
            _kv_out(t, shape, dtype, name)
    t, n, m, f, nf = out
    _check(lib().st_kv_evict(batch._p, mass.data_ptr(), mass.shape[1], budget, sink, recent, t.data_ptr(), n.data_ptr(),
                             m.data_ptr(), f.data_ptr(), nf.data_ptr(), _kv_stream(stream)))
    return out
