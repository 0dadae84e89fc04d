"""Thin ctypes binding of libhs.so with the C ABI's names.

Argument marshalling only: every function passes device pointers
(``tensor.data_ptr()``), sizes and the current torch CUDA stream to the
library and returns the tensors it wrote.  Workspaces and outputs are torch
allocations when the caller does not pass them.  Every step of the path runs
in the library's kernels; if the library cannot be built or loaded, these
functions raise instead of computing anything another way.
"""
from __future__ import annotations

import ctypes
import math
import os
import threading

import torch

from . import build as _build

HS_OK = 0
HS_ERR_INVALID_ARG = 1
HS_ERR_UNSUPPORTED = 2
HS_ERR_CUDA = 3
HS_ERR_WORKSPACE = 4
HS_ERR_TIMEOUT = 5
HS_FNV64_OFFSET_BASIS = 0xCBF29CE484222325
HS_TOPK_MAX_K = 1024
HS_MERGE_QUERIES_MAX = 256
HS_KV_E4M3 = 0
HS_KV_INT8 = 1
HS_KV_BF16 = 0
HS_KV_FP16 = 1
HS_KV_MAX_REQUESTS = 16384
HS_ROTARY_HALF = 0
HS_ROTARY_INTERLEAVED = 1
HS_SAMPLE_MAX_VOCAB = 524160

_STATUS = {0: "HS_OK", 1: "HS_ERR_INVALID_ARG", 2: "HS_ERR_UNSUPPORTED", 3: "HS_ERR_CUDA",
           4: "HS_ERR_WORKSPACE", 5: "HS_ERR_TIMEOUT"}

_lock = threading.Lock()
_lib = None


class HsError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("%s: %s" % (_STATUS.get(status, str(status)), msg))
        self.status = status


def library_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = True) -> ctypes.CDLL:
    """Load libhs.so (building it first if it is missing or stale)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if build_if_missing:
                _build.build()
            if not os.path.exists(_build.LIB):
                raise RuntimeError("libhs.so is missing: run paper_2607_22578_gb300.build.build()")
            lib = ctypes.CDLL(_build.LIB)
            P, i64, i32, u64, sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32,
                                    ctypes.c_uint64, ctypes.c_size_t)
            st = ctypes.c_int
            lib.hs_last_error.restype = ctypes.c_char_p
            lib.hs_version.restype = ctypes.c_char_p
            lib.hs_fingerprint.argtypes = [P, i64, i32, P, u64, P, P]
            lib.hs_fingerprint.restype = st
            lib.hs_unique_inverse_workspace.argtypes = [i64]
            lib.hs_unique_inverse_workspace.restype = sz
            lib.hs_unique_inverse.argtypes = [P, P, i64, i32, P, P, P, P, P, sz, P]
            lib.hs_unique_inverse.restype = st
            lib.hs_unique_inverse_noalloc.argtypes = [P, P, i64, i32, P, P, P, P, P]
            lib.hs_unique_inverse_noalloc.restype = st
            lib.hs_retrieve_topk_workspace.argtypes = [i64, i64, i32, i32]
            lib.hs_retrieve_topk_workspace.restype = sz
            lib.hs_retrieve_topk.argtypes = [P, i64, P, i64, i32, i32, P, P, P, sz, P]
            lib.hs_retrieve_topk.restype = st
            lib.hs_retrieve_topk_n.argtypes = [P, i64, P, P, i64, i32, i32, P, P, P, sz, P]
            lib.hs_retrieve_topk_n.restype = st
            lib.hs_retrieve_topk_fanout.argtypes = [P, i64, P, P, i64, P, i64, i32, i32, P, P,
                                                    P, sz, P]
            lib.hs_retrieve_topk_fanout.restype = st
            lib.hs_merge_queries.argtypes = [P, i64, i32, u64, P, P, P, P, P, P, P]
            lib.hs_merge_queries.restype = st
            lib.hs_rerank_topk.argtypes = [P, i64, P, P, i64, i32, P, i32, i32, P, i64, P, P, P]
            lib.hs_rerank_topk.restype = st
            lib.hs_cache_bytes.argtypes = [i64, i32, i32]
            lib.hs_cache_bytes.restype = sz
            lib.hs_cache_init.argtypes = [P, sz, i64, i32, i32, P]
            lib.hs_cache_init.restype = st
            lib.hs_cache_lookup.argtypes = [P, sz, i64, i32, i32, P, P, P, i64, P, P, P, P, P, P, P]
            lib.hs_cache_lookup.restype = st
            lib.hs_cache_insert.argtypes = [P, sz, i64, i32, i32, P, P, i64, P, P, P, P, P, P, P, P]
            lib.hs_cache_insert.restype = st
            lib.hs_cache_stats.argtypes = [P, P, P, P]
            lib.hs_cache_stats.restype = st
            lib.hs_segment_sum.argtypes = [P, P, i64, P, i64, P, P]
            lib.hs_segment_sum.restype = st
            lib.hs_scatter_results.argtypes = [P, i64, i64, P, i64, P, P]
            lib.hs_scatter_results.restype = st
            lib.hs_get_device_error.argtypes = [P]
            lib.hs_get_device_error.restype = st
            lib.hs_launch_count.restype = ctypes.c_uint64
            lib.hs_debug_scan_wait.argtypes = [u64, i64]
            lib.hs_debug_scan_wait.restype = st
            lib.hs_merge_rows_workspace.argtypes = [i64]
            lib.hs_merge_rows_workspace.restype = sz
            lib.hs_merge_rows.argtypes = [P, i64, i32, P, u64, P, P, P, P, P, sz, P]
            lib.hs_merge_rows.restype = st
            lib.hs_debug_merge_key_mask.argtypes = [u64]
            lib.hs_debug_merge_key_mask.restype = st
            lib.hs_debug_retrieve_wait.argtypes = [u64, i32]
            lib.hs_debug_retrieve_wait.restype = st
            lib.hs_memcpy_async.argtypes = [P, P, sz, P]
            lib.hs_memcpy_async.restype = st
            lib.hs_debug_stream_rows.argtypes = [P, i64, i32, P, i32, P, i32, P]
            lib.hs_debug_stream_rows.restype = st
            lib.hs_kv_tables.argtypes = [P, P, i64, P, i32, P, i32, P, i64, P, P, P, P, P, i64, P]
            lib.hs_kv_tables.restype = st
            lib.hs_kv_release.argtypes = [P, i64, P, i32, P, i32, P, i64, P, P, P]
            lib.hs_kv_release.restype = st
            lib.hs_kv_append.argtypes = [P, P, P, i32, i64, i64, i64, P, P]
            lib.hs_kv_append.restype = st
            lib.hs_kv_attend_workspace.argtypes = [i32, i32, i32, i32]
            lib.hs_kv_attend_workspace.restype = sz
            lib.hs_kv_attend.argtypes = [P, P, i32, i64, i32, i64, i64, P, P, i64, P, i32, P, i32,
                                         ctypes.c_float, i32, i32, P, P, P, sz, P]
            lib.hs_kv_attend.restype = st
            lib.hs_kv_fork.argtypes = [P, P, i64, P, P, i64, i32, P, i32, P, P, i64, P, P, P, P, P, P]
            lib.hs_kv_fork.restype = st
            lib.hs_kv_fork_n.argtypes = [P, P, i64, P, P, i64, P, P, i32, P, i32, P, P, i64, P, P, P, P, P, P]
            lib.hs_kv_fork_n.restype = st
            lib.hs_kv_copy.argtypes = [P, P, P, P, i64, P, P]
            lib.hs_kv_copy.restype = st
            lib.hs_kv_release_shared.argtypes = [P, i64, P, i32, P, i32, P, P, P, i64, P, P, P]
            lib.hs_kv_release_shared.restype = st
            lib.hs_kv_compact_workspace.argtypes = [i64]
            lib.hs_kv_compact_workspace.restype = sz
            lib.hs_kv_compact.argtypes = [P, i64, P, i32, P, P, i32, P, P, i64, P, P, P, P, P, P, sz, P]
            lib.hs_kv_compact.restype = st
            f64 = ctypes.c_double
            lib.hs_rotary_frequencies.argtypes = [f64, i32, f64, f64, f64, f64, P]
            lib.hs_rotary_frequencies.restype = st
            lib.hs_rotary.argtypes = [P, i64, i64, P, i64, i64, i32, i64, i32, i32, i32, i32, P,
                                      ctypes.c_float, i32, P, P, P, i64, P, P]
            lib.hs_rotary.restype = st
            lib.hs_sample.argtypes = [P, i32, i64, i64, i64, P, i64, P, P, P, P, P, P, P, P, P, P]
            lib.hs_sample.restype = st
            _lib = lib
    return _lib


def _check(status: int) -> None:
    if status != HS_OK:
        raise HsError(status, load().hs_last_error().decode())


# The current stream's handle without a Stream object: 0.2 us of a call's host
# time where torch.cuda.current_stream() takes 2.9.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _raw_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _on(stream, device):
    """What torch.cuda.stream takes for a call's ``stream``."""
    if stream is None or isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream), device=device)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _cuda(t: torch.Tensor, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t


def _rows(t: torch.Tensor, n: int) -> torch.Tensor:
    """The first n rows of t: t itself where it has no more."""
    return t if t.shape[0] == n else t[:n]


def hs_version() -> str:
    return load().hs_version().decode()


def hs_fingerprint(tokens: torch.Tensor, lens: torch.Tensor | None = None,
                   seed_state: int = HS_FNV64_OFFSET_BASIS, fp_out: torch.Tensor | None = None,
                   stream=None) -> torch.Tensor:
    """fp[i] = FNV-1a-64 over row i's little-endian token octets (int64 tensor
    holding the uint64 bit patterns)."""
    _cuda(tokens, "tokens")
    if tokens.dtype != torch.int32 or tokens.dim() != 2:
        raise TypeError("tokens must be a 2-D int32 tensor")
    n, stride = tokens.shape
    if lens is not None:
        _cuda(lens, "lens")
        if lens.dtype != torch.int32 or lens.numel() != n:
            raise TypeError("lens must be int32 [n_rows]")
    if fp_out is None:
        fp_out = torch.empty(n, dtype=torch.int64, device=tokens.device)
    _check(load().hs_fingerprint(_ptr(tokens), n, stride, _ptr(lens), seed_state & (2**64 - 1),
                                 _ptr(fp_out), _stream(stream)))
    return fp_out


def hs_unique_inverse_workspace(n_rows: int) -> int:
    return int(load().hs_unique_inverse_workspace(n_rows))


def hs_unique_inverse(fp: torch.Tensor, tokens: torch.Tensor, lens: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None, out: tuple | None = None,
                      stream=None):
    """Exact unique rows.  Returns (n_unique_dev [1] int32, unique_idx [n]
    int32, inverse [n] int32); only the first n_unique entries of unique_idx
    are meaningful."""
    _cuda(fp, "fp")
    _cuda(tokens, "tokens")
    n, stride = tokens.shape
    dev = tokens.device
    if out is None:
        out = (torch.empty(1, dtype=torch.int32, device=dev),
               torch.empty(max(n, 1), dtype=torch.int32, device=dev),
               torch.empty(max(n, 1), dtype=torch.int32, device=dev))
    nu, uidx, inv = out
    if workspace is None:
        workspace = torch.empty(hs_unique_inverse_workspace(n), dtype=torch.uint8, device=dev)
    _check(load().hs_unique_inverse(_ptr(fp), _ptr(tokens), n, stride, _ptr(lens), _ptr(nu),
                                    _ptr(uidx), _ptr(inv), _ptr(workspace), workspace.numel(),
                                    _stream(stream)))
    return nu, _rows(uidx, n), _rows(inv, n)


def hs_merge_rows_workspace(n_rows: int) -> int:
    return int(load().hs_merge_rows_workspace(int(n_rows)))


def hs_merge_rows(tokens: torch.Tensor, lens: torch.Tensor | None = None,
                  seed_state: int = HS_FNV64_OFFSET_BASIS, workspace: torch.Tensor | None = None,
                  out: tuple | None = None, stream=None):
    """Fingerprint and exact merge in one pass.  Returns (fp [n] int64 (uint64
    bits), n_unique_dev [1] int32, unique_idx [n] int32, inverse [n] int32);
    `out`, if given, is that tuple of preallocated tensors."""
    _cuda(tokens, "tokens")
    n, stride = tokens.shape
    dev = tokens.device
    if out is None:
        out = (torch.empty(max(n, 1), dtype=torch.int64, device=dev),
               torch.empty(1, dtype=torch.int32, device=dev),
               torch.empty(max(n, 1), dtype=torch.int32, device=dev),
               torch.empty(max(n, 1), dtype=torch.int32, device=dev))
    fp, nu, uidx, inv = out
    if workspace is None:
        workspace = torch.empty(hs_merge_rows_workspace(n), dtype=torch.uint8, device=dev)
    _check(load().hs_merge_rows(_ptr(tokens), n, stride, _ptr(lens), int(seed_state), _ptr(fp),
                                _ptr(nu), _ptr(uidx), _ptr(inv), _ptr(workspace),
                                workspace.numel(), _stream(stream)))
    return _rows(fp, n), nu, _rows(uidx, n), _rows(inv, n)


def hs_debug_merge_key_mask(mask: int = 0) -> None:
    """Test hook of hs_merge_rows: key the table by fp & mask (0 restores
    all ones; see hs.h)."""
    _check(load().hs_debug_merge_key_mask(int(mask)))


def hs_memcpy_async(dst: torch.Tensor, src: torch.Tensor, stream=None) -> torch.Tensor:
    """Copy src into dst (equal byte sizes, contiguous; host, pinned host or
    device on either side) on `stream` through the C ABI.  Returns dst."""
    if not dst.is_contiguous() or not src.is_contiguous():
        raise ValueError("dst and src must be contiguous")
    nbytes = dst.numel() * dst.element_size()
    if nbytes != src.numel() * src.element_size():
        raise ValueError("dst and src differ in size")
    if not (dst.is_cuda or src.is_cuda):
        raise ValueError("one side must be on the GPU")
    _check(load().hs_memcpy_async(ctypes.c_void_p(dst.data_ptr()), ctypes.c_void_p(src.data_ptr()),
                                  nbytes, _stream(stream)))
    return dst


def hs_debug_retrieve_wait(limit_ns: int = 0, withhold_first: int = 0) -> None:
    """Test hook of the retrieval's bounded waits: the wait limit (0: 2 s)
    and whether every CTA withholds its first stage (see hs.h)."""
    _check(load().hs_debug_retrieve_wait(int(limit_ns), int(withhold_first)))


def hs_unique_inverse_noalloc(fp: torch.Tensor, tokens: torch.Tensor,
                              lens: torch.Tensor | None = None, out: tuple | None = None,
                              stream=None):
    """hs_unique_inverse without a workspace, for callers that cannot
    allocate device memory (at most 65536 rows; the scratch is a fixed array
    inside the library).  Pass preallocated `out` = (n_unique_dev [1],
    unique_idx [n], inverse [n]) int32 tensors to allocate nothing here
    either."""
    _cuda(fp, "fp")
    _cuda(tokens, "tokens")
    n, stride = tokens.shape
    dev = tokens.device
    if out is None:
        out = (torch.empty(1, dtype=torch.int32, device=dev),
               torch.empty(max(n, 1), dtype=torch.int32, device=dev),
               torch.empty(max(n, 1), dtype=torch.int32, device=dev))
    nu, uidx, inv = out
    _check(load().hs_unique_inverse_noalloc(_ptr(fp), _ptr(tokens), n, stride, _ptr(lens),
                                            _ptr(nu), _ptr(uidx), _ptr(inv), _stream(stream)))
    return nu, _rows(uidx, n), _rows(inv, n)


def hs_retrieve_topk_workspace(n_queries: int, n_corpus: int, dim: int, k: int) -> int:
    return int(load().hs_retrieve_topk_workspace(n_queries, n_corpus, dim, k))


def hs_retrieve_topk(queries: torch.Tensor, corpus: torch.Tensor, k: int,
                     workspace: torch.Tensor | None = None, out: tuple | None = None,
                     stream=None):
    """Top-k inner products of bf16 query rows against bf16 corpus rows.
    Returns (scores fp32 [Q, k], ids int32 [Q, k])."""
    _cuda(queries, "queries")
    _cuda(corpus, "corpus")
    if queries.element_size() != 2 or corpus.element_size() != 2:
        raise TypeError("queries and corpus must hold bf16 (2-byte) elements")
    Q, d = queries.shape
    N, d2 = corpus.shape
    if d != d2:
        raise ValueError("dimension mismatch")
    dev = queries.device
    if out is None:
        out = (torch.empty((Q, k), dtype=torch.float32, device=dev),
               torch.empty((Q, k), dtype=torch.int32, device=dev))
    scores, ids = out
    if workspace is None:
        workspace = torch.empty(hs_retrieve_topk_workspace(Q, N, d, k), dtype=torch.uint8,
                                device=dev)
    _check(load().hs_retrieve_topk(_ptr(queries), Q, _ptr(corpus), N, d, k, _ptr(scores),
                                   _ptr(ids), _ptr(workspace), workspace.numel(), _stream(stream)))
    return scores, ids


def hs_retrieve_topk_n(queries: torch.Tensor, n_queries_dev: torch.Tensor, corpus: torch.Tensor,
                       k: int, workspace: torch.Tensor | None = None, out: tuple | None = None,
                       stream=None):
    """hs_retrieve_topk over the first n_queries_dev[0] rows of `queries`
    (a device int32 scalar, read when the kernels run).  Returns (scores,
    ids) shaped like `queries` rows x k; rows past the count are left as
    they were."""
    _cuda(queries, "queries")
    _cuda(corpus, "corpus")
    _cuda(n_queries_dev, "n_queries_dev")
    if n_queries_dev.dtype != torch.int32:
        raise TypeError("n_queries_dev must be int32")
    if queries.element_size() != 2 or corpus.element_size() != 2:
        raise TypeError("queries and corpus must hold bf16 (2-byte) elements")
    Q, d = queries.shape
    N, d2 = corpus.shape
    if d != d2:
        raise ValueError("dimension mismatch")
    dev = queries.device
    if out is None:
        out = (torch.empty((Q, k), dtype=torch.float32, device=dev),
               torch.empty((Q, k), dtype=torch.int32, device=dev))
    scores, ids = out
    if workspace is None:
        workspace = torch.empty(hs_retrieve_topk_workspace(Q, N, d, k), dtype=torch.uint8,
                                device=dev)
    _check(load().hs_retrieve_topk_n(_ptr(queries), Q, _ptr(n_queries_dev), _ptr(corpus), N, d,
                                     k, _ptr(scores), _ptr(ids), _ptr(workspace),
                                     workspace.numel(), _stream(stream)))
    return scores, ids


def hs_retrieve_topk_fanout(queries: torch.Tensor, n_queries_dev: torch.Tensor | None,
                            inverse: torch.Tensor, corpus: torch.Tensor, k: int,
                            workspace: torch.Tensor | None = None, out: tuple | None = None,
                            stream=None):
    """Retrieval whose results go to every merged row: row o of the returned
    (scores [n_out, k], ids [n_out, k]) is the top-k of query inverse[o]
    (n_out = inverse.numel()).  n_queries_dev (device int32 scalar) or None
    gives the query count, as for hs_retrieve_topk_n."""
    _cuda(queries, "queries")
    _cuda(corpus, "corpus")
    _cuda(inverse, "inverse")
    if inverse.dtype != torch.int32:
        raise TypeError("inverse must be int32")
    if n_queries_dev is not None:
        _cuda(n_queries_dev, "n_queries_dev")
        if n_queries_dev.dtype != torch.int32:
            raise TypeError("n_queries_dev must be int32")
    if queries.element_size() != 2 or corpus.element_size() != 2:
        raise TypeError("queries and corpus must hold bf16 (2-byte) elements")
    Q, d = queries.shape
    N, d2 = corpus.shape
    if d != d2:
        raise ValueError("dimension mismatch")
    n_out = inverse.numel()
    dev = queries.device
    if out is None:
        out = (torch.empty((n_out, k), dtype=torch.float32, device=dev),
               torch.empty((n_out, k), dtype=torch.int32, device=dev))
    scores, ids = out
    if workspace is None:
        workspace = torch.empty(hs_retrieve_topk_workspace(Q, N, d, k), dtype=torch.uint8,
                                device=dev)
    _check(load().hs_retrieve_topk_fanout(_ptr(queries), Q, _ptr(n_queries_dev), _ptr(inverse),
                                          n_out, _ptr(corpus), N, d, k, _ptr(scores), _ptr(ids),
                                          _ptr(workspace), workspace.numel(), _stream(stream)))
    return scores, ids


def hs_merge_queries(queries: torch.Tensor, seed_state: int = HS_FNV64_OFFSET_BASIS,
                     fp_in: torch.Tensor | None = None, out: tuple | None = None, stream=None):
    """Fingerprint, exact merge and gather of a query batch (at most
    HS_MERGE_QUERIES_MAX rows of bf16 vectors) in one launch.  Returns
    (fp [n] int64, n_unique_dev [1] int32, unique_idx [n] int32,
    inverse [n] int32, unique_queries [n, dim]); the first n_unique rows of
    unique_queries are the unique query vectors.  ``out`` may supply those
    five tensors preallocated; ``fp_in`` replaces the computed fingerprints."""
    _cuda(queries, "queries")
    if queries.element_size() != 2 or queries.dim() != 2:
        raise TypeError("queries must be a 2-D tensor of bf16 (2-byte) elements")
    n, d = queries.shape
    dev = queries.device
    if fp_in is not None:
        _cuda(fp_in, "fp_in")
        if fp_in.dtype != torch.int64 or fp_in.numel() != n:
            raise TypeError("fp_in must be int64 [n]")
    if out is None:
        out = (torch.empty(max(n, 1), dtype=torch.int64, device=dev),
               torch.empty(1, dtype=torch.int32, device=dev),
               torch.empty(max(n, 1), dtype=torch.int32, device=dev),
               torch.empty(max(n, 1), dtype=torch.int32, device=dev),
               torch.empty((max(n, 1), d), dtype=queries.dtype, device=dev))
    fp, nu, uidx, inv, uq = out
    _check(load().hs_merge_queries(_ptr(queries), n, d, seed_state & (2**64 - 1), _ptr(fp_in),
                                   _ptr(fp), _ptr(nu), _ptr(uidx), _ptr(inv), _ptr(uq),
                                   _stream(stream)))
    return _rows(fp, n), nu, _rows(uidx, n), _rows(inv, n), _rows(uq, n)


def hs_scatter_results(src: torch.Tensor, mapping: torch.Tensor, dst: torch.Tensor | None = None,
                       stream=None) -> torch.Tensor:
    """dst[i] = src[mapping[i]] row-wise (rows are the first dimension)."""
    _cuda(src, "src")
    _cuda(mapping, "map")
    if mapping.dtype != torch.int32:
        raise TypeError("map must be int32")
    n = mapping.numel()
    row_bytes = src.element_size()
    if src.dim() > 1:
        if src.shape[0] == 0:
            raise IndexError("src has no rows")
        row_bytes *= src.numel() // src.shape[0]
    if dst is None:
        dst = torch.empty((n,) + tuple(src.shape[1:]), dtype=src.dtype, device=src.device)
    _check(load().hs_scatter_results(_ptr(src), src.shape[0], row_bytes, _ptr(mapping), n,
                                     _ptr(dst), _stream(stream)))
    return dst


def hs_rerank_topk(rerank_queries: torch.Tensor, rerank_corpus: torch.Tensor,
                   candidates: torch.Tensor, k2: int, n_queries_dev: torch.Tensor | None = None,
                   inverse: torch.Tensor | None = None, out: tuple | None = None, stream=None):
    """Rescore each query's candidates (int32 [Q, k1] corpus ids) by the
    inner product of bf16 rerank vectors and keep the best k2.  Returns
    (scores fp32, ids int32), one row per query, or one per entry of
    ``inverse`` (row o = query inverse[o]) when it is given."""
    _cuda(rerank_queries, "rerank_queries")
    _cuda(rerank_corpus, "rerank_corpus")
    _cuda(candidates, "candidates")
    if rerank_queries.element_size() != 2 or rerank_corpus.element_size() != 2:
        raise TypeError("rerank vectors must hold bf16 (2-byte) elements")
    if candidates.dtype != torch.int32 or candidates.dim() != 2:
        raise TypeError("candidates must be int32 [Q, k1]")
    Q, d = rerank_queries.shape
    N, d2 = rerank_corpus.shape
    if d != d2:
        raise ValueError("dimension mismatch")
    if candidates.shape[0] != Q:
        raise ValueError("candidates must have one row per query")
    k1 = candidates.shape[1]
    for t, name in ((n_queries_dev, "n_queries_dev"), (inverse, "inverse")):
        if t is not None:
            _cuda(t, name)
            if t.dtype != torch.int32:
                raise TypeError("%s must be int32" % name)
    rows = inverse.numel() if inverse is not None else Q
    dev = rerank_queries.device
    if out is None:
        out = (torch.empty((rows, k2), dtype=torch.float32, device=dev),
               torch.empty((rows, k2), dtype=torch.int32, device=dev))
    scores, ids = out
    _check(load().hs_rerank_topk(_ptr(rerank_queries), Q, _ptr(n_queries_dev),
                                 _ptr(rerank_corpus), N, d, _ptr(candidates), k1, int(k2),
                                 _ptr(inverse), rows if inverse is not None else 0, _ptr(scores),
                                 _ptr(ids), _stream(stream)))
    return scores, ids


class ResultCache:
    """Device-resident fingerprint -> retrieval result table that persists
    across batches (asynchronous cache reuse, Section 3.3 (II)): ``capacity``
    entries of a dim-wide query vector and its k scores and ids, in one
    uint8 tensor allocated here (the library itself allocates nothing)."""

    def __init__(self, capacity: int, dim: int, k: int, device=None, stream=None):
        self.capacity, self.dim, self.k = int(capacity), int(dim), int(k)
        nbytes = int(load().hs_cache_bytes(self.capacity, self.dim, self.k))
        if nbytes == 0:
            raise ValueError("invalid cache shape")
        self.mem = torch.empty(nbytes, dtype=torch.uint8, device=device or "cuda")
        hs_cache_init(self, stream)

    def _args(self):
        return (_ptr(self.mem), self.mem.numel(), self.capacity, self.dim, self.k)


def hs_cache_init(cache: ResultCache, stream=None) -> None:
    """Empty the cache (every entry free, counters zero)."""
    _check(load().hs_cache_init(*cache._args(), _stream(stream)))


def hs_cache_bytes(capacity: int, dim: int, k: int) -> int:
    return int(load().hs_cache_bytes(capacity, dim, k))


def hs_cache_lookup(cache: ResultCache, queries: torch.Tensor, fp: torch.Tensor,
                    fp_rows: torch.Tensor | None = None, n_queries_dev: torch.Tensor | None = None,
                    out: tuple | None = None, miss: tuple | None = None, stream=None):
    """Look the merged queries up in the cache.  Hits get their cached
    (scores, ids) rows in ``out``; misses are listed in ``miss`` =
    (miss_list [Q] int32, n_miss_dev [1] int32, miss_queries [Q, dim]) with
    their vectors gathered for retrieval.  Query u's key is fp[fp_rows[u]]
    (fp[u] if fp_rows is None).  Returns (out, miss)."""
    for t, name in ((queries, "queries"), (fp, "fp")):
        _cuda(t, name)
    Q, d = queries.shape
    dev = queries.device
    if out is None:
        out = (torch.empty((Q, cache.k), dtype=torch.float32, device=dev),
               torch.empty((Q, cache.k), dtype=torch.int32, device=dev))
    if miss is None:
        miss = (torch.empty(max(Q, 1), dtype=torch.int32, device=dev),
                torch.empty(1, dtype=torch.int32, device=dev),
                torch.empty((max(Q, 1), d), dtype=queries.dtype, device=dev))
    _check(load().hs_cache_lookup(*cache._args(), _ptr(queries), _ptr(fp), _ptr(fp_rows), Q,
                                  _ptr(n_queries_dev), _ptr(out[0]), _ptr(out[1]), _ptr(miss[0]),
                                  _ptr(miss[1]), _ptr(miss[2]), _stream(stream)))
    return out, miss


def hs_cache_insert(cache: ResultCache, miss: tuple, fp: torch.Tensor, miss_scores: torch.Tensor,
                    miss_ids: torch.Tensor, out: tuple, fp_rows: torch.Tensor | None = None,
                    stream=None):
    """Insert the retrieved results of the misses of ``hs_cache_lookup``
    (rows of miss_scores / miss_ids follow the miss list) into the cache and
    write them to the queries' rows of ``out``."""
    miss_list, n_miss, miss_q = miss
    _check(load().hs_cache_insert(*cache._args(), _ptr(miss_list), _ptr(n_miss),
                                  miss_list.numel(), _ptr(miss_q), _ptr(fp), _ptr(fp_rows),
                                  _ptr(miss_scores), _ptr(miss_ids), _ptr(out[0]), _ptr(out[1]),
                                  _stream(stream)))
    return out


def hs_cache_stats(cache: ResultCache, stream=None):
    """(hits, misses) counted since the cache was initialised (synchronises)."""
    h, m = ctypes.c_uint64(0), ctypes.c_uint64(0)
    _check(load().hs_cache_stats(_ptr(cache.mem), ctypes.addressof(h), ctypes.addressof(m),
                                 _stream(stream)))
    return int(h.value), int(m.value)


def hs_segment_sum(phi: torch.Tensor, inverse: torch.Tensor, max_groups: int,
                   n_groups_dev: torch.Tensor | None = None, out: torch.Tensor | None = None,
                   stream=None) -> torch.Tensor:
    """out[u] = sum of phi[i] over rows with inverse[i] == u (float64
    [max_groups]; entries past the group count, n_groups_dev[0] if given,
    are 0): the priority contribution of each fused node."""
    _cuda(phi, "phi")
    _cuda(inverse, "inverse")
    if phi.dtype != torch.float64 or inverse.dtype != torch.int32:
        raise TypeError("phi must be float64 and inverse int32")
    if phi.numel() != inverse.numel():
        raise ValueError("phi and inverse differ in length")
    if n_groups_dev is not None:
        _cuda(n_groups_dev, "n_groups_dev")
        if n_groups_dev.dtype != torch.int32:
            raise TypeError("n_groups_dev must be int32")
    if out is None:
        out = torch.empty(max(int(max_groups), 1), dtype=torch.float64, device=phi.device)
    _check(load().hs_segment_sum(_ptr(phi), _ptr(inverse), phi.numel(), _ptr(n_groups_dev),
                                 int(max_groups), _ptr(out), _stream(stream)))
    return _rows(out, int(max_groups))


class _KvCacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p),
                ("v_scale", ctypes.c_void_p), ("n_blocks", ctypes.c_int64),
                ("n_kv_heads", ctypes.c_int32), ("block_tokens", ctypes.c_int32),
                ("dim", ctypes.c_int32), ("format", ctypes.c_int32)]


_KV_CODES = {torch.float8_e4m3fn: HS_KV_E4M3, torch.int8: HS_KV_INT8}
_KV_DTYPES = {torch.bfloat16: HS_KV_BF16, torch.float16: HS_KV_FP16}


class KvCache:
    """Paged cache of keys and values, 8 bits a value: codes ``k`` and ``v``
    [n_blocks, n_kv_heads, block_tokens, dim] (torch.float8_e4m3fn or
    torch.int8) and float32 scales [n_blocks, n_kv_heads]; a code stands for
    itself times its block and head's scale.  Allocated here, or ``of``
    tensors that a program has."""

    def __init__(self, n_blocks: int, block_tokens: int, n_kv_heads: int, dim: int,
                 dtype: torch.dtype = torch.float8_e4m3fn, device=None):
        if dtype not in _KV_CODES:
            raise TypeError("a cache holds torch.float8_e4m3fn or torch.int8")
        shape = (int(n_blocks), int(n_kv_heads), int(block_tokens), int(dim))
        dev = device or "cuda"
        self._take(*(torch.empty(shape, dtype=dtype, device=dev) for _ in range(2)),
                   *(torch.zeros(shape[:2], dtype=torch.float32, device=dev) for _ in range(2)))

    @classmethod
    def of(cls, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor,
           v_scale: torch.Tensor) -> "KvCache":
        self = cls.__new__(cls)
        self._take(k, v, k_scale, v_scale)
        return self

    def _take(self, k, v, k_scale, v_scale):
        for t, name in ((k, "k"), (v, "v"), (k_scale, "k_scale"), (v_scale, "v_scale")):
            _cuda(t, name)
        if k.dtype not in _KV_CODES or v.dtype != k.dtype:
            raise TypeError("k and v must both be torch.float8_e4m3fn or torch.int8")
        if k.dim() != 4 or v.shape != k.shape:
            raise ValueError("k and v must be [n_blocks, n_kv_heads, block_tokens, dim]")
        for t in (k_scale, v_scale):
            if t.dtype != torch.float32 or t.shape != k.shape[:2]:
                raise TypeError("scales must be float32 [n_blocks, n_kv_heads]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_blocks, self.n_kv_heads, self.block_tokens, self.dim = k.shape
        self._struct = _KvCacheStruct(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                                      v_scale.data_ptr(), *k.shape, _KV_CODES[k.dtype])
        self._at = ctypes.addressof(self._struct)


# The checks of these calls read each attribute once: a property is 0.1 us of
# host time, a small function's call 0.3, an allocation 1.5 (a view of one 1.7),
# and a decoding step's kernels are 4 to 12 us.
_I32 = torch.int32


def _i32(t, name: str, n: int | None = None):
    """The address of a contiguous int32 CUDA tensor of n elements."""
    if t.dtype is not _I32 or not t.is_cuda or not t.is_contiguous():
        raise TypeError("%s must be a contiguous int32 CUDA tensor" % name)
    if n is not None and t.numel() != n:
        raise ValueError("%s must have %d elements" % (name, n))
    return t.data_ptr()


def _kv_cursor(t, name: str):
    if t.dtype != torch.int64 or not t.is_cuda or t.numel() != 2 or not t.is_contiguous():
        raise TypeError("%s must be a contiguous int64 CUDA tensor of 2 elements" % name)
    return t.data_ptr()


def hs_kv_tables(have: torch.Tensor, fresh: torch.Tensor, table: torch.Tensor, pool: torch.Tensor,
                 cursor: torch.Tensor, block_tokens: int, max_tokens: int,
                 n_req_dev: torch.Tensor | None = None, out: tuple | None = None, stream=None):
    """Blocks and slots for the ``fresh[r]`` new tokens of requests that have
    ``have[r]`` in the cache.  ``table`` [n_req, width] gets the new blocks,
    taken from the ring ``pool`` [n_blocks] at ``cursor`` = {taken, given}
    (int64 [2]).  Returns (slots [max_tokens], starts [n_req + 1], lens
    [n_req], cursor [2]), or writes them to ``out``; max_tokens is the number
    of new tokens, or more (slot -1 past them)."""
    n = have.numel()
    at = table.shape
    if len(at) != 2 or at[0] != n:
        raise ValueError("table must be [n_req, width]")
    if not (have.dtype is _I32 and fresh.dtype is _I32 and table.dtype is _I32
            and pool.dtype is _I32 and have.is_cuda and fresh.is_cuda and table.is_cuda
            and pool.is_cuda and have.is_contiguous() and fresh.is_contiguous()
            and table.is_contiguous() and pool.is_contiguous()):
        raise TypeError("have, fresh, table and pool must be contiguous int32 CUDA tensors")
    if fresh.numel() != n:
        raise ValueError("fresh must have %d elements" % n)
    cp = _kv_cursor(cursor, "cursor")
    if out is None:
        dev = have.device
        slots = torch.empty(max_tokens, dtype=_I32, device=dev)
        starts = torch.empty(n + 1, dtype=_I32, device=dev)
        lens = torch.empty_like(have)
        after = torch.empty_like(cursor)
        outs = (after.data_ptr(), starts.data_ptr(), lens.data_ptr(), slots.data_ptr())
    else:
        slots, starts, lens, after = out
        outs = (_kv_cursor(after, "cursor out"), _i32(starts, "starts", n + 1),
                _i32(lens, "lens", n), _i32(slots, "slots", max_tokens))
    _check((_lib or load()).hs_kv_tables(
        have.data_ptr(), fresh.data_ptr(), n,
        None if n_req_dev is None else _i32(n_req_dev, "n_req_dev"), block_tokens,
        table.data_ptr(), at[1], pool.data_ptr(), pool.numel(), cp, *outs, max_tokens,
        _stream(stream)))
    return slots, starts, lens, after


def hs_kv_release(lens: torch.Tensor, table: torch.Tensor, pool: torch.Tensor,
                  cursor: torch.Tensor, block_tokens: int,
                  n_req_dev: torch.Tensor | None = None, out: torch.Tensor | None = None,
                  stream=None) -> torch.Tensor:
    """The blocks of ``lens[r]`` tokens of each finished request (0: it goes
    on) go back into the ring.  Returns the cursor after that."""
    n = lens.numel()
    if table.dim() != 2 or table.shape[0] != n:
        raise ValueError("table must be [n_req, width]")
    if out is None:
        out = cursor.new_empty(2)
    _check(load().hs_kv_release(
        _i32(lens, "lens"), n, None if n_req_dev is None else _i32(n_req_dev, "n_req_dev"),
        int(block_tokens), _i32(table, "table"), table.shape[1], _i32(pool, "pool"),
        pool.numel(), _kv_cursor(cursor, "cursor"), _kv_cursor(out, "cursor out"),
        _stream(stream)))
    return out


def _kv_heads(t, name: str, dim: int):
    """t's data pointer and dtype code: a CUDA tensor [tokens, heads, dim] of
    bf16 or fp16 values whose heads are contiguous."""
    dtype = _KV_DTYPES.get(t.dtype)
    if dtype is None or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor of bfloat16 or float16" % name)
    if t.dim() != 3 or t.shape[2] != dim or t.stride(2) != 1:
        raise ValueError("%s must be [tokens, heads, dim] with contiguous heads of the cache's dim"
                         % name)
    return t.data_ptr(), dtype


def hs_kv_append(cache: KvCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
                 stream=None) -> None:
    """Write new keys and values [tokens, n_kv_heads, dim] (views with strides
    of their own, the same for both, are fine) into their slots, rounded to
    the cache's codes; block scales grow as they have to."""
    kp, dtype = _kv_heads(k, "k", cache.dim)
    vp, vtype = _kv_heads(v, "v", cache.dim)
    shape, by = k.shape, k.stride()
    if v.shape != shape or shape[1] != cache.n_kv_heads or vtype != dtype:
        raise ValueError("k and v must both be [tokens, n_kv_heads, dim] of one dtype")
    T = shape[0]
    other = v.stride()
    if other != by:                             # of an axis of length 1 they say nothing
        if (T > 1 and other[0] != by[0]) or (shape[1] > 1 and other[1] != by[1]):
            raise ValueError("k and v must have the same strides")
        by = (by[0] if T > 1 else 0, by[1] if shape[1] > 1 else 0)
    _check((_lib or load()).hs_kv_append(cache._at, kp, vp, dtype, T, by[0], by[1],
                                         _i32(slots, "slots", T), _stream(stream)))


def hs_kv_attend_workspace(cache: KvCache, n_heads: int, max_q: int) -> int:
    """Bytes of hs_kv_attend's workspace, which is zeroed once."""
    return int(load().hs_kv_attend_workspace(int(n_heads), cache.n_kv_heads, cache.dim, int(max_q)))


def hs_kv_attend(cache: KvCache, q: torch.Tensor, lens: torch.Tensor, table: torch.Tensor,
                 starts: torch.Tensor | None = None, max_q: int | None = None,
                 scale: float | None = None, causal: bool = True, window: int = 0,
                 n_req_dev: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                 out: tuple | None = None, stream=None):
    """Attention of queries q [tokens, n_heads, dim] over the cache.  Request
    r has lens[r] tokens there, in the blocks of row r of ``table``, and the
    queries starts[r] .. starts[r + 1] - 1, at its last positions; without
    ``starts`` every request has tokens / n_req of them.  ``max_q`` is the
    most queries of a request (all of them, if it is not given).  Returns
    (out, shaped and typed like q, and lse float32 [tokens, n_heads])."""
    dtype = _KV_DTYPES.get(q.dtype)
    shape, by = q.shape, q.stride()
    if dtype is None or not q.is_cuda or len(shape) != 3 or shape[2] != cache.dim or by[2] != 1:
        _kv_heads(q, "q", cache.dim)
    T, heads, dim = shape
    n = lens.numel()
    at = table.shape
    if len(at) != 2 or at[0] != n:
        raise ValueError("table must be [n_req, width]")
    if not (lens.dtype is _I32 and table.dtype is _I32 and lens.is_cuda and table.is_cuda
            and lens.is_contiguous() and table.is_contiguous()):
        raise TypeError("lens and table must be contiguous int32 CUDA tensors")
    if starts is None:
        if n and T % n:
            raise ValueError("without starts, every request has as many queries")
        each = T // n if n else 0
        if max_q is not None and max_q != each:
            raise ValueError("max_q is not what every request has")
        max_q, sp = each, None
    else:
        sp = _i32(starts, "starts", n + 1)
        if max_q is None:
            max_q = T
    if out is None:
        o = torch.empty_like(q, memory_format=torch.contiguous_format)
        lse = torch.empty((T, heads), dtype=torch.float32, device=q.device)
    else:
        o, lse = out
        if o.dtype != q.dtype or o.shape != shape or not o.is_cuda or not o.is_contiguous():
            raise ValueError("out must be contiguous and like q")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != shape[:2]
                                or not lse.is_cuda or not lse.is_contiguous()):
            raise ValueError("lse must be contiguous float32 [tokens, n_heads]")
    if workspace is None:                       # zeroed on the stream that uses it
        with torch.cuda.stream(_on(stream, q.device)):
            workspace = torch.zeros(hs_kv_attend_workspace(cache, heads, max_q),
                                    dtype=torch.uint8, device=q.device)
    _check((_lib or load()).hs_kv_attend(
        cache._at, q.data_ptr(), dtype, T, heads, by[0], by[1], lens.data_ptr(), sp, n,
        None if n_req_dev is None else _i32(n_req_dev, "n_req_dev"), max_q, table.data_ptr(),
        at[1], dim ** -0.5 if scale is None else scale, 1 if causal else 0, window, o.data_ptr(),
        None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes,
        _stream(stream)))
    return o, lse


def hs_kv_fork(src: torch.Tensor, dst: torch.Tensor, lens: torch.Tensor, table: torch.Tensor,
               shared: torch.Tensor, pool: torch.Tensor, cursor: torch.Tensor, block_tokens: int,
               out: tuple | None = None, stream=None):
    """Row dst[i] of ``table`` begins as row src[i] stands: it names the same
    full blocks, counted in ``shared`` [n_blocks], and a new block from the ring
    for the tokens left over.  ``table`` and ``shared`` change in place.  Returns
    (lens [n_req], cursor [2], source, target, tokens [n_fork]), or writes them
    to ``out``; the last three are hs_kv_copy's lists."""
    return _fork(src, dst, lens, table, shared, pool, cursor, block_tokens, None, out, stream)


def hs_kv_fork_n(src: torch.Tensor, dst: torch.Tensor, lens: torch.Tensor, n_req_dev: torch.Tensor,
                 table: torch.Tensor, shared: torch.Tensor, pool: torch.Tensor,
                 cursor: torch.Tensor, block_tokens: int, out: tuple | None = None, stream=None):
    """hs_kv_fork where ``n_req_dev`` [1] says how many of the rows are requests.
    Returns a sixth, or writes it to the sixth of ``out``: that number, or one
    more than the last row that is made."""
    return _fork(src, dst, lens, table, shared, pool, cursor, block_tokens, n_req_dev, out, stream)


def _fork(src, dst, lens, table, shared, pool, cursor, block_tokens, n_req_dev, out, stream):
    n, n_req = src.numel(), lens.numel()
    at = table.shape
    if len(at) != 2 or at[0] != n_req:
        raise ValueError("table must be [n_req, width]")
    blocks = pool.numel()
    if not (src.dtype is _I32 and dst.dtype is _I32 and lens.dtype is _I32 and table.dtype is _I32
            and shared.dtype is _I32 and pool.dtype is _I32 and src.is_cuda and dst.is_cuda
            and lens.is_cuda and table.is_cuda and shared.is_cuda and pool.is_cuda
            and src.is_contiguous() and dst.is_contiguous() and lens.is_contiguous()
            and table.is_contiguous() and shared.is_contiguous() and pool.is_contiguous()):
        raise TypeError("src, dst, lens, table, shared and pool must be contiguous int32 CUDA "
                        "tensors")
    if dst.numel() != n or shared.numel() != blocks:
        raise ValueError("dst must be as long as src, shared as long as pool")
    cp = _kv_cursor(cursor, "cursor")
    if out is None:
        new = torch.empty_like
        after, moved, source, target, tokens = new(lens), new(cursor), new(src), new(src), new(src)
        outs = (after.data_ptr(), moved.data_ptr(), source.data_ptr(), target.data_ptr(),
                tokens.data_ptr())
        made = None if n_req_dev is None else new(n_req_dev)
    else:
        made = None
        if n_req_dev is None:
            after, moved, source, target, tokens = out
        else:
            after, moved, source, target, tokens, made = out
        outs = (_i32(after, "lens out", n_req), _kv_cursor(moved, "cursor out"),
                _i32(source, "source", n), _i32(target, "target", n), _i32(tokens, "tokens", n))
    _check((_lib or load()).hs_kv_fork_n(
        src.data_ptr(), dst.data_ptr(), n, lens.data_ptr(), outs[0], n_req,
        None if n_req_dev is None else _i32(n_req_dev, "n_req_dev", 1),
        None if n_req_dev is None else _i32(made, "n_req out", 1), block_tokens,
        table.data_ptr(), at[1], shared.data_ptr(), pool.data_ptr(), blocks, cp, *outs[1:],
        _stream(stream)))
    lists = after, moved, source, target, tokens
    return lists if n_req_dev is None else lists + (made,)


def hs_kv_copy(cache: KvCache, source: torch.Tensor, target: torch.Tensor,
               tokens: torch.Tensor | None = None, n_dev: torch.Tensor | None = None,
               stream=None) -> None:
    """Codes of the first ``tokens[i]`` tokens (all, without it) and scales of
    block source[i] to block target[i], for the first ``n_dev`` pairs (all,
    without it); -1 in either list is no pair."""
    n = source.numel()
    _check((_lib or load()).hs_kv_copy(
        cache._at, _i32(source, "source"), _i32(target, "target", n),
        None if tokens is None else _i32(tokens, "tokens", n), n,
        None if n_dev is None else _i32(n_dev, "n_dev", 1), _stream(stream)))


def hs_kv_release_shared(lens: torch.Tensor, table: torch.Tensor, shared: torch.Tensor,
                         pool: torch.Tensor, cursor: torch.Tensor, block_tokens: int,
                         n_req_dev: torch.Tensor | None = None, out: tuple | None = None,
                         stream=None):
    """hs_kv_release where blocks may have several holders: those that are left
    without any go back into the ring.  Returns (shared, cursor) after that, or
    writes them to ``out``, whose first may be ``shared`` itself."""
    n, blocks = lens.numel(), pool.numel()
    at = table.shape
    if len(at) != 2 or at[0] != n:
        raise ValueError("table must be [n_req, width]")
    if not (lens.dtype is _I32 and table.dtype is _I32 and shared.dtype is _I32
            and pool.dtype is _I32 and lens.is_cuda and table.is_cuda and shared.is_cuda
            and pool.is_cuda and lens.is_contiguous() and table.is_contiguous()
            and shared.is_contiguous() and pool.is_contiguous()):
        raise TypeError("lens, table, shared and pool must be contiguous int32 CUDA tensors")
    if shared.numel() != blocks:
        raise ValueError("shared must be as long as pool")
    cp = _kv_cursor(cursor, "cursor")
    if out is None:
        left, after = torch.empty_like(shared), torch.empty_like(cursor)
        outs = (left.data_ptr(), after.data_ptr())
    else:
        left, after = out
        outs = (_i32(left, "shared out", blocks), _kv_cursor(after, "cursor out"))
    _check((_lib or load()).hs_kv_release_shared(
        lens.data_ptr(), n, None if n_req_dev is None else _i32(n_req_dev, "n_req_dev"),
        block_tokens, table.data_ptr(), at[1], shared.data_ptr(), outs[0], pool.data_ptr(), blocks,
        cp, outs[1], _stream(stream)))
    return left, after


def hs_kv_compact_workspace(n_blocks: int) -> int:
    """Bytes of hs_kv_compact's workspace."""
    return int(load().hs_kv_compact_workspace(int(n_blocks)))


def hs_kv_compact(lens: torch.Tensor, table: torch.Tensor, shared: torch.Tensor, block_tokens: int,
                  n_req_dev: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                  out: tuple | None = None, stream=None):
    """The U blocks in use to numbers below U.  Returns (table, shared [n_blocks],
    pool [n_blocks], cursor [2], source, target [max(1, n_blocks / 2)], moves [1])
    after that, or writes them to ``out``, whose first two may be ``table`` and
    ``shared`` themselves; source, target and moves are hs_kv_copy's lists and
    n_dev, for every layer's cache."""
    if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
        raise TypeError("workspace must be a contiguous CUDA tensor")
    n, blocks = lens.numel(), shared.numel()
    at = table.shape
    if len(at) != 2 or at[0] != n:
        raise ValueError("table must be [n_req, width]")
    if not (lens.dtype is _I32 and table.dtype is _I32 and shared.dtype is _I32 and lens.is_cuda
            and table.is_cuda and shared.is_cuda and lens.is_contiguous()
            and table.is_contiguous() and shared.is_contiguous()):
        raise TypeError("lens, table and shared must be contiguous int32 CUDA tensors")
    room = max(1, blocks // 2)
    if out is None:
        dev, new = shared.device, torch.empty_like
        named, left, pool = new(table), new(shared), new(shared)
        after = torch.empty(2, dtype=torch.int64, device=dev)
        source = torch.empty(room, dtype=_I32, device=dev)
        target, moves = new(source), torch.empty(1, dtype=_I32, device=dev)
        outs = (named.data_ptr(), left.data_ptr(), pool.data_ptr(), after.data_ptr(),
                source.data_ptr(), target.data_ptr(), moves.data_ptr())
    else:
        named, left, pool, after, source, target, moves = out
        if named.shape != at:
            raise ValueError("table out must be shaped like table")
        outs = (_i32(named, "table out"), _i32(left, "shared out", blocks),
                _i32(pool, "pool", blocks), _kv_cursor(after, "cursor out"),
                _i32(source, "source", room), _i32(target, "target", room),
                _i32(moves, "moves", 1))
    if workspace is None:
        size, dev = hs_kv_compact_workspace(blocks), table.device
        if stream is None:
            workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        else:                                   # of the stream that uses it: it is freed on return
            with torch.cuda.stream(_on(stream, dev)):
                workspace = torch.empty(size, dtype=torch.uint8, device=dev)
    _check((_lib or load()).hs_kv_compact(
        lens.data_ptr(), n, None if n_req_dev is None else _i32(n_req_dev, "n_req_dev"),
        block_tokens, table.data_ptr(), outs[0], at[1], shared.data_ptr(), outs[1], blocks,
        *outs[2:], workspace.data_ptr(), workspace.nbytes, _stream(stream)))
    return named, left, pool, after, source, target, moves


_ROTARY_LAYOUTS = {"half": HS_ROTARY_HALF, "interleaved": HS_ROTARY_INTERLEAVED}


def hs_rotary_frequencies(rot_dim: int, base: float = 10000.0, factor: float = 1.0,
                          original_len: float = 0.0, slow: float = 1.0,
                          fast: float = 4.0) -> torch.Tensor:
    """How far each pair turns in a token, as 64-bit fractions of a turn (a host
    int64 tensor of the uint64 bits; see hs.h)."""
    turns = torch.empty(max(int(rot_dim) // 2, 0), dtype=torch.int64)
    _check(load().hs_rotary_frequencies(float(base), int(rot_dim), float(factor),
                                        float(original_len), float(slow), float(fast),
                                        turns.data_ptr() or None))
    return turns


class Rotary:
    """Rotary positions as a model has them: how far each pair of the first
    ``rot_dim`` values of a head turns in a token, which values are a pair
    (``layout`` "half" or "interleaved") and the factor on what is turned."""

    def __init__(self, rot_dim: int, base: float = 10000.0, layout: str = "half",
                 factor: float = 1.0, original_len: float = 0.0, slow: float = 1.0,
                 fast: float = 4.0, magnitude: float = 1.0, device=None):
        turns = hs_rotary_frequencies(rot_dim, base, factor, original_len, slow, fast)
        self._take(turns, layout, magnitude, device)

    @classmethod
    def of(cls, inv_freq, layout: str = "half", magnitude: float = 1.0, device=None) -> "Rotary":
        """From each pair's radians a token (a sequence of floats)."""
        turns = [round(float(f) / (2 * math.pi) * 2.0 ** 64) % 2 ** 64 for f in inv_freq]
        if not turns:
            raise ValueError("inv_freq is empty")
        self = cls.__new__(cls)
        self._take(torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turns]), layout,
                   magnitude, device)
        return self

    def _take(self, turns, layout, magnitude, device):
        if layout not in _ROTARY_LAYOUTS:
            raise ValueError("layout is neither half nor interleaved")
        self.turns = turns.to(device or "cuda")
        self.rot_dim, self.magnitude = 2 * turns.numel(), float(magnitude)
        self.layout = layout
        self._layout = _ROTARY_LAYOUTS[layout]


def hs_rotary(x: torch.Tensor, rotary: Rotary, positions: torch.Tensor | None = None,
              lens: torch.Tensor | None = None, starts: torch.Tensor | None = None,
              n_req_dev: torch.Tensor | None = None, inverse: bool = False,
              out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """x [tokens, heads, dim] (bf16 or fp16, strides of its own are fine) turned
    by its tokens' positions: ``positions`` (int32), or those of requests with
    ``lens[r]`` tokens of which starts[r] .. starts[r + 1] - 1 are the last.
    ``inverse`` turns back: the gradient of x from that of the result.  Returns
    ``out`` (which may be x), or a new tensor; tokens behind the last request's
    are not written."""
    shape, by = x.shape, x.stride()
    dtype = _KV_DTYPES.get(x.dtype)
    turns = rotary.turns
    if not turns.is_cuda:
        raise TypeError("rotary's turns must be on a CUDA device")
    if dtype is None or not x.is_cuda:
        raise TypeError("x must be a CUDA tensor of bfloat16 or float16")
    if len(shape) != 3 or by[2] != 1:
        raise ValueError("x must be [tokens, heads, dim] with contiguous heads")
    T = shape[0]
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
        to = (shape[1] * shape[2], shape[2])
    else:
        to = out.stride()
        if out.dtype != x.dtype or out.shape != shape or not out.is_cuda or to[2] != 1:
            raise ValueError("out must be like x, with contiguous heads")
    pp = lp = sp = np_ = None
    n = 0
    if positions is not None:
        if lens is not None or starts is not None:
            raise ValueError("positions, or lens and starts, not both")
        pp = _i32(positions, "positions", T)
    elif lens is None or starts is None:
        raise ValueError("positions, or lens and starts, are needed")
    else:
        n = lens.numel()
        lp, sp = _i32(lens, "lens"), _i32(starts, "starts", n + 1)
        np_ = None if n_req_dev is None else _i32(n_req_dev, "n_req_dev")
    _check((_lib or load()).hs_rotary(
        x.data_ptr(), by[0], by[1], out.data_ptr(), to[0], to[1], dtype, T, shape[1], shape[2],
        rotary.rot_dim, rotary._layout, turns.data_ptr(), rotary.magnitude,
        1 if inverse else 0, pp, lp, sp, n, np_, _stream(stream)))
    return out


def _f32(t, name: str, n: int):
    if t.dtype is not torch.float32 or not t.is_cuda or not t.is_contiguous():
        raise TypeError("%s must be a contiguous float32 CUDA tensor" % name)
    if t.numel() != n:
        raise ValueError("%s must have %d elements" % (name, n))
    return t.data_ptr()


def hs_sample(logits: torch.Tensor, u: torch.Tensor, temperature: torch.Tensor | None = None,
              top_k: torch.Tensor | None = None, top_p: torch.Tensor | None = None,
              min_p: torch.Tensor | None = None, row_of: torch.Tensor | None = None,
              n_dev: torch.Tensor | None = None, out: tuple | None = None, stream=None):
    """One token for each uniform number u[i] in [0, 1), from row row_of[i] (or
    i) of logits [rows, vocab] (bf16 or fp16, rows may lie apart): temperature
    (float32; 0 is the largest logit), then the first top_k (int32; <= 0: all),
    the fewest with top_p of their weight, those within min_p of the largest's.
    With ``n_dev`` the first n_dev[0] draws.  Returns (tokens int32, logprob
    float32 of the token among what is kept, kept int32), or writes them to
    ``out``, whose last two may be None."""
    dtype = _KV_DTYPES.get(logits.dtype)
    if dtype is None or not logits.is_cuda:
        raise TypeError("logits must be a CUDA tensor of bfloat16 or float16")
    shape, by = logits.shape, logits.stride()
    if len(shape) != 2 or (by[1] != 1 and shape[1] != 1):
        raise ValueError("logits must be [rows, vocab] with contiguous rows")
    n = u.numel()
    up = _f32(u, "u", n)
    if out is None:
        tokens = torch.empty_like(u, dtype=_I32)
        logprob = torch.empty_like(u)
        kept = torch.empty_like(tokens)
        outs = (tokens.data_ptr(), logprob.data_ptr(), kept.data_ptr())
    else:
        tokens, logprob, kept = out
        outs = (_i32(tokens, "tokens", n), None if logprob is None else _f32(logprob, "logprob", n),
                None if kept is None else _i32(kept, "kept", n))
    _check((_lib or load()).hs_sample(
        logits.data_ptr(), dtype, shape[0], shape[1], by[0],
        None if row_of is None else _i32(row_of, "row_of", n), n,
        None if n_dev is None else _i32(n_dev, "n_dev", 1),
        None if temperature is None else _f32(temperature, "temperature", n),
        None if top_k is None else _i32(top_k, "top_k", n),
        None if top_p is None else _f32(top_p, "top_p", n),
        None if min_p is None else _f32(min_p, "min_p", n), up, *outs, _stream(stream)))
    return tokens, logprob, kept


def hs_launch_count() -> int:
    """Kernels launched by the library in this process (diagnostics)."""
    return int(load().hs_launch_count())


def hs_get_device_error(stream=None) -> None:
    """Synchronise the stream; raise HsError if a kernel reported a problem."""
    _check(load().hs_get_device_error(_stream(stream)))


def hs_debug_scan_wait(limit_ns: int = 0, withhold_tile: int = -1) -> None:
    """Test hook of hs_unique_inverse's bounded look-back wait (see hs.h);
    hs_debug_scan_wait() restores the defaults."""
    _check(load().hs_debug_scan_wait(int(limit_ns), int(withhold_tile)))


def hs_debug_stream_rows(tokens: torch.Tensor, lens: torch.Tensor | None = None, pattern: int = 0,
                         checksum: torch.Tensor | None = None, blocks_per_sm: int = 4,
                         stream=None) -> torch.Tensor:
    """Read the rows' valid prefixes with one access pattern (diagnostics,
    see hs.h); returns the xor checksum tensor it folded them into."""
    n, stride = tokens.shape
    if checksum is None:
        checksum = torch.zeros(1, dtype=torch.int32, device=tokens.device)
    _check(load().hs_debug_stream_rows(tokens.data_ptr(), n, stride,
                                        None if lens is None else lens.data_ptr(), int(pattern),
                                        checksum.data_ptr(), int(blocks_per_sm), _stream(stream)))
    return checksum
