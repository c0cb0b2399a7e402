"""ctypes binding over the C ABI in include/unique.h -- argument marshalling only.

Every function has the name of the C entry point without the ``unique_`` prefix and
passes ``tensor.data_ptr()`` / the current torch HIP stream straight through. torch is
used for device memory and streams; every step of the computation runs in the HIP library.
There is no fallback: if the library is missing and cannot be built, ``load()`` raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from . import build as _build

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = 0, 1, 2, 3, 4
DTYPE_CODE = {torch.float32: 0, torch.bfloat16: 1}

EXPORTS = ("unique_workspace_bytes", "unique_page_stats_record_bytes", "unique_update_page_stats", "unique_score_select_topk",
           "unique_page_scores", "unique_select_topk", "unique_decode_step", "unique_decode_step_static", "unique_sparse_paged_decode", "unique_dense_paged_decode",
           "unique_page_record_bytes", "unique_quantise_pages", "unique_restore_pages", "unique_quantised_workspace_bytes", "unique_quantised_paged_decode",
           "unique_account_workspace_bytes", "unique_weighted_paged_decode", "unique_evict_pages", "unique_status_string",
           "unique_last_error", "unique_version")


class CacheDesc(C.Structure):
    """Mirror of ``unique_cache_desc``."""
    _fields_ = [("dtype", C.c_int32), ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("page_size", C.c_int32), ("batch", C.c_int32),
                ("max_pages_per_seq", C.c_int32), ("max_seq_len_hint", C.c_int32),
                ("num_phys_pages", C.c_int64), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p),
                ("page_stats", C.c_void_p), ("page_table", C.c_void_p), ("seq_lens", C.c_void_p),
                ("stats_dtype", C.c_int32), ("force_recent_pages", C.c_int32),
                ("kv_page_stride", C.c_int64), ("kv_head_stride", C.c_int64),
                ("min_seq_len_hint", C.c_int32), ("reserved0", C.c_int32)]


class UniqueError(RuntimeError):
    def __init__(self, code: int, status: str, detail: str):
        super().__init__(f"unique status {code} ({status}): {detail}")
        self.code = code


def _p(t):
    return None if t is None else t.data_ptr()


# torch.cuda.current_stream() builds a Stream object on every call (2.6 of the 5 us that a call spent in Python); its
# handle alone costs 0.1 us. Before torch has touched the GPU the current stream is the default one.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


class Library:
    def __init__(self, path: str):
        self.path = path
        self.c = C.CDLL(path)
        for name in EXPORTS:
            getattr(self.c, name)  # raises AttributeError if a declared symbol is not exported
        for name in ("unique_status_string", "unique_last_error", "unique_version"):
            getattr(self.c, name).restype = C.c_char_p
        self.c.unique_status_string.argtypes = [C.c_int]
        self.c.unique_workspace_bytes.argtypes = [C.POINTER(CacheDesc), C.c_int32, C.POINTER(C.c_size_t)]
        self.c.unique_page_stats_record_bytes.argtypes = [C.POINTER(CacheDesc)]
        self.c.unique_page_stats_record_bytes.restype = C.c_int64
        self.c.unique_update_page_stats.argtypes = [C.POINTER(CacheDesc), C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        self.c.unique_score_select_topk.argtypes = [C.POINTER(CacheDesc), C.c_void_p, C.c_int32, C.c_float,
                                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                                                    C.c_void_p]
        self.c.unique_page_scores.argtypes = [C.POINTER(CacheDesc), C.c_void_p, C.c_float, C.c_void_p, C.c_int32,
                                              C.c_void_p]
        self.c.unique_select_topk.argtypes = [C.POINTER(CacheDesc), C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                              C.c_void_p, C.c_void_p]
        self.c.unique_sparse_paged_decode.argtypes = [C.POINTER(CacheDesc), C.c_void_p, C.c_void_p, C.c_void_p,
                                                      C.c_int32, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p,
                                                      C.c_size_t, C.c_void_p]
        self.c.unique_decode_step.argtypes = [C.POINTER(CacheDesc), C.c_void_p, C.c_int32, C.c_float, C.c_float,
                                              C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                              C.c_size_t, C.c_void_p]
        self.c.unique_decode_step_static.argtypes = [C.POINTER(CacheDesc), C.c_void_p, C.c_int32, C.c_float, C.c_float,
                                                     C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                                     C.c_void_p]
        self.c.unique_dense_paged_decode.argtypes = [C.POINTER(CacheDesc), C.c_void_p, C.c_float, C.c_void_p,
                                                     C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]

        desc, ptr, i32 = C.POINTER(CacheDesc), C.c_void_p, C.c_int32
        self.c.unique_page_record_bytes.argtypes = [desc]
        self.c.unique_page_record_bytes.restype = C.c_int64
        self.c.unique_quantise_pages.argtypes = [desc, ptr, ptr, i32, ptr, ptr, C.c_int64, ptr]
        self.c.unique_restore_pages.argtypes = [desc, ptr, ptr, i32, ptr, ptr, C.c_int64, ptr, ptr, ptr]
        self.c.unique_quantised_workspace_bytes.argtypes = [desc, i32, C.POINTER(C.c_size_t)]
        self.c.unique_quantised_paged_decode.argtypes = [desc, ptr, ptr, ptr, ptr, i32, C.c_float, ptr, ptr, ptr, C.c_size_t, ptr]
        self.c.unique_account_workspace_bytes.argtypes = [desc, C.POINTER(C.c_size_t)]
        self.c.unique_weighted_paged_decode.argtypes = [desc, ptr, C.c_float, C.c_float, ptr, ptr, i32, ptr, ptr, ptr, C.c_size_t, ptr]
        self.c.unique_evict_pages.argtypes = [desc, i32, i32, i32, ptr, ptr, i32, ptr, ptr, ptr, ptr, i32, ptr, C.c_size_t, ptr]

    # -- helpers -----------------------------------------------------------------------------
    def check(self, rc: int) -> None:
        if rc != OK:
            raise UniqueError(rc, self.c.unique_status_string(rc).decode(), self.c.unique_last_error().decode())

    def version(self) -> str:
        return self.c.unique_version().decode()

    def last_error(self) -> str:
        return self.c.unique_last_error().decode()

    def status_string(self, rc: int) -> str:
        return self.c.unique_status_string(rc).decode()

    # -- the ABI, one method per entry point ---------------------------------------------------
    def workspace_bytes(self, desc: CacheDesc, top_k: int) -> int:
        n = C.c_size_t(0)
        self.check(self.c.unique_workspace_bytes(C.byref(desc), top_k, C.byref(n)))
        return int(n.value)

    def page_stats_record_bytes(self, desc: CacheDesc) -> int:
        return int(self.c.unique_page_stats_record_bytes(C.byref(desc)))

    def update_page_stats(self, desc: CacheDesc, tok_begin=None, tok_end=None, max_pages_touched_per_seq: int = 0):
        self.check(self.c.unique_update_page_stats(C.byref(desc), _p(tok_begin), _p(tok_end),
                                                   max_pages_touched_per_seq, _stream()))

    def score_select_topk(self, desc: CacheDesc, q, top_k: int, lam: float, sel_pages, sel_count, scores_out,
                          workspace):
        self.check(self.c.unique_score_select_topk(C.byref(desc), _p(q), top_k, lam, _p(sel_pages), _p(sel_count),
                                                   _p(scores_out), _p(workspace),
                                                   workspace.numel() * workspace.element_size(), _stream()))

    def page_scores(self, desc: CacheDesc, q, lam: float, scores):
        self.check(self.c.unique_page_scores(C.byref(desc), _p(q), lam, _p(scores), int(scores.shape[-1]), _stream()))

    def select_topk(self, desc: CacheDesc, scores, top_k: int, sel_pages, sel_count):
        self.check(self.c.unique_select_topk(C.byref(desc), _p(scores), int(scores.shape[-1]), top_k, _p(sel_pages),
                                             _p(sel_count), _stream()))

    def sparse_paged_decode(self, desc: CacheDesc, q, sel_pages, sel_count, sel_stride: int, sm_scale: float, out,
                            lse_out, workspace):
        self.check(self.c.unique_sparse_paged_decode(C.byref(desc), _p(q), _p(sel_pages), _p(sel_count), sel_stride,
                                                     sm_scale, _p(out), _p(lse_out), _p(workspace),
                                                     workspace.numel() * workspace.element_size(), _stream()))

    def decode_step(self, desc: CacheDesc, q, top_k: int, lam: float, sm_scale: float, refresh_tail: bool, sel_pages,
                    sel_count, out, lse_out, workspace):
        self.check(self.c.unique_decode_step(C.byref(desc), _p(q), top_k, lam, sm_scale, int(refresh_tail),
                                             _p(sel_pages), _p(sel_count), _p(out), _p(lse_out), _p(workspace),
                                             workspace.numel() * workspace.element_size(), _stream()))

    def decode_step_static(self, desc: CacheDesc, q, top_k: int, lam: float, sm_scale: float, refresh_tail: bool,
                           sel_pages, sel_count, out, lse_out):
        self.check(self.c.unique_decode_step_static(C.byref(desc), _p(q), top_k, lam, sm_scale, int(refresh_tail),
                                                    _p(sel_pages), _p(sel_count), _p(out), _p(lse_out), _stream()))

    def dense_paged_decode(self, desc: CacheDesc, q, sm_scale: float, out, lse_out, workspace):
        self.check(self.c.unique_dense_paged_decode(C.byref(desc), _p(q), sm_scale, _p(out), _p(lse_out),
                                                    _p(workspace), workspace.numel() * workspace.element_size(),
                                                    _stream()))

    def page_record_bytes(self, desc: CacheDesc) -> int:
        return int(self.c.unique_page_record_bytes(C.byref(desc)))

    def quantised_workspace_bytes(self, desc: CacheDesc, top_k: int) -> int:
        n = C.c_size_t(0)
        self.check(self.c.unique_quantised_workspace_bytes(C.byref(desc), top_k, C.byref(n)))
        return int(n.value)

    def account_workspace_bytes(self, desc: CacheDesc) -> int:
        n = C.c_size_t(0)
        self.check(self.c.unique_account_workspace_bytes(C.byref(desc), C.byref(n)))
        return int(n.value)

    # (written out: a helper per argument costs a microsecond in a call of six)
    def quantise_pages(self, desc: CacheDesc, records, record_table=None, tok_begin=None, tok_end=None,
                       max_pages_touched_per_seq: int = 0):
        rc = self.c.unique_quantise_pages(desc, None if tok_begin is None else tok_begin.data_ptr(),
                                          None if tok_end is None else tok_end.data_ptr(), max_pages_touched_per_seq,
                                          records.data_ptr(), None if record_table is None else record_table.data_ptr(),
                                          records.shape[0], _stream())
        if rc:
            self.check(rc)

    def restore_pages(self, desc: CacheDesc, records, k_out, v_out, record_table=None, tok_begin=None, tok_end=None,
                      max_pages_touched_per_seq: int = 0):
        rc = self.c.unique_restore_pages(desc, None if tok_begin is None else tok_begin.data_ptr(),
                                         None if tok_end is None else tok_end.data_ptr(), max_pages_touched_per_seq,
                                         records.data_ptr(), None if record_table is None else record_table.data_ptr(),
                                         records.shape[0], k_out.data_ptr(), v_out.data_ptr(), _stream())
        if rc:
            self.check(rc)

    def quantised_paged_decode(self, desc: CacheDesc, records, q, sel_pages, sel_count, sm_scale: float, out, lse_out,
                               workspace):
        if sel_pages is None:
            rc = self.c.unique_quantised_paged_decode(desc, records.data_ptr(), q.data_ptr(), None, _p(sel_count), 0, sm_scale,
                                                      out.data_ptr(), _p(lse_out), workspace.data_ptr(), workspace.nbytes, _stream())
        else:
            rc = self.c.unique_quantised_paged_decode(desc, records.data_ptr(), q.data_ptr(), sel_pages.data_ptr(), _p(sel_count),
                                                      sel_pages.shape[-1], sm_scale, out.data_ptr(), _p(lse_out),
                                                      workspace.data_ptr(), workspace.nbytes, _stream())
        if rc:
            self.check(rc)

    def weighted_paged_decode(self, desc: CacheDesc, q, sm_scale: float, decay: float, weights_in, weights_out, out, lse_out,
                              workspace):
        rc = self.c.unique_weighted_paged_decode(desc, q.data_ptr(), sm_scale, decay, _p(weights_in), weights_out.data_ptr(),
                                                 weights_out.shape[-1], out.data_ptr(), _p(lse_out), workspace.data_ptr(),
                                                 workspace.nbytes, _stream())
        if rc:
            self.check(rc)

    def evict_pages(self, desc: CacheDesc, budget_pages: int, sink_pages: int, recent_pages: int, weights_in, weights_out,
                    page_table_out, seq_lens_out, freed_pages, freed_count, workspace):
        rc = self.c.unique_evict_pages(desc, budget_pages, sink_pages, recent_pages, weights_in.data_ptr(), weights_out.data_ptr(),
                                       weights_in.shape[-1], page_table_out.data_ptr(), seq_lens_out.data_ptr(),
                                       freed_pages.data_ptr(), freed_count.data_ptr(), freed_pages.shape[-1], workspace.data_ptr(),
                                       workspace.nbytes, _stream())
        if rc:
            self.check(rc)


_lib: Library | None = None


def load() -> Library:
    """Open the built library (building it first only if no built library exists)."""
    global _lib
    if _lib is None:
        path = _build.LIB_PATH
        if not os.path.exists(path):
            path = _build.build_library()
        _lib = Library(path)
    return _lib


STATIC_SCRATCH_BYTES = 8 << 20  # UNIQUE_STATIC_SCRATCH_BYTES
STD_BLOCK_BYTES = 128  # bytes after the means in a page_stats record (fp32 stds + pad)


def stats_record_bytes(num_kv_heads: int, head_dim: int, stats_dtype) -> int:
    return num_kv_heads * head_dim * (2 if stats_dtype == torch.bfloat16 else 4) + STD_BLOCK_BYTES


def make_desc(*, q_heads: int, k_cache, v_cache, page_stats, page_table, seq_lens,
              max_seq_len_hint: int = 0, stats_dtype=torch.float32, force_recent_pages: int = 0,
              min_seq_len_hint: int = 0) -> CacheDesc:
    """Fill a ``unique_cache_desc`` from tensors laid out as include/unique.h describes (shape checks only)."""
    P, Hkv, S, D = k_cache.shape
    # the (S, D) tile of one (page, head) must be contiguous; page and head strides are passed through
    assert k_cache.dtype in DTYPE_CODE and k_cache.stride()[2:] == (D, 1)
    assert v_cache is None or (v_cache.shape == k_cache.shape and v_cache.dtype == k_cache.dtype
                               and v_cache.stride() == k_cache.stride())
    assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.dim() == 2
    assert seq_lens.dtype == torch.int32 and seq_lens.shape == (page_table.shape[0],)
    if page_stats is not None:
        assert page_stats.dtype == torch.uint8 and page_stats.is_contiguous()
        assert page_stats.shape == (P, stats_record_bytes(Hkv, D, stats_dtype))
    return CacheDesc(DTYPE_CODE[k_cache.dtype], q_heads, Hkv, D, S, page_table.shape[0], page_table.shape[1],
                     max_seq_len_hint, P, k_cache.data_ptr(), 0 if v_cache is None else v_cache.data_ptr(),
                     0 if page_stats is None else page_stats.data_ptr(),
                     page_table.data_ptr(), seq_lens.data_ptr(), DTYPE_CODE[stats_dtype], int(force_recent_pages),
                     k_cache.stride(0), k_cache.stride(1), int(min_seq_len_hint), 0)


def make_shape_desc(*, q_heads: int, kv_heads: int, head_dim: int, page_size: int, dtype, num_pages: int, page_table, seq_lens,
                    max_seq_len_hint: int = 0) -> CacheDesc:
    """A ``unique_cache_desc`` without full-precision pages, for the calls on 4-bit records and on page accounts."""
    assert page_table.dtype == torch.int32 and page_table.is_contiguous() and page_table.dim() == 2
    assert seq_lens.dtype == torch.int32 and seq_lens.is_contiguous() and seq_lens.shape == (page_table.shape[0],)
    return CacheDesc(DTYPE_CODE[dtype], q_heads, kv_heads, head_dim, page_size, page_table.shape[0], page_table.shape[1],
                     max_seq_len_hint, num_pages, 0, 0, 0, page_table.data_ptr(), seq_lens.data_ptr(), 0, 0, 0, 0, 0, 0)
