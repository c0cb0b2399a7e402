"""Buffer owner for one decode workload: allocates the caller-side device tensors (statistics cache,
selection, outputs, workspace) with torch and forwards to the C ABI through ``binding``. No arithmetic
of the method happens here."""
from __future__ import annotations

import torch

from . import binding
from .workloads import Workload


class DecodeSession:
    def __init__(self, wl: Workload, top_k: int | None = None, max_seq_len_hint: int | None = None,
                 want_scores: bool = True, lib: binding.Library | None = None, stats_dtype=torch.float32,
                 force_recent_pages: int = 0, min_seq_len_hint: int | None = None, track_weights: bool = False):
        assert wl.k_cache.is_cuda, "the workload must live on the GPU"
        self.lib = lib or binding.load()
        self.wl = wl
        self.top_k = int(top_k if top_k is not None else wl.top_k)
        dev = wl.k_cache.device
        P = wl.num_phys_pages
        self.stats_dtype = stats_dtype
        rec = binding.stats_record_bytes(wl.Hkv, wl.D, stats_dtype)
        mean_bytes = rec - binding.STD_BLOCK_BYTES
        # one record per physical page, every byte 0xFF (NaN in fp32 and in bf16) until a kernel writes it
        self.page_stats = torch.full((P, rec), 0xFF, device=dev, dtype=torch.uint8)
        # views into the records: means [P, Hkv, D] (fp32 or bf16) and stds [P, Hkv] (fp32)
        self.page_mean = self.page_stats[:, :mean_bytes].view(stats_dtype).view(P, wl.Hkv, wl.D)
        self.page_std = self.page_stats[:, mean_bytes:mean_bytes + 4 * wl.Hkv].view(torch.float32)
        self.page_pad = self.page_stats[:, mean_bytes + 4 * wl.Hkv:]
        if max_seq_len_hint is None:
            max_seq_len_hint = int(wl.seq_lens.max().item()) + int(wl.meta.get("spare_tokens", 0))
        if min_seq_len_hint is None:
            # Today's shortest is a lower bound as long as sequences only grow. Where pages have accounts they may be evicted: no bound is known
            # then (a caller whose budget gives one can say so).
            min_seq_len_hint = 0 if track_weights else min(int(wl.seq_lens.min().item()), max_seq_len_hint)
        self.desc = binding.make_desc(q_heads=wl.H, k_cache=wl.k_cache, v_cache=wl.v_cache,
                                      page_stats=self.page_stats, stats_dtype=stats_dtype,
                                      page_table=wl.page_table, seq_lens=wl.seq_lens,
                                      max_seq_len_hint=max_seq_len_hint, min_seq_len_hint=min_seq_len_hint,
                                      force_recent_pages=force_recent_pages)
        self.force_recent_pages = int(force_recent_pages)
        self.sel_pages = torch.full((wl.B, wl.Hkv, self.top_k), -7, device=dev, dtype=torch.int32)
        self.sel_count = torch.full((wl.B, wl.Hkv), -7, device=dev, dtype=torch.int32)
        self.scores = (torch.full((wl.B, wl.Hkv, wl.max_pages), float("nan"), device=dev, dtype=torch.float32)
                       if want_scores else None)
        self.out = torch.zeros((wl.B, wl.H, wl.D), device=dev, dtype=wl.dtype)
        self.lse = torch.zeros((wl.B, wl.H), device=dev, dtype=torch.float32)
        self.out_dense = torch.zeros_like(self.out)
        self.lse_dense = torch.zeros_like(self.lse)
        assert self.lib.page_stats_record_bytes(self.desc) == self.page_stats.shape[1]
        self.workspace_bytes = self.lib.workspace_bytes(self.desc, self.top_k)
        self.page_weights = None
        if track_weights:  # accounts of the pages for weighted_paged_decode
            self.page_weights = torch.zeros((wl.B, wl.Hkv, wl.max_pages), device=dev, dtype=torch.float32)
            self.workspace_bytes = max(self.workspace_bytes, self.lib.account_workspace_bytes(self.desc))
        self.workspace = torch.empty((max(self.workspace_bytes, 256),), device=dev, dtype=torch.uint8)
        assert self.workspace.data_ptr() % 256 == 0

    # one method per entry point, same names
    def update_page_stats(self, tok_begin=None, tok_end=None, max_pages_touched_per_seq: int = 0):
        self.lib.update_page_stats(self.desc, tok_begin, tok_end, max_pages_touched_per_seq)

    def score_select_topk(self, lam: float | None = None):
        self.lib.score_select_topk(self.desc, self.wl.q, self.top_k, self.wl.lam if lam is None else lam,
                                   self.sel_pages, self.sel_count, self.scores, self.workspace)

    def page_scores(self, scores, lam: float | None = None):
        self.lib.page_scores(self.desc, self.wl.q, self.wl.lam if lam is None else lam, scores)

    def select_topk(self, scores):
        self.lib.select_topk(self.desc, scores, self.top_k, self.sel_pages, self.sel_count)

    def sparse_paged_decode(self, sm_scale: float = 0.0, sel_pages=None, sel_count=None):
        sel_pages = self.sel_pages if sel_pages is None else sel_pages
        sel_count = self.sel_count if sel_count is None else sel_count
        self.lib.sparse_paged_decode(self.desc, self.wl.q, sel_pages, sel_count, int(sel_pages.shape[-1]), sm_scale,
                                     self.out, self.lse, self.workspace)

    def decode_step(self, refresh_tail: bool = True, sm_scale: float = 0.0, lam: float | None = None):
        self.lib.decode_step(self.desc, self.wl.q, self.top_k, self.wl.lam if lam is None else lam, sm_scale,
                             refresh_tail, self.sel_pages, self.sel_count, self.out, self.lse, self.workspace)

    def decode_step_static(self, refresh_tail: bool = True, sm_scale: float = 0.0, lam: float | None = None):
        self.lib.decode_step_static(self.desc, self.wl.q, self.top_k, self.wl.lam if lam is None else lam, sm_scale,
                                    refresh_tail, self.sel_pages, self.sel_count, self.out, self.lse)

    def dense_paged_decode(self, sm_scale: float = 0.0):
        self.lib.dense_paged_decode(self.desc, self.wl.q, sm_scale, self.out_dense, self.lse_dense, self.workspace)

    def weighted_paged_decode(self, sm_scale: float = 0.0, decay: float = 1.0, weights_in=None, weights_out=None):
        """``dense_paged_decode`` that adds each page's share to its account: ``page_weights``, or from one array to another (an
        output without an input: nothing so far)."""
        assert self.page_weights is not None, "a session made with track_weights=True has the accounts and the workspace"
        assert _current_device() == self.page_weights.get_device()
        if weights_out is None:
            weights_in, weights_out = self.page_weights if weights_in is None else weights_in, self.page_weights
        _check_accounts(self.page_weights.shape, self.page_weights.get_device(), weights_in, weights_out)
        self.lib.weighted_paged_decode(self.desc, self.wl.q, sm_scale, decay, weights_in, weights_out, self.out_dense,
                                       self.lse_dense, self.workspace)

    def sparse_step(self):
        """score + select + sparse decode (statistics assumed current)."""
        self.score_select_topk()
        self.sparse_paged_decode()


def _check_accounts(shape, device: int, *weights):
    for w in weights:
        assert w is None or (w.dtype is torch.float32 and w.is_contiguous() and w.shape == shape and w.get_device() == device)


# Device tensors of the current device are asked for throughout: a host address would fault the GPU, another device's stream fail the
# launch. (Written out in the calls below, where a helper costs as much as what it checks.)
_current_device = torch._C._cuda_getDevice


class QuantisedCache:
    """A pool of 4-bit page records with its page table: tokens go in from full-precision pages, come back out of it, and are
    attended to in it. ``records`` may be given (uint8, ``num_pages`` records in all); ``top_k`` is the longest list of
    pages that ``paged_decode`` will be given."""

    def __init__(self, *, q_heads: int, kv_heads: int, head_dim: int, page_size: int, dtype, num_pages: int, page_table, seq_lens,
                 max_seq_len: int = 0, top_k: int = 0, records=None, lib: binding.Library | None = None):
        assert page_table.is_cuda, "the page table must live on the GPU"
        self.lib = lib or binding.load()
        dev, self._device = page_table.device, page_table.get_device()
        assert _current_device() == self._device == seq_lens.get_device() and (records is None or records.get_device() == self._device)
        self.page_table, self.seq_lens, self.dtype = page_table, seq_lens, dtype
        self.desc = binding.make_shape_desc(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, page_size=page_size, dtype=dtype,
                                            num_pages=num_pages, page_table=page_table, seq_lens=seq_lens, max_seq_len_hint=max_seq_len)
        record = self.lib.page_record_bytes(self.desc)
        if records is None:
            records = torch.zeros((num_pages, record), device=dev, dtype=torch.uint8)
        assert records.dtype == torch.uint8 and records.is_contiguous() and records.shape[0] == num_pages
        assert records.numel() == num_pages * record
        self.records = records
        self._tile, self._table_shape = (kv_heads, page_size, head_dim), tuple(page_table.shape)
        self._out_shape = (page_table.shape[0], q_heads, head_dim)
        B = page_table.shape[0]
        self.out = torch.zeros(self._out_shape, device=dev, dtype=dtype)
        self.lse = torch.zeros((B, q_heads), device=dev, dtype=torch.float32)
        self.workspace = torch.empty((self.lib.quantised_workspace_bytes(self.desc, top_k),), device=dev, dtype=torch.uint8)

    def _full_desc(self, k, v, table):
        """The descriptor with full-precision pages instead of the pool (a copy: a third of the time of ``binding.make_desc``)."""
        shape = k.shape
        assert _current_device() == self._device == k.get_device() == v.get_device()
        assert k.dtype is v.dtype is self.dtype and shape[1:] == self._tile and v.shape == shape
        d = binding.CacheDesc.from_buffer_copy(self.desc)
        d.num_phys_pages, d.k_cache, d.v_cache = shape[0], k.data_ptr(), v.data_ptr()
        if not (k.is_contiguous() and v.is_contiguous()):
            stride = k.stride()
            assert v.stride() == stride and stride[2:] == (self._tile[2], 1) and stride[0] and stride[1]  # (0 would stand for the default)
            d.kv_page_stride, d.kv_head_stride = stride[:2]
        if table is not None:
            assert table.get_device() == self._device and table.dtype is torch.int32
            assert table.is_contiguous() and table.shape == self._table_shape
            d.page_table = table.data_ptr()
        return d

    def quantise_pages(self, k_cache, v_cache, page_table=None, tok_begin=None, tok_end=None, max_pages_touched_per_seq: int | None = None):
        """Tokens of full-precision pages, found by ``page_table`` (default: the pool's own), into records: all, or those of a range of
        each sequence. ``max_pages_touched_per_seq`` bounds the pages that a range overlaps (those beyond it are left as they are) and so the
        launch; without it a launch is as large as for all tokens."""
        if tok_begin is not None:
            assert tok_begin.get_device() == tok_end.get_device() == self._device and tok_begin.dtype is tok_end.dtype is torch.int32
            assert tok_begin.is_contiguous() and tok_end.is_contiguous() and tok_begin.numel() == tok_end.numel() == self._table_shape[0]
        if max_pages_touched_per_seq is None:
            max_pages_touched_per_seq = self._table_shape[1]
        self.lib.quantise_pages(self._full_desc(k_cache, v_cache, page_table), self.records, self.page_table, tok_begin, tok_end,
                                max_pages_touched_per_seq)

    def restore_pages(self, k_out, v_out, page_table=None, tok_begin=None, tok_end=None, max_pages_touched_per_seq: int | None = None):
        """The values of the records' tokens into full-precision pages."""
        if tok_begin is not None:
            assert tok_begin.get_device() == tok_end.get_device() == self._device and tok_begin.dtype is tok_end.dtype is torch.int32
            assert tok_begin.is_contiguous() and tok_end.is_contiguous() and tok_begin.numel() == tok_end.numel() == self._table_shape[0]
        if max_pages_touched_per_seq is None:
            max_pages_touched_per_seq = self._table_shape[1]
        self.lib.restore_pages(self._full_desc(k_out, v_out, page_table), self.records, k_out, v_out, self.page_table, tok_begin,
                               tok_end, max_pages_touched_per_seq)

    def paged_decode(self, q, sel_pages=None, sel_count=None, sm_scale: float = 0.0):
        """Attention over every page, or over the pages of a selection. -> ``out``, ``lse`` (the same tensors every time)."""
        assert _current_device() == self._device == q.get_device()
        assert q.dtype is self.dtype and q.is_contiguous() and q.shape == self._out_shape
        if sel_pages is not None:
            assert sel_pages.get_device() == sel_count.get_device() == self._device
            assert sel_pages.dtype is sel_count.dtype is torch.int32 and sel_pages.is_contiguous() and sel_count.is_contiguous()
            assert sel_pages.dim() == 3 and sel_pages.shape[:2] == sel_count.shape == (self._out_shape[0], self._tile[0])
        else:
            assert sel_count is None, "counts without lists"
        self.lib.quantised_paged_decode(self.desc, self.records, q, sel_pages, sel_count, sm_scale, self.out, self.lse, self.workspace)
        return self.out, self.lse


class PageAccounts:
    """Accounts of a paged cache's pages, and the policy by which pages with small ones are evicted: a sequence of more than
    ``budget_pages`` keeps its first ``sink_pages``, its last ``recent_pages`` and the best of the others. ``page_table`` and
    ``seq_lens`` are the cache's own, which ``evict_pages`` changes; the ids that it frees are in ``freed_pages`` (-1 behind the
    ``freed_count`` of a sequence)."""

    def __init__(self, *, budget_pages: int, sink_pages: int = 0, recent_pages: int = 1, q_heads: int, kv_heads: int, head_dim: int,
                 page_size: int, dtype, num_pages: int, page_table, seq_lens, max_seq_len: int = 0, weights=None,
                 lib: binding.Library | None = None):
        assert page_table.is_cuda, "the page table must live on the GPU"
        self.lib = lib or binding.load()
        dev, (B, max_pages), self._device = page_table.device, page_table.shape, page_table.get_device()
        assert _current_device() == self._device == seq_lens.get_device()
        self.page_table, self.seq_lens = page_table, seq_lens
        self.policy = (int(budget_pages), int(sink_pages), int(recent_pages))
        self.desc = binding.make_shape_desc(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, page_size=page_size, dtype=dtype,
                                            num_pages=num_pages, page_table=page_table, seq_lens=seq_lens, max_seq_len_hint=max_seq_len)
        self.weights = torch.zeros((B, kv_heads, max_pages), device=dev, dtype=torch.float32) if weights is None else weights
        self._shape = (B, kv_heads, max_pages)
        _check_accounts(self._shape, self._device, self.weights)
        self.freed_pages = torch.full((B, max(max_pages - self.policy[0], 1)), -1, device=dev, dtype=torch.int32)
        self.freed_count = torch.zeros((B,), device=dev, dtype=torch.int32)
        self.workspace = torch.empty((self.lib.account_workspace_bytes(self.desc),), device=dev, dtype=torch.uint8)

    def evict_pages(self, weights_in=None, weights_out=None, page_table_out=None, seq_lens_out=None):
        """In place by default; inputs that are given are read and outputs that are given are written instead of the own arrays (accounts
        given as the input alone stay as they are: what becomes of them goes to ``weights``)."""
        weights_in = self.weights if weights_in is None else weights_in
        weights_out = self.weights if weights_out is None else weights_out
        assert _current_device() == self._device
        _check_accounts(self._shape, self._device, weights_in, weights_out)
        for given, mine in ((page_table_out, self.page_table), (seq_lens_out, self.seq_lens)):
            assert given is None or (given.get_device() == self._device and given.dtype is torch.int32 and given.is_contiguous()
                                     and given.shape == mine.shape)
        self.lib.evict_pages(self.desc, *self.policy, weights_in, weights_out, self.page_table if page_table_out is None else page_table_out,
                             self.seq_lens if seq_lens_out is None else seq_lens_out, self.freed_pages, self.freed_count, self.workspace)
