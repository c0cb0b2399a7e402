"""Buffer owner for one decode workload: allocates the caller-side device tensors (statistics cache,
selection, outputs, workspace) with torch and forwards to the C ABI through ``binding``. No arithmetic
of the method happens here."""
from __future__ import annotations

import math

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


class PagePool:
    """The free pages of a paged cache, and the places of new tokens: ``place_tokens`` extends ``page_table`` and ``seq_lens`` (the cache's
    own) and says where each row of new tokens goes. ``free_pages`` is a stack of ids with ``free_count`` (one number) in use; by default all of the pool's pages
    are free. ``shared_pages``: how many pages at the beginning of a row belong to someone else and do not go back when its sequence ends.
    ``next_positions``: the positions of the next tokens, for caches that evict pages; without it they are the lengths."""

    def __init__(self, *, q_heads: int, kv_heads: int, head_dim: int, page_size: int, dtype, num_pages: int, page_table, seq_lens, max_new_tokens: int,
                 free_pages=None, free_count=None, shared_pages=None, next_positions=None, lib: binding.Library | None = None):
        assert page_table.is_cuda, "the page table must live on the GPU"
        self.lib = lib or binding.load()
        dev, B, self._device = page_table.device, page_table.shape[0], page_table.get_device()
        self.page_table, self.seq_lens, self.shared_pages, self.next_positions = page_table, seq_lens, shared_pages, next_positions
        self.desc = binding.make_shape_desc(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, page_size=page_size, dtype=dtype,
                                            num_pages=num_pages, page_table=page_table, seq_lens=seq_lens)
        assert (free_pages is None) == (free_count is None), "a stack and its size, or neither"
        if free_pages is None:
            free_pages = torch.arange(num_pages, device=dev, dtype=torch.int32)
            free_count = torch.full((1,), num_pages, device=dev, dtype=torch.int32)
        self.free_pages, self.free_count = free_pages, free_count
        i32 = dict(device=dev, dtype=torch.int32)
        self.token_starts, self.placed = torch.zeros((B + 1,), **i32), torch.zeros((B,), **i32)
        self.positions = torch.full((max_new_tokens,), -1, **i32)
        self.slots = torch.full((max_new_tokens,), -1, device=dev, dtype=torch.int64)
        self._batch, self._table_shape = (B,), tuple(page_table.shape)
        for t, shape in ((seq_lens, self._batch), (free_count, (1,)), (shared_pages, self._batch), (next_positions, self._batch)):
            self._check(t, shape)
        self._check(free_pages, tuple(free_pages.shape[:1]))
        p = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
        self._place = binding.Placement(shared_pages=p(shared_pages), next_positions=p(next_positions), free_pages=p(free_pages),
                                        free_count=p(free_count), free_count_out=p(free_count), page_table_out=p(page_table),
                                        seq_lens_out=p(seq_lens), next_positions_out=p(next_positions), placed=p(self.placed),
                                        token_starts=p(self.token_starts), positions=p(self.positions), slots=p(self.slots),
                                        free_capacity=free_pages.shape[0], max_new_tokens=max_new_tokens)
        self.workspace = torch.empty((self.lib.place_workspace_bytes(self.desc, max_new_tokens),), device=dev, dtype=torch.uint8)

    def _check(self, t, shape):
        assert t is None or (t.get_device() == self._device and t.dtype is torch.int32 and t.is_contiguous() and t.shape == shape)

    def place_tokens(self, new_tokens, freed_pages=None, freed_count=None, page_table_out=None, seq_lens_out=None, next_positions_out=None,
                     free_count_out=None):
        """``new_tokens`` [batch]: how many each sequence gets, negative: it has ended. ``freed_pages`` and ``freed_count``: what an eviction left, which
        goes back first. In place by default; outputs that are given are written instead (a page table that is given must hold the
        table's entries: only those that change are written). -> ``positions``, ``slots``, ``token_starts``, ``placed`` (the same tensors every time)."""
        assert _current_device() == self._device
        self._check(new_tokens, self._batch)
        place = binding.Placement.from_buffer_copy(self._place)
        place.new_tokens = new_tokens.data_ptr()
        if freed_pages is not None:
            self._check(freed_pages, (self._batch[0], freed_pages.shape[-1]))
            self._check(freed_count, self._batch)
            place.freed_pages, place.freed_count, place.freed_stride = freed_pages.data_ptr(), freed_count.data_ptr(), freed_pages.shape[1]
        else:
            assert freed_count is None, "counts without pages"
        if page_table_out is not None:
            self._check(page_table_out, self._table_shape)
            place.page_table_out = page_table_out.data_ptr()
        if seq_lens_out is not None:
            self._check(seq_lens_out, self._batch)
            place.seq_lens_out = seq_lens_out.data_ptr()
        if next_positions_out is not None:
            assert self.next_positions is not None, "positions of their own are wanted from the beginning or not at all"
            self._check(next_positions_out, self._batch)
            place.next_positions_out = next_positions_out.data_ptr()
        if free_count_out is not None:
            self._check(free_count_out, (1,))
            place.free_count_out = free_count_out.data_ptr()
        self.lib.place_tokens(self.desc, place, self.workspace)
        return self.positions, self.slots, self.token_starts, self.placed


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, factor: float = 1.0, trained_len: int = 0, low_turns: float = 1.0,
                       high_turns: float = 32.0):
    """Angle per position of each channel pair, ``base ** (-2 i / rotary_dim)``, float64 [rotary_dim / 2] on the host. For contexts ``factor`` times as long as
    those trained on: without ``trained_len`` all positions are divided by ``factor``; with it only pairs that turn less than ``low_turns`` times over
    ``trained_len`` positions, those that turn ``high_turns`` times or more are left, and between them the two are mixed in proportion to the turns."""
    assert rotary_dim >= 0 and rotary_dim % 2 == 0 and base > 0 and factor > 0 and trained_len >= 0 and high_turns > low_turns
    f = float(base) ** (-2.0 * torch.arange(rotary_dim // 2, dtype=torch.float64) / max(rotary_dim, 1))
    if trained_len == 0:
        return f / factor
    keep = ((trained_len * f / (2.0 * math.pi) - low_turns) / (high_turns - low_turns)).clamp(0.0, 1.0)
    return keep * f + (1.0 - keep) * f / factor


class CacheWriter:
    """Writes new tokens into a paged cache: queries and keys normalised per head (where there are weights), turned by their positions (where there are
    ``frequencies``, float64, see ``rotary_frequencies``; sines and cosines are multiplied by ``magnitude``), keys and values to their slots."""

    def __init__(self, *, q_heads: int, k_cache, v_cache, q_weight=None, k_weight=None, eps: float = 1e-6, frequencies=None, magnitude: float = 1.0,
                 interleaved: bool = False, lib: binding.Library | None = None):
        assert k_cache.is_cuda, "the cache must live on the GPU"
        self.lib = lib or binding.load()
        self._device, dev = k_cache.get_device(), k_cache.device
        P, Hkv, S, D = k_cache.shape
        assert k_cache.dtype in binding.DTYPE_CODE and k_cache.stride()[2:] == (D, 1)
        assert v_cache.shape == k_cache.shape and v_cache.dtype is k_cache.dtype and v_cache.stride() == k_cache.stride()
        assert v_cache.get_device() == self._device
        self.k_cache, self.v_cache, self.dtype = k_cache, v_cache, k_cache.dtype
        self.desc = binding.CacheDesc(binding.DTYPE_CODE[k_cache.dtype], q_heads, Hkv, D, S, 1, 1, 0, P, k_cache.data_ptr(), v_cache.data_ptr(), 0, 0, 0,
                                      0, 0, k_cache.stride(0), k_cache.stride(1), 0, 0)
        assert (q_weight is None) == (k_weight is None), "weights of both or of neither"
        for w in (q_weight, k_weight):
            assert w is None or (w.get_device() == self._device and w.dtype is self.dtype and w.is_contiguous() and w.shape == (D,))
        self.weights = q_weight, k_weight
        self.frequencies = torch.empty((0,), device=dev, dtype=torch.float64) if frequencies is None else frequencies.to(dev).contiguous()
        assert self.frequencies.dtype is torch.float64 and self.frequencies.dim() == 1, "angles of far positions need 64 bits"
        self._q_shape, self._kv_shape = (q_heads, D), (Hkv, D)
        R = 2 * self.frequencies.shape[0]
        assert R % 16 == 0 and R <= D
        self._transform = binding.HeadTransform(0 if q_weight is None else q_weight.data_ptr(), 0 if k_weight is None else k_weight.data_ptr(),
                                                self.frequencies.data_ptr() if R else 0, eps, magnitude, R, int(interleaved))

    def append_tokens(self, q, k, v, positions, slots, q_out=None):
        """Rows of heads ``q`` [rows, q_heads, D], ``k`` and ``v`` [rows, kv_heads, D], each row's heads packed (parts of wider rows are fine), to the
        ``slots`` and positions that ``PagePool.place_tokens`` gives. Rows whose slot is negative are left out. -> ``q_out`` (``q`` itself is allowed if
        it is contiguous; by default a new tensor, zero in rows that are left out)."""
        rows = slots.shape[0]
        assert _current_device() == self._device == q.get_device() == k.get_device() == v.get_device()
        assert q.dtype is k.dtype is v.dtype is self.dtype
        assert q.shape == (rows, *self._q_shape) and k.shape == v.shape == (rows, *self._kv_shape)
        for x in (q, k, v):
            stride = x.stride()
            assert stride[2] == 1 and (stride[1] == x.shape[2] or x.shape[1] == 1)
        assert positions.get_device() == slots.get_device() == self._device and positions.dtype is torch.int32 and slots.dtype is torch.int64
        assert positions.shape == slots.shape == (rows,) and positions.is_contiguous() and slots.is_contiguous()
        if q_out is None:
            q_out = torch.zeros((rows, *self._q_shape), device=q.device, dtype=self.dtype)
        else:
            assert q_out.get_device() == self._device and q_out.dtype is self.dtype and q_out.is_contiguous() and q_out.shape == q.shape
        self.lib.append_tokens(self.desc, q, k, v, positions, slots, self._transform, q_out)
        return q_out


class PrefixGroups:
    """Sequences of a paged cache whose contexts begin with the same pages, and attention over such a batch: group ``g`` has the members
    ``members[group_starts[g]:group_starts[g + 1]]`` (without ``members`` the sequences of these numbers), whose rows of ``page_table`` begin with the same
    ``prefix_pages[g]`` full pages. The bounds must be true: at most ``max_members`` of a group, ``max_prefix_pages`` pages of a prefix and, if it is
    known, ``max_own_tokens`` tokens of any member behind its prefix (without it, as many as a row of ``page_table`` or ``max_seq_len`` has room for: a small batch in a wide table is
    then served as a large one, two sequences of 300 tokens in 13 instead of 7 us)."""

    def __init__(self, *, q_heads: int, k_cache, v_cache, page_table, seq_lens, group_starts, prefix_pages, members=None, max_members: int,
                 max_prefix_pages: int, max_own_tokens: int = 0, max_seq_len: int = 0, lib: binding.Library | None = None):
        assert k_cache.is_cuda, "the cache must live on the GPU"
        self.lib = lib or binding.load()
        self._device, dev = k_cache.get_device(), k_cache.device
        self.desc = binding.make_desc(q_heads=q_heads, k_cache=k_cache, v_cache=v_cache, page_stats=None, page_table=page_table, seq_lens=seq_lens,
                                      max_seq_len_hint=max_seq_len)
        B, n = page_table.shape[0], prefix_pages.shape[0]
        for t, shape in ((page_table, page_table.shape), (seq_lens, (B,)), (group_starts, (n + 1,)), (prefix_pages, (n,)), (members, None)):
            assert t is None or (t.get_device() == self._device and t.dtype is torch.int32 and t.is_contiguous() and shape in (None, t.shape))
        assert v_cache.get_device() == self._device and (members is None or (members.dim() == 1 and members.shape[0] >= B))
        self._held = k_cache, v_cache, page_table, seq_lens, group_starts, prefix_pages, members
        S = k_cache.shape[2]
        self.groups = binding.PrefixGroupsDesc(group_starts.data_ptr(), 0 if members is None else members.data_ptr(), prefix_pages.data_ptr(), n,
                                               max_members, max_prefix_pages, -(-max_own_tokens // S))
        self.dtype, self._q_shape = k_cache.dtype, (B, q_heads, k_cache.shape[3])
        self.out = torch.zeros(self._q_shape, device=dev, dtype=self.dtype)
        self.lse = torch.zeros((B, q_heads), device=dev, dtype=torch.float32)
        self.workspace = torch.empty((self.lib.shared_prefix_workspace_bytes(self.desc, self.groups),), device=dev, dtype=torch.uint8)

    def paged_decode(self, q, sm_scale: float = 0.0):
        """Attention of one new token per sequence over all of its pages. -> ``out``, ``lse`` (the same tensors every time; rows of sequences that
        no group lists stay as they are)."""
        assert _current_device() == self._device == q.get_device()
        assert q.dtype is self.dtype and q.is_contiguous() and q.shape == self._q_shape
        self.lib.shared_prefix_decode(self.desc, self.groups, q, sm_scale, self.out, self.lse, self.workspace)
        return self.out, self.lse
