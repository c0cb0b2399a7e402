"""Kernels of the calls around the cache that small tests do not reach: long runs of rows, large tables, caches beyond 4 GB or 96 MB, many heads, bounds that are too low, and the steps
together with statistics and a sparse decode."""
import random

import pytest
import torch

import oracle
from paper_2605_27740_amd.session import DecodeSession, PagePool
from paper_2605_27740_amd.workloads import Workload
from tests import harness as Hn
from tests import serving_ref as R
from tests import test_serving_gpu as G

pytestmark = pytest.mark.gpu
DEV, DTYPES, i32, say = G.DEV, G.DTYPES, G.i32, G.say
BF16, FP32 = DTYPES


# ------------------------------------------------------------------ places

LONG = [  # sequences, tokens of a page, entries of a row, pages of the long rows, rows: one workgroup, two launches, three
    (20, 8, 2000, (511, 513, 700, 1025, 1999), 100), (30, 8, 20_000, (8191, 8193, 12_000, 17_000), 100), (1100, 16, 5000, (2047, 2049, 4100), 300)]


@pytest.mark.parametrize("B,S,width,long,rows", LONG)
@pytest.mark.parametrize("in_place", [False, True])
def test_long_rows_are_given_back(gpu_lib, B, S, width, long, rows, in_place):
    """Sequences that end with more pages than a workgroup or wave takes at once, beside others; with shared pages and without."""
    say(f"long rows {B} {width} in_place={in_place}")
    r = random.Random(B)
    c, total = G.place_case(B, B, S, 12, 12 * S, 1, 0.0, ended=0.2, evicted=2)
    c["table"] = [row + [-1] * (width - 12) for row in c["table"]]
    c["new"] = [min(t, 1) for t in c["new"]]
    for i, pages in enumerate(long):
        b = i * (B - 1) // (len(long) - 1)
        c["lens"][b], c["new"][b] = pages * S - r.randrange(S), -1
        c["table"][b] = list(range(total, total + pages)) + [-1] * (width - pages)
        c["shared"][b] = r.choice([0, 3, pages - 2])
        total += pages
    for b in range(B // 2, B // 2 + 3):  # and some that go on
        c["new"][b] = 20
    c["free"] = c["free"][:c["free_count"]] + [-7] * total
    c["rows"] = rows
    G.check_place(c, total, in_place=in_place)


# ------------------------------------------------------------------ queries, keys and values

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,Hkv,rows", [(16, 4, 6000), (8, 1, 9001), (4, 4, 7777)])
def test_append_two_steps_a_wave(gpu_lib, dtype, D, interleaved, H, Hkv, rows):
    """More than 8192 steps of heads (4 to 16 heads each), an odd number of them to a token, or heads that do not fill the last."""
    say(f"append {dtype} D={D} interleaved={interleaved} {(H, Hkv, rows)}")
    G.run_append(dtype, H, Hkv, D, 16, rows, rotary=D // 2 if rows % 2 else D, interleaved=interleaved, norm=True, magnitude=1.0, fused=rows % 2 == 0)


@pytest.mark.parametrize("dtype,norm", [(BF16, False), (FP32, True), (FP32, False), (BF16, True)])
@pytest.mark.parametrize("D,interleaved", [(64, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_of_long_prompts(gpu_lib, dtype, norm, D, interleaved, in_place):
    """16384 rows and more: without norm or in fp32 a step a wave, whose heads are asked for behind the slot."""
    say(f"append long {dtype} norm={norm} D={D} interleaved={interleaved} in_place={in_place}")
    G.run_append(dtype, 8, 2, D, 32, 16_500, rotary=D, interleaved=interleaved, norm=norm, magnitude=1.1, fused=not in_place, in_place=in_place)


# ------------------------------------------------------------------ shared prefixes

# Shapes whose prefixes are shared when the table is widened: element type, query heads, KV heads, channels, tokens of a page, members
SHARED = [(BF16, 8, 2, 128, 16, 3), (BF16, 8, 2, 128, 16, 40), (BF16, 8, 2, 64, 16, 3), (BF16, 8, 1, 64, 32, 40), (FP32, 8, 2, 128, 16, 3), (FP32, 8, 1, 64, 32, 40),
          (BF16, 4, 4, 128, 32, 40), (FP32, 2, 2, 128, 8, 5)]
STREAM = 96 << 20  # bytes of keys and values that the host's bounds must pass for loads that spare the caches


def columns_of(B, dtype, Hkv, D, S):
    return (256 << 20) // (B * Hkv * S * D * 2 * (torch.finfo(dtype).bits // 8)) + 768 // S + 1


def in_large_pool(c, dtype, pages):
    """The case's pages as the last ones of a pool of so many, in a table that is wide enough for its prefixes to be shared."""
    P, Hkv, S, D = c["k"].shape
    k, v = (torch.empty((pages, Hkv, S, D), dtype=dtype, device=DEV) for _ in range(2))
    k[-P:], v[-P:] = c["k"].to(DEV), c["v"].to(DEV)
    table = torch.where(c["table"] < 0, -1, c["table"] + (pages - P))
    columns = columns_of(len(c["lens"]), dtype, Hkv, D, S)
    table = torch.nn.functional.pad(table, (0, max(columns - table.shape[1], 0)), value=-1)
    return dict(k_cache=k, v_cache=v, page_table=table.to(DEV))


@pytest.mark.parametrize("dtype,H,Hkv,D,S,members", SHARED)
def test_prefix_streamed(gpu_lib, dtype, H, Hkv, D, S, members):
    """Pools of more than 96 MB, whose keys and values are read past the caches: 64 and 128 rows, both types and head sizes; prefixes of many tiles, members shorter than
    theirs, own pages."""
    say(f"streamed {dtype} {(H, Hkv, D, S, members)}")
    c = G.prefix_case(dtype, H, Hkv, D, S, [([30 + 7 * i if i % 4 else -i for i in range(members)], 1000 // S), ([5, 100], 3)], seed=members)
    page = Hkv * S * D * 2 * (torch.finfo(dtype).bits // 8)
    pages = STREAM // page + c["k"].shape[0] + 5
    G.check_prefix(c, G.make_groups(c, H, **in_large_pool(c, dtype, pages)).paged_decode(c["q"].to(DEV)), dtype)


@pytest.mark.parametrize("dtype,H,Hkv,D,S,members", SHARED[:6])
def test_prefix_shared_far_pages_and_no_lse(gpu_lib, dtype, H, Hkv, D, S, members):
    """Pages of a shared prefix beyond 2^31 elements of the cache and 2^32 bytes; no lse is wanted."""
    say(f"far {dtype} {(H, Hkv, D, S, members)}")
    c = G.prefix_case(dtype, H, Hkv, D, S, [([30, 100, 0] + [9] * (members - 3), 40)], seed=7, poison=False)
    P = c["k"].shape[0]
    groups = G.make_groups(c, H, **in_large_pool(c, dtype, (1 << 31) // (Hkv * S * D) + P + 9))
    q = c["q"].to(DEV)
    G.check_prefix(c, groups.paged_decode(q), dtype)
    want = groups.out.clone()
    groups.out.zero_()
    groups.lse.fill_(-7.0)
    groups.lib.shared_prefix_decode(groups.desc, groups.groups, q, 0.0, groups.out, None, groups.workspace)
    torch.cuda.synchronize()
    assert torch.equal(groups.out, want) and (groups.lse == -7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,Hkv,D,S", [(16, 16, 128, 16), (32, 32, 64, 8), (128, 16, 64, 16), (64, 32, 128, 32)])
def test_prefix_many_kv_heads(gpu_lib, dtype, H, Hkv, D, S):
    say(f"heads {dtype} {(H, Hkv, D, S)}")
    c = G.prefix_case(dtype, H, Hkv, D, S, [([17] * 9, 20), ([1, -2, 3], 4), ([100], 7)], seed=Hkv)
    G.check_both(c, H, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_prefix_bounds_that_are_too_low(gpu_lib, dtype):
    """Of a prefix that is longer than the host's bound, the pages behind that count as own ones, as far as those go."""
    S, first, second = 16, 6, 3
    c = G.prefix_case(dtype, 8, 2, 64, S, [([30, 100, 70, 1], first), ([200, 90], second)], seed=4, poison=False)
    G.check_both(c, 8, dtype, max_prefix_pages=4)
    G.check_both(c, 8, dtype, max_prefix_pages=0)
    for bound in (4, 1):
        lens = c["lens"].clone()
        for members, pages in ((c["members"][:4], first), (c["members"][4:], second)):
            lens[members.long()] = lens[members.long()].clamp(max=(min(pages, bound) + 4) * S)
        d = dict(c, lens=lens)
        want = R.attend(d["q"], d["k"], d["v"], d["table"], lens)
        G.check_prefix(d, G.make_groups(c, 8, max_prefix_pages=bound, max_own_tokens=4 * S).paged_decode(c["q"].to(DEV)), dtype, want)


# ------------------------------------------------------------------ together

class SparseServer(G.Server):
    """A server that decodes by the pages it selects: statistics of the pages that new tokens touch, scores, selection and sparse attention behind placement and append."""

    def __init__(self, seed, dtype, **geo):
        super().__init__(seed, dtype, **geo)
        H, Hkv, D, S, B, _ = self.geo
        self.wl = Workload("server", dtype, B, H, Hkv, D, S, 5, 0.5, self.q, self.kc, self.vc, self.table, self.lens)
        self.sess = DecodeSession(self.wl, max_seq_len_hint=self.table.shape[1] * S, min_seq_len_hint=0)
        self.before = torch.zeros_like(self.lens)
        self.sess.update_page_stats()  # of the prefix

    def step(self):
        self.before.copy_(self.lens)
        super().step()
        self.sess.update_page_stats(self.before, self.lens, 2)
        self.sess.decode_step(refresh_tail=False)

    def check(self):
        super().check()
        H, Hkv, D, S, B, _ = self.geo
        oc, q = Hn.oracle_cache(self.wl)
        sel, count = self.sess.sel_pages.cpu().numpy(), self.sess.sel_count.cpu().numpy()
        for b in range(B):
            if self.lens[b] == 0:
                assert (count[b] == 0).all() and (self.sess.out[b] == 0).all()
                continue
            for h in range(Hkv):
                mean, std = Hn.check_stats_row(self.sess, oc, b, h)
                scores = oracle.page_scores(oc, q, b, h, self.wl.lam, mean, std)
                Hn.check_selection_row(sel[b, h], int(count[b, h]), scores, self.sess.top_k, f"row ({b},{h})")
                for g in range(H // Hkv):
                    Hn.check_attention_head(self.sess.out, self.sess.lse, oc, q, b, h * (H // Hkv) + g, sel[b, h, :count[b, h]], self.dtype, where=f"({b},{h})")


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_server_places_appends_and_decodes_sparsely(gpu_lib, dtype, captured):
    """Placement, append, the dense attention over the shared prefix, page statistics of the touched pages and a decode step, twenty times, against the host's copy and the oracle; eager,
    or one graph replayed."""
    s = SparseServer(31, dtype, H=8, Hkv=2, D=64, S=8, B=5, width=60, pages=300)
    graph = None
    for i in range(20):
        s.inputs(G.asked(s.r, i, s.geo[4]))
        if captured and graph is None and i == 2:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                s.step()
        if graph is not None:
            graph.replay()
        else:
            s.step()
        s.check()
        s.admit()
        if i % 4 == 0:
            (torch.randn((512, 512), device=DEV) @ torch.randn((512, 512), device=DEV)).sum().item()


def test_a_pool_from_nothing_to_nothing(gpu_lib):
    """A pool's first step: nothing but free pages, prompts of one token and of many pages, places, heads, statistics and a decode step; then all end and every page is free."""
    B, S, Hkv, D, pages = 4, 16, 2, 128, 64
    say("from nothing")
    g = torch.Generator().manual_seed(3)
    kc, vc = (torch.zeros((pages, Hkv, S, D), dtype=BF16, device=DEV) for _ in range(2))
    table, lens = torch.full((B, 16), -1, dtype=torch.int32, device=DEV), i32([0] * B)
    pool = PagePool(q_heads=8, kv_heads=Hkv, head_dim=D, page_size=S, dtype=BF16, num_pages=pages, page_table=table, seq_lens=lens, max_new_tokens=600)
    new = [1, 200, 0, 250]
    positions, slots, starts, placed = pool.place_tokens(i32(new))
    assert placed.tolist() == new and lens.tolist() == new
    x = torch.randn((600, 8 + 2 * Hkv, D), generator=g).to(BF16).to(DEV)
    q = G.CacheWriter(q_heads=8, k_cache=kc, v_cache=vc).append_tokens(*x.split([8, Hkv, Hkv], 1), positions, slots)
    last = (starts[1:] - 1).clamp(min=0).long()
    wl = Workload("nothing", BF16, B, 8, Hkv, D, S, 3, 0.5, q[last].contiguous(), kc, vc, table, lens)
    sess = DecodeSession(wl, max_seq_len_hint=256)
    Hn.full_check(wl, sess, rows=[(b, h) for b in (0, 1, 3) for h in range(Hkv)])
    pool.place_tokens(i32([-1] * B))
    torch.cuda.synchronize()
    assert sorted(pool.free_pages.tolist()) == list(range(pages)) and int(pool.free_count) == pages and (table == -1).all() and lens.tolist() == [0] * B
