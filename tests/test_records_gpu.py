"""4-bit page records, attention over them, page accounts and eviction on the GPU against plain 64-bit counterparts (records_ref.py)."""
import itertools
import math

import pytest
import torch

from paper_2605_27740_amd import binding
from paper_2605_27740_amd import workloads as W
from paper_2605_27740_amd.session import DecodeSession, PageAccounts, QuantisedCache
from tests import records_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float32]


def say(*a):
    print(*a, flush=True)


def tables(lens, S, g, spare=3, extra_cols=0):
    """A permuted page table of the sequences, -1 behind their pages; -> table, pages in the pool."""
    pages = [-(-n // S) for n in lens]
    pool = sum(pages) + spare
    ids = torch.randperm(pool, generator=g).int()
    t = torch.full((len(lens), max(max(pages), 1) + extra_cols), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        t[b, :n] = ids[at:at + n]
        at += n
    return t, pool


def geometry(H, Hkv, D, S, dtype, pool, table, lens, **more):
    return dict(q_heads=H, kv_heads=Hkv, head_dim=D, page_size=S, dtype=dtype, num_pages=pool, page_table=table.to(DEV),
                seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV), **more)


# ------------------------------------------------------------------ tokens to records and back

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,S,Hkv", [(128, 16, 8), (64, 8, 2), (128, 32, 1), (64, 32, 4), (128, 8, 32), (64, 16, 16)])
def test_records_are_the_bytes_of_the_format(gpu_lib, dtype, D, S, Hkv):
    """Every token of odd lengths, then ranges that begin and end inside pages: bytes of other tokens and of unused pages stay."""
    say(f"quantise {dtype} D={D} S={S} Hkv={Hkv}")
    g = torch.Generator().manual_seed(D + S + Hkv)
    lens = [3 * S + 5, 1, 0, 2 * S, S - 1]
    table, pool = tables(lens, S, g)
    k, v = (torch.randn((pool, Hkv, S, D), generator=g).to(dtype) for _ in range(2))
    k[..., 5] *= 100
    want = torch.full((pool, Hkv, R.tile_bytes(S, D)), 0xA5, dtype=torch.uint8)
    k2, v2 = (torch.randn((pool, Hkv, S, D), generator=g).to(dtype) for _ in range(2))
    begin, end = [S // 2, 0, 0, S - 1, 2], [2 * S + 3, 9, 5, S + 1, 2]
    for turn, (kk, vv, lo, hi) in enumerate(((k, v, [0] * 5, lens), (k2, v2, begin, end))):
        (kc, ks), (vc, vs) = R.encode(kk), R.encode(vv)
        for b, n in enumerate(lens):
            for t in range(lo[b], min(hi[b], n)):
                ph = int(table[b, t // S])
                for h in range(Hkv):
                    at = ph, h, t % S
                    R.write_token(want[ph, h], S, D, t % S, kc[at], ks[at], vc[at], vs[at])
        if turn == 0:
            cache = QuantisedCache(records=torch.full((pool, Hkv * R.tile_bytes(S, D)), 0xA5, dtype=torch.uint8, device=DEV),
                                   **geometry(Hkv, Hkv, D, S, dtype, pool, table, lens))
            cache.quantise_pages(kk.to(DEV), vv.to(DEV))
        else:
            cache.quantise_pages(kk.to(DEV), vv.to(DEV), None, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lo, hi)), 4)
        torch.cuda.synchronize()
        assert torch.equal(cache.records.cpu().view(want.shape), want), f"turn {turn}"

    ko, vo = (torch.full((pool, Hkv, S, D), -77.0, dtype=dtype, device=DEV) for _ in range(2))
    kx, vx = (x.view(pool, Hkv, S, D) for x in R.values_of(want.flatten(0, 1), S, D))
    for lo, hi, ranged in (([S // 2, 0, 0, 1, 0], [S + 1, 1, 1, 2 * S, 1], True), ([0] * 5, lens, False)):
        if ranged:
            cache.restore_pages(ko, vo, None, *(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lo, hi)), 3)
        else:
            cache.restore_pages(ko, vo)
        torch.cuda.synchronize()
        mine = torch.zeros((pool, 1, S, 1), dtype=torch.bool)
        for b, n in enumerate(lens):
            for t in range(lo[b], min(hi[b], n)):
                mine[int(table[b, t // S]), 0, t % S] = True
        for got, ref in ((ko, kx), (vo, vx)):
            assert torch.equal(got.cpu().double(), torch.where(mine, ref, torch.full((), -77.0, dtype=torch.float64)))


@pytest.mark.parametrize("dtype", DTYPES)
def test_records_of_extreme_values(gpu_lib, dtype):
    """Zeros of both signs, denormals, the largest numbers, ties between levels, blocks with infinities and NaN."""
    D, S, Hkv = 128, 8, 1
    x = torch.zeros((1, 1, S, D))
    g = torch.Generator().manual_seed(0)
    x[0, 0, 0] = torch.randn(D, generator=g) * 1e-40
    x[0, 0, 1] = torch.randn(D, generator=g) * 1e38
    x[0, 0, 1, :4] = torch.tensor([torch.finfo(dtype).max, -torch.finfo(dtype).max, 1e-30, -0.0])
    x[0, 0, 2] = torch.linspace(-8, 8, D)
    x[0, 0, 3, ::3] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.75, -0.25, -5.0]).repeat(4)[:43]
    x[0, 0, 4] = 1.0
    x[0, 0, 4, 7], x[0, 0, 4, 40], x[0, 0, 4, 100] = float("inf"), float("nan"), float("-inf")
    x[0, 0, 5] = torch.pow(2.0, torch.arange(D) - 100.0)
    x = x.to(dtype)
    table = torch.zeros((1, 1), dtype=torch.int32)
    cache = QuantisedCache(**geometry(1, 1, D, S, dtype, 1, table, [6]))
    cache.quantise_pages(x.to(DEV), x.to(DEV))
    k, v = (torch.zeros((1, 1, S, D), dtype=dtype, device=DEV) for _ in range(2))
    cache.restore_pages(k, v)
    torch.cuda.synchronize()
    want = R.values(*R.encode(x))
    want[:, :, 6:] = 0
    for got in (k, v):
        got = got.cpu().double()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def test_two_tables_strides_and_pages_outside_the_pools(gpu_lib):
    """Full-precision pages that exist for the last tokens only, K and V side by side in one buffer; ids outside either pool are skipped."""
    D, S, Hkv, lens = 128, 16, 4, [70, 33, 129]
    g = torch.Generator().manual_seed(1)
    table, pool = tables(lens, S, g, extra_cols=2)
    stage = torch.full_like(table, -1)
    stage[0, 3:5], stage[1, 1:3], stage[2, 8] = torch.tensor([4, 0]), torch.tensor([3, 99]), 1  # 99: not a page
    table[0, 4] = pool + 5                                                                   # not a record
    kv = torch.randn((6, Hkv, 2, S, D), generator=g).bfloat16().to(DEV)
    k, v = kv[:, :, 0], kv[:, :, 1]
    geo = geometry(8, Hkv, D, S, torch.bfloat16, pool, table, lens)
    cache = QuantisedCache(**geo)
    cache.quantise_pages(k, v, stage.to(DEV))
    out = torch.zeros_like(kv)
    cache.restore_pages(out[:, :, 0], out[:, :, 1], stage.to(DEV))
    torch.cuda.synchronize()
    want = torch.zeros((6, Hkv, 2, S, D), dtype=torch.float64)
    for ph, n in ((4, 16), (3, 16), (1, 1)):  # (page 0 has no record, 99 does not exist)
        want[ph, :, :, :n] = R.values(*R.encode(kv[ph].cpu()))[:, :, :n]
    assert torch.equal(out.cpu().double(), want)
    written = {int(table[0, 3]), int(table[1, 1]), int(table[2, 8])}
    assert {i for i in range(pool) if cache.records[i].any()} == written


# ------------------------------------------------------------------ attention over records

def random_records(pool, Hkv, S, D, g, device="cpu"):
    """Any codes, scales of 2^-3 to 2^1 and now and then 2^-20: what quantising gives, and a bit more."""
    n = R.tile_bytes(S, D)
    rec = torch.randint(0, 256, (pool, Hkv, n), generator=g, dtype=torch.uint8, device=device)
    rec[..., S * D:] = rec[..., S * D:] % 5 + 124
    rec[..., S * D + 3::17] = 107
    return rec


def check_decode(cache, rec, q, table, lens, Hkv, S, D, lists=None, scale=None, rows=None):
    """out and lse of `rows` (all: None) against 64 bits."""
    out, lse = cache.out.cpu().double(), cache.lse.cpu().double()
    H, dtype = q.shape[1], q.dtype
    G = H // Hkv
    scale = 1 / math.sqrt(D) if scale is None else scale
    for b, h in rows or itertools.product(range(len(lens)), range(Hkv)):
        P = -(-lens[b] // S)
        pages = range(P) if lists is None else [p for p in lists[b][h] if 0 <= p < P]
        pages = [p for p in pages if 0 <= int(table[b, p]) < rec.shape[0]]
        if pages:
            ids = table[b, pages].long()
            k, v = R.values_of(rec[ids.to(rec.device), h].cpu(), S, D)
            tok = (torch.tensor(pages)[:, None] * S + torch.arange(S)).reshape(-1) < lens[b]
            k, v = k.reshape(-1, D)[tok], v.reshape(-1, D)[tok]
        else:
            k = v = torch.zeros((0, D))
        a = R.Attended(q[b, h * G:(h + 1) * G].cpu(), k, v, scale)
        got = out[b, h * G:(h + 1) * G]
        part = 2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -23
        tol = a.out_tolerance(dtype, part)
        assert (got - a.out).abs().le(tol).all(), (b, h, ((got - a.out).abs() / tol).max())
        if len(k) == 0:
            assert (got == 0).all() and (lse[b, h * G:(h + 1) * G] == -math.inf).all()
        else:
            assert (lse[b, h * G:(h + 1) * G] - a.lse).abs().le(a.slack + 2.0 ** -22 * a.lse.abs()).all(), (b, h)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("D,S", [(128, 16), (64, 8), (128, 8), (64, 32), (128, 32), (64, 16)])
def test_decode_over_records(gpu_lib, dtype, G, D, S):
    """Lengths from nothing to some hundred pages; slots that hold no token carry codes and scales of NaN."""
    Hkv = 2 if G > 2 else 8
    lens = [0, 1, S - 1, S, 5 * S + 3, 33 * S + 1, 301 * S - 2]
    say(f"decode over records {dtype} G={G} D={D} S={S}")
    g = torch.Generator().manual_seed(G * 1000 + D + S)
    table, pool = tables(lens, S, g)
    rec = random_records(pool, Hkv, S, D, g)
    for b, n in enumerate(lens):
        if n % S:
            tile = rec[int(table[b, n // S])]
            for i in range(2 * (D // 32)):
                tile[:, S * D + i * S + n % S:S * D + (i + 1) * S] = 255
    unused = set(range(pool)) - set(table[table >= 0].tolist())
    rec[sorted(unused)] = 255
    q = torch.randn((len(lens), Hkv * G, D), generator=g).to(dtype)
    cache = QuantisedCache(records=rec.to(DEV).view(pool, -1), **geometry(Hkv * G, Hkv, D, S, dtype, pool, table, lens))
    cache.out.fill_(7), cache.lse.fill_(7)
    cache.paged_decode(q.to(DEV))
    torch.cuda.synchronize()
    check_decode(cache, rec, q, table, lens, Hkv, S, D)
    first = cache.out.clone(), cache.lse.clone()
    cache.paged_decode(q.to(DEV))
    assert torch.equal(first[0], cache.out) and torch.equal(first[1], cache.lse)
    cache.paged_decode(q.to(DEV), sm_scale=0.37)
    torch.cuda.synchronize()
    check_decode(cache, rec, q, table, lens, Hkv, S, D, scale=0.37)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("G,D,S,top_k", [(4, 128, 16, 40), (8, 64, 8, 7), (1, 128, 32, 130), (2, 64, 16, 1), (8, 128, 8, 300)])
def test_decode_over_lists_of_records(gpu_lib, dtype, G, D, S, top_k):
    """Lists in any order with entries that are no pages, counts from none to more than the sequence has, and one table entry outside the pool."""
    Hkv, lens = 4, [0, 3, 9 * S + 1, 200 * S - 1]
    g = torch.Generator().manual_seed(top_k)
    table, pool = tables(lens, S, g)
    table[3, 5] = pool
    rec = random_records(pool, Hkv, S, D, g)
    q = torch.randn((4, Hkv * G, D), generator=g).to(dtype)
    sel = torch.full((4, Hkv, top_k), -1, dtype=torch.int32)
    count = torch.randint(0, top_k + 1, (4, Hkv), generator=g, dtype=torch.int32)
    count[3, 0], count[3, 1] = 0, top_k
    for b, h in itertools.product(range(4), range(Hkv)):
        some = torch.randperm(220, generator=g)[:top_k] - 5  # -5 .. 214, pages or not
        sel[b, h, :some.numel()] = some.int()
    cache = QuantisedCache(records=rec.to(DEV).view(pool, -1), top_k=top_k, **geometry(Hkv * G, Hkv, D, S, dtype, pool, table, lens))
    cache.paged_decode(q.to(DEV), sel.to(DEV), count.to(DEV))
    torch.cuda.synchronize()
    lists = [[sel[b, h, :count[b, h]].tolist() for h in range(Hkv)] for b in range(4)]
    check_decode(cache, rec, q, table, lens, Hkv, S, D, lists=lists)


def test_every_page_listed_is_every_page(gpu_lib):
    """The same attention as a list and as a whole, within the rounding of sums in another order."""
    Hkv, G, D, S, lens = 2, 4, 128, 16, [5000, 77]
    g = torch.Generator().manual_seed(4)
    table, pool = tables(lens, S, g)
    rec = random_records(pool, Hkv, S, D, g)
    q = torch.randn((2, Hkv * G, D), generator=g).to(DEV)
    k = 313
    sel = torch.arange(k, dtype=torch.int32, device=DEV).expand(2, Hkv, k).contiguous()
    count = torch.tensor([[313] * 2, [5] * 2], dtype=torch.int32, device=DEV)
    cache = QuantisedCache(records=rec.to(DEV).view(pool, -1), top_k=k, **geometry(Hkv * G, Hkv, D, S, torch.float32, pool, table, lens))
    dense = [x.clone() for x in cache.paged_decode(q)]
    listed = cache.paged_decode(q, sel, count)
    for x, y in zip(dense, listed):
        assert (x - y).abs().max() <= 1e-5 * x.abs().max()


@pytest.mark.parametrize("batch,context,S", [(4, 60_001, 16), (40, 9_000, 32), (2, 130_000, 8)])
def test_large_pools_of_records(gpu_lib, batch, context, S):
    """Pools beyond what the caches hold, cut rows, ragged lengths; a few rows against 64 bits."""
    Hkv, G, D = 8, 4, 128
    lens = [context - (context * 3 // 4 * b // batch) - b for b in range(batch)]
    lens[1] = 17
    say(f"large pool {batch} x {context}, S={S}")
    g = torch.Generator().manual_seed(batch)
    table, pool = tables(lens, S, g)
    dg = torch.Generator(device=DEV).manual_seed(batch)
    rec = random_records(pool, Hkv, S, D, dg, DEV)
    q = torch.randn((batch, Hkv * G, D), generator=g).bfloat16()
    cache = QuantisedCache(records=rec.view(pool, -1), max_seq_len=context, **geometry(Hkv * G, Hkv, D, S, torch.bfloat16, pool, table, lens))
    cache.paged_decode(q.to(DEV))
    torch.cuda.synchronize()
    check_decode(cache, rec, q, table, lens, Hkv, S, D, rows=[(0, 0), (1, 3), (batch - 1, 7)])


def test_records_beyond_four_gigabytes(gpu_lib):
    """Offsets that pass 32 bits: the pages of a sequence at the end of a pool of 5 GB, written, attended to and read back."""
    Hkv, G, D, S, lens = 8, 4, 128, 16, [100]
    pool = 5_000_000_000 // (Hkv * R.tile_bytes(S, D))
    g = torch.Generator().manual_seed(9)
    table = torch.tensor([[pool - 1, 0, pool - 7, pool - 2, 5, pool - 3, pool - 4]], dtype=torch.int32)
    stage = torch.arange(7, dtype=torch.int32).view(1, 7)
    k, v = (torch.randn((7, Hkv, S, D), generator=g).bfloat16() for _ in range(2))
    cache = QuantisedCache(**geometry(Hkv * G, Hkv, D, S, torch.bfloat16, pool, table, lens))
    cache.quantise_pages(k.to(DEV), v.to(DEV), stage.to(DEV))
    q = torch.randn((1, Hkv * G, D), generator=g).bfloat16()
    cache.paged_decode(q.to(DEV))
    torch.cuda.synchronize()
    rec = R.tiles_of(k.flatten(0, 1), v.flatten(0, 1)).view(7, Hkv, -1)
    check_decode(cache, rec, q, stage, lens, Hkv, S, D)
    ko, vo = torch.zeros_like(k, device=DEV), torch.zeros_like(v, device=DEV)
    cache.restore_pages(ko, vo, stage.to(DEV))
    mine = (torch.arange(7 * S) < 100).view(7, 1, S, 1)
    assert torch.equal(ko.cpu().double(), R.values(*R.encode(k)) * mine) and torch.equal(vo.cpu().double(), R.values(*R.encode(v)) * mine)


# ------------------------------------------------------------------ page accounts

def paged(lens, H, Hkv, D, S, dtype, seed, spare_tokens=0):
    wl = W.build("accounts", seed, dtype=dtype, B=len(lens), H=H, Hkv=Hkv, D=D, S=S, seq_lens=[max(n, 1) for n in lens], top_k=4, key_mode="shift",
                 plant_mode="one_percent", permute=True, spare_tokens=spare_tokens)
    wl.seq_lens = torch.tensor(lens, dtype=torch.int32)
    return wl


def check_weighted(wl, sess, before, after, decay, scale=None, rows=None):
    out, lse, got = sess.out_dense.cpu().double(), sess.lse_dense.cpu().double(), after.cpu().double()
    S, D, G = wl.S, wl.D, wl.G
    k_cache, v_cache, table, lens = wl.k_cache.cpu(), wl.v_cache.cpu(), wl.page_table.cpu(), wl.seq_lens.tolist()
    for b, h in rows or itertools.product(range(wl.B), range(wl.Hkv)):
        n = lens[b]
        P = -(-n // S)
        ids = table[b, :P].long()
        k, v = (x[ids, h].reshape(-1, D)[:n] for x in (k_cache, v_cache))
        a = R.Attended(wl.q[b, h * G:(h + 1) * G].cpu(), k, v, 1 / math.sqrt(D) if scale is None else scale)
        tol = a.out_tolerance(wl.dtype, 2.0 ** -23)
        assert (out[b, h * G:(h + 1) * G] - a.out).abs().le(tol).all(), (b, h)
        want_lse = lse[b, h * G:(h + 1) * G]
        assert (want_lse == a.lse).logical_or((want_lse - a.lse).abs() <= a.slack + 2.0 ** -22 * a.lse.abs()).all(), (b, h)
        share = torch.zeros((G, P * S), dtype=torch.float64)
        share[:, :n] = a.p
        share = share.view(G, P, S).sum(-1)
        old = 0 if before is None else decay * before[b, h, :P].cpu().double()
        want = old + share.sum(0)
        # the share through its logarithm: two roundings of a number of the size of the logits more
        tol = ((a.slack + 2.0 ** -22 * (4 + a.lse.abs() + a.lse.abs().max()))[:, None] * share).sum(0) + 2.0 ** -22 * want.abs() + 1e-37
        assert (got[b, h, :P] - want).abs().le(tol).all(), (b, h, ((got[b, h, :P] - want).abs() / tol).max())
        if n:
            assert abs(float(share.sum()) - G) < 1e-9


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("G,D,S", [(1, 128, 16), (2, 64, 8), (4, 128, 8), (8, 128, 32), (8, 64, 16), (4, 64, 32), (8, 128, 16)])
def test_weighted_decode(gpu_lib, dtype, G, D, S):
    Hkv, lens = 4, [0, 1, S, 7 * S + 2, 260 * S - 3, 40 * S + 1]
    say(f"weighted decode {dtype} G={G} D={D} S={S}")
    wl = paged(lens, Hkv * G, Hkv, D, S, dtype, 40 + G).to(DEV)
    sess = DecodeSession(wl, track_weights=True)
    w0 = torch.rand((wl.B, Hkv, wl.max_pages), device=DEV)
    w1 = torch.full_like(w0, -5.0)
    sess.weighted_paged_decode(decay=0.75, weights_in=w0, weights_out=w1)
    torch.cuda.synchronize()
    check_weighted(wl, sess, w0, w1, 0.75)
    pages = (wl.seq_lens.cpu() + S - 1) // S
    for b in range(wl.B):
        assert (w1[b, :, int(pages[b]):] == -5.0).all()
    w2 = w0.clone()
    sess.weighted_paged_decode(decay=0.75, weights_in=w2, weights_out=w2)                      # in place: the same bits
    for b in range(wl.B):
        assert torch.equal(w2[b, :, :int(pages[b])], w1[b, :, :int(pages[b])])
    w3 = torch.full_like(w0, float("nan"))
    sess.weighted_paged_decode(decay=0.3, weights_in=None, weights_out=w3, sm_scale=0.2)       # from nothing
    torch.cuda.synchronize()
    check_weighted(wl, sess, None, w3, 0.0, scale=0.2)
    assert torch.isnan(w3[0]).all()


def test_weighted_decode_of_large_batches(gpu_lib):
    """Ragged batches beyond the caches' size, a row with one chunk, 300 rows; a table entry outside the pool weighs nothing."""
    for lens, Hkv in (([60_001, 2_000, 31, 45_000], 8), ([700 + 13 * b for b in range(40)], 8)):
        say(f"weighted decode of {len(lens)} x {max(lens)}")
        wl = paged(lens, Hkv * 4, Hkv, 128, 16, torch.bfloat16, 55).to(DEV)
        sess = DecodeSession(wl, track_weights=True)
        sess.weighted_paged_decode()
        torch.cuda.synchronize()
        rows = [(0, 0), (1, 5), (len(lens) - 1, 7)]
        check_weighted(wl, sess, None, sess.page_weights, 1.0, rows=rows)
        dense = DecodeSession(wl)
        dense.dense_paged_decode()
        assert (dense.out_dense.float() - sess.out_dense.float()).abs().max() <= 2.0 ** -7 * dense.out_dense.abs().max()
    wl.page_table[0, 3] = -1
    sess.weighted_paged_decode(weights_in=None, weights_out=sess.page_weights)
    torch.cuda.synchronize()
    assert (sess.page_weights[0, :, 3] == 0).all() and abs(float(sess.page_weights[0].sum()) - 32) < 1e-3


# ------------------------------------------------------------------ eviction

def check_evict(acc, table, lens, weights, S, policy, table_out, lens_out, weights_out):
    want = R.evict(table, lens, weights, S, *policy)
    for b, (keep, freed, n) in enumerate(want):
        P = -(-int(lens[b]) // S)
        assert int(lens_out[b]) == n and int(acc.freed_count[b]) == len(freed), b
        assert acc.freed_pages[b].tolist() == freed + [-1] * (acc.freed_pages.shape[1] - len(freed)), b
        assert table_out[b, :P].tolist() == table[b, keep].tolist() + [-1] * (P - len(keep)), b
        got, ref = weights_out[b, :, :P], torch.zeros((weights.shape[1], P))
        ref[:, :len(keep)] = weights[b][:, keep]
        assert torch.equal(got.nan_to_num(-9.0), ref.nan_to_num(-9.0)), b


@pytest.mark.parametrize("S,Hkv,budget,sinks,recent", [(16, 8, 20, 1, 4), (8, 1, 1, 0, 1), (32, 2, 64, 60, 4), (16, 32, 7, 0, 7), (8, 4, 300, 2, 1)])
def test_evict(gpu_lib, S, Hkv, budget, sinks, recent):
    """Lengths around the budget and far above it, ties, NaN; in place and into other arrays."""
    say(f"evict S={S} Hkv={Hkv} budget={budget}")
    g = torch.Generator().manual_seed(budget)
    lens = [0, 1, budget * S, budget * S + 1, (budget + 1) * S, (budget + 3) * S - 1, 5 * budget * S + 3, 1500 * S - 5]
    table, pool = tables(lens, S, g, extra_cols=3)
    weights = torch.rand((len(lens), Hkv, table.shape[1]), generator=g)
    weights[6] = (weights[6] * 3).round()          # ties
    weights[7, :, 40:60] = float("nan")
    weights[7, :, 700:] = 0.0
    weights[5] *= 1e-42                             # denormal accounts
    geo = geometry(Hkv * 2, Hkv, 64, S, torch.bfloat16, pool, table, lens)
    acc = PageAccounts(budget_pages=budget, sink_pages=sinks, recent_pages=recent, weights=weights.to(DEV), **geo)
    t_out, l_out, w_out = torch.full_like(geo["page_table"], 77), torch.full_like(geo["seq_lens"], 77), torch.full_like(acc.weights, 77.0)
    acc.evict_pages(weights_out=w_out, page_table_out=t_out, seq_lens_out=l_out)
    torch.cuda.synchronize()
    args = table, torch.tensor(lens), weights, S, (budget, sinks, recent)
    check_evict(acc, *args, t_out.cpu(), l_out.cpu(), w_out.cpu())
    for b, n in enumerate(lens):
        P = -(-n // S)
        assert (t_out[b, P:] == 77).all() and (w_out[b, :, P:] == 77).all()
    assert torch.equal(geo["page_table"].cpu(), table) and torch.equal(acc.weights.cpu().nan_to_num(-1), weights.nan_to_num(-1))
    acc.freed_pages.fill_(5)
    acc.evict_pages()
    torch.cuda.synchronize()
    check_evict(acc, *args, geo["page_table"].cpu(), geo["seq_lens"].cpu(), acc.weights.cpu())


@pytest.mark.parametrize("pages,budget", [(5000, 4096), (20_000, 900), (40_000, 39_000), (70_000, 100)])
def test_evict_from_long_sequences(gpu_lib, pages, budget):
    say(f"evict {pages} -> {budget}")
    S, Hkv = 16, 4
    g = torch.Generator().manual_seed(pages)
    lens = [pages * S - 3, pages * 5 * S // 7]
    table, pool = tables(lens, S, g)
    weights = torch.rand((2, Hkv, table.shape[1]), generator=g) ** 8
    geo = geometry(Hkv, Hkv, 64, S, torch.bfloat16, pool, table, lens)
    acc = PageAccounts(budget_pages=budget, sink_pages=4, recent_pages=16, weights=weights.to(DEV), **geo)
    acc.evict_pages()
    torch.cuda.synchronize()
    check_evict(acc, table, torch.tensor(lens), weights, S, (budget, 4, 16), geo["page_table"].cpu(), geo["seq_lens"].cpu(), acc.weights.cpu())


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("captured", [False, True])
def test_a_decode_loop_that_quantises_and_evicts(gpu_lib, captured):
    """What a server does per token: append, statistics and records of the new token, sparse attention over the selected records, dense attention that keeps
    accounts, eviction down to a budget. Eager, or from one HIP graph replayed for every token; every step's results are checked."""
    H, Hkv, D, S, budget = 16, 4, 128, 16, 12
    lens = [9 * S + 13, 200, 12 * S - 1]
    wl = paged(lens, H, Hkv, D, S, torch.bfloat16, 77, spare_tokens=8 * S)
    wl.k_cache, wl.v_cache = wl.k_cache.nan_to_num(0.0), wl.v_cache.nan_to_num(0.0)
    wl = wl.to(DEV)
    sess = DecodeSession(wl, track_weights=True, top_k=4)
    cache = QuantisedCache(q_heads=H, kv_heads=Hkv, head_dim=D, page_size=S, dtype=wl.dtype, num_pages=wl.num_phys_pages, page_table=wl.page_table,
                           seq_lens=wl.seq_lens, max_seq_len=wl.max_pages * S, top_k=4)
    acc = PageAccounts(budget_pages=budget, sink_pages=1, recent_pages=2, q_heads=H, kv_heads=Hkv, head_dim=D, page_size=S, dtype=wl.dtype,
                       num_pages=wl.num_phys_pages, page_table=wl.page_table, seq_lens=wl.seq_lens, max_seq_len=wl.max_pages * S, weights=sess.page_weights)
    sess.update_page_stats()
    cache.quantise_pages(wl.k_cache, wl.v_cache)
    begin, end = torch.zeros_like(wl.seq_lens), torch.zeros_like(wl.seq_lens)
    new = torch.zeros((2, wl.B, Hkv, D), dtype=wl.dtype, device=DEV)
    rows = torch.arange(wl.B, device=DEV)

    def append():  # the engine's part
        n = wl.seq_lens.long()
        page = wl.page_table[rows, n // S].long()
        wl.k_cache[page, :, n % S] = new[0]
        wl.v_cache[page, :, n % S] = new[1]
        begin.copy_(wl.seq_lens)
        wl.seq_lens.add_(1)
        end.copy_(wl.seq_lens)

    def step():
        append()
        sess.update_page_stats(begin, end, 1)
        cache.quantise_pages(wl.k_cache, wl.v_cache, None, begin, end, 1)
        sess.score_select_topk()
        cache.paged_decode(wl.q, sess.sel_pages, sess.sel_count)
        sess.weighted_paged_decode(decay=0.9, weights_in=sess.page_weights, weights_out=sess.page_weights)

    spare = {b: wl.page_table[b, -(-lens[b] // S):].tolist() for b in range(wl.B)}
    wl.page_table[:] = torch.where(torch.arange(wl.max_pages, device=DEV) < ((wl.seq_lens + S - 1) // S)[:, None], wl.page_table, -1)
    graph = None
    for i in range(70):
        for b in range(wl.B):  # a free page where the next token begins one
            n = int(wl.seq_lens[b])
            if n % S == 0:
                wl.page_table[b, n // S] = spare[b].pop()
        torch.manual_seed(i)
        new.copy_(torch.randn(new.shape))
        wl.q.copy_(torch.randn(wl.q.shape))
        before_w, before_t, before_n = sess.page_weights.clone(), wl.page_table.cpu(), (wl.seq_lens + 1).cpu()
        if captured and graph is None and i == 1:
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            keep = [x.clone() for x in (wl.seq_lens, sess.page_weights, wl.page_table)]
            with torch.cuda.stream(s):
                step(), acc.evict_pages()
            torch.cuda.current_stream().wait_stream(s)
            for x, y in zip((wl.seq_lens, sess.page_weights, wl.page_table), keep):
                x.copy_(y)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is not None:
            graph.replay()
        else:
            step()
        torch.cuda.synchronize()
        mid = sess.page_weights.clone()
        check_weighted(wl, sess, before_w, mid, 0.9, rows=[(i % 3, i % 4)])
        rec = R.tiles_of(wl.k_cache.cpu().flatten(0, 1), wl.v_cache.cpu().flatten(0, 1)).view(wl.num_phys_pages, Hkv, -1) if i % 10 == 9 else None
        if rec is not None:
            sel, cnt = sess.sel_pages.cpu(), sess.sel_count.cpu()
            lists = [[sel[b, h, :cnt[b, h]].tolist() for h in range(Hkv)] for b in range(wl.B)]
            check_decode(cache, rec, wl.q.cpu(), wl.page_table.cpu(), wl.seq_lens.tolist(), Hkv, S, D, lists=lists)
        acc.evict_pages()
        torch.cuda.synchronize()
        check_evict(acc, before_t, before_n, mid.cpu(), S, acc.policy, wl.page_table.cpu(), wl.seq_lens.cpu(), sess.page_weights.cpu())
        for b in range(wl.B):
            spare[b] += acc.freed_pages[b, :int(acc.freed_count[b])].tolist()
    assert max(wl.seq_lens.tolist()) <= budget * S and int(wl.page_table.max()) < wl.num_phys_pages


def test_calls_run_on_the_current_stream(gpu_lib):
    """Two streams with workspaces of their own, each behind a long kernel of its stream."""
    H, Hkv, D, S, lens = 8, 2, 64, 8, [900, 333]
    g = torch.Generator().manual_seed(2)
    table, pool = tables(lens, S, g)
    q = torch.randn((2, H, D), generator=g).to(DEV)
    k, v = (torch.randn((pool, Hkv, S, D), generator=g).to(DEV) for _ in range(2))
    caches = [QuantisedCache(**geometry(H, Hkv, D, S, torch.float32, pool, table, lens)) for _ in range(3)]
    caches[2].quantise_pages(k, v)
    want = [x.clone() for x in caches[2].paged_decode(q)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    big = torch.randn((4096, 4096), device=DEV)
    late = [torch.zeros_like(k) for _ in range(2)]
    torch.cuda.synchronize()
    for s, c, x in zip(streams, caches, late):
        with torch.cuda.stream(s):
            for _ in range(4):
                big @ big
            x.copy_(k)
            c.quantise_pages(x, v)
            c.paged_decode(q)
    torch.cuda.synchronize()
    for c in caches[:2]:
        assert torch.equal(c.out, want[0]) and torch.equal(c.lse, want[1])


def test_all_calls_in_one_graph_replayed(gpu_lib):
    """Quantise, restore, both forms of attention over records, weighted attention and an eviction in place in one HIP graph; every replay, on other
    inputs and with eager work between, equals the eager calls bit for bit."""
    H, Hkv, D, S, lens, budget = 16, 4, 128, 16, [1000, 37, 700], 40
    wl = paged(lens, H, Hkv, D, S, torch.bfloat16, 12).to(DEV)
    wl.k_cache.nan_to_num_(0.0), wl.v_cache.nan_to_num_(0.0)
    geo = dict(q_heads=H, kv_heads=Hkv, head_dim=D, page_size=S, dtype=wl.dtype, num_pages=wl.num_phys_pages, page_table=wl.page_table, seq_lens=wl.seq_lens)
    sess, cache = DecodeSession(wl, track_weights=True), QuantisedCache(top_k=8, **geo)
    acc = PageAccounts(budget_pages=budget, sink_pages=1, recent_pages=2, weights=sess.page_weights, **geo)
    k_out, v_out = torch.zeros_like(wl.k_cache), torch.zeros_like(wl.v_cache)
    listed = torch.zeros_like(cache.out)
    sel = torch.arange(8, dtype=torch.int32, device=DEV).expand(3, Hkv, 8).contiguous()
    count = torch.full((3, Hkv), 8, dtype=torch.int32, device=DEV)
    start = [wl.page_table.clone(), wl.seq_lens.clone()]

    def calls():
        cache.quantise_pages(wl.k_cache, wl.v_cache)
        cache.restore_pages(k_out, v_out)
        listed.copy_(cache.paged_decode(wl.q, sel, count)[0])
        cache.paged_decode(wl.q)
        sess.weighted_paged_decode(decay=0.5, weights_in=sess.page_weights, weights_out=sess.page_weights)
        acc.evict_pages()

    def begin(seed):
        torch.manual_seed(seed)
        wl.page_table.copy_(start[0]), wl.seq_lens.copy_(start[1])
        wl.q.copy_(torch.randn(wl.q.shape))
        wl.k_cache.copy_(torch.randn(wl.k_cache.shape))
        wl.v_cache.copy_(torch.randn(wl.v_cache.shape))
        sess.page_weights.copy_(torch.rand(sess.page_weights.shape))
        for x in (cache.records, k_out, v_out, listed, cache.out, sess.out_dense, acc.freed_pages):
            x.zero_()

    def results():
        torch.cuda.synchronize()
        return [x.clone() for x in (cache.records, k_out, v_out, listed, cache.out, cache.lse, sess.out_dense, sess.lse_dense, sess.page_weights, wl.page_table,
                                    wl.seq_lens, acc.freed_pages, acc.freed_count)]

    begin(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        calls()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in range(1, 5):
        begin(seed)
        calls()
        want = results()
        assert int(acc.freed_count.max()) > 0
        begin(seed)
        graph.replay()
        for x, y in zip(results(), want):
            assert torch.equal(x, y), seed


def test_bounds_below_the_table(gpu_lib):
    """A length bound far below the table's width, and accounts wider than the bound: the calls read and write the sequences' part only."""
    H, Hkv, D, S, lens, budget = 8, 2, 64, 8, [100, 61], 6
    wl = paged(lens, H, Hkv, D, S, torch.float32, 31, spare_tokens=400)
    wl = wl.to(DEV)
    geo = dict(q_heads=H, kv_heads=Hkv, head_dim=D, page_size=S, dtype=wl.dtype, num_pages=wl.num_phys_pages, page_table=wl.page_table, seq_lens=wl.seq_lens,
               max_seq_len=104)
    sess = DecodeSession(wl, track_weights=True, max_seq_len_hint=104)
    sess.page_weights.fill_(3.0)
    sess.weighted_paged_decode(decay=0.0)
    torch.cuda.synchronize()
    check_weighted(wl, sess, None, sess.page_weights, 0.0)
    assert (sess.page_weights[0, :, 13:] == 3).all() and (sess.page_weights[1, :, 8:] == 3).all()
    cache = QuantisedCache(**geo)
    cache.quantise_pages(wl.k_cache, wl.v_cache)
    q = wl.q.cpu()
    cache.paged_decode(wl.q)
    torch.cuda.synchronize()
    rec = R.tiles_of(wl.k_cache.cpu().nan_to_num(0.0).flatten(0, 1), wl.v_cache.cpu().nan_to_num(0.0).flatten(0, 1)).view(wl.num_phys_pages, Hkv, -1)
    check_decode(cache, rec, q, wl.page_table.cpu(), lens, Hkv, S, D)
    before = wl.page_table.cpu().clone(), wl.seq_lens.cpu().clone(), sess.page_weights.cpu().clone()
    acc = PageAccounts(budget_pages=budget, sink_pages=0, recent_pages=1, weights=sess.page_weights, **geo)
    acc.evict_pages()
    torch.cuda.synchronize()
    check_evict(acc, *before, S, (budget, 0, 1), wl.page_table.cpu(), wl.seq_lens.cpu(), sess.page_weights.cpu())
    assert torch.equal(wl.page_table.cpu()[:, 13:], before[0][:, 13:]) and (sess.page_weights[0, :, 13:] == 3).all()


@pytest.mark.parametrize("batch,tokens", [(300, 90), (33, 700)])
def test_many_sequences(gpu_lib, batch, tokens):
    """More rows than compute units, short sequences among them, fp32 records with eight heads; every row of some sequences."""
    Hkv, G, D, S = 8, 8, 128, 16
    lens = [(tokens * (b % 7 + 1)) // 7 for b in range(batch)]
    g = torch.Generator().manual_seed(batch)
    table, pool = tables(lens, S, g)
    rec = random_records(pool, Hkv, S, D, g)
    q = torch.randn((batch, Hkv * G, D), generator=g)
    cache = QuantisedCache(records=rec.to(DEV).view(pool, -1), **geometry(Hkv * G, Hkv, D, S, torch.float32, pool, table, lens))
    cache.paged_decode(q.to(DEV))
    torch.cuda.synchronize()
    check_decode(cache, rec, q, table, lens, Hkv, S, D, rows=[(b, h) for b in (0, 6, batch - 1) for h in range(Hkv)])


@pytest.mark.parametrize("pages", [600, 3000, 7000, 12_000])
@pytest.mark.parametrize("kind", ["equal", "zero", "two values", "wide", "infinite", "nan", "signs", "rising"])
def test_evict_whatever_the_accounts(gpu_lib, kind, pages):
    """Accounts that a search for the separating one could stumble over; budgets that only the pages kept in any case fill, and ones page more or less."""
    S, Hkv = 8, 2
    g = torch.Generator().manual_seed(pages)
    lens = [pages * S - 1] * 2
    table, pool = tables(lens, S, g)
    w = torch.rand((2, Hkv, pages), generator=g)
    if kind == "equal":
        w[:] = 0.125
    elif kind == "zero":
        w[:] = 0.0
    elif kind == "two values":
        w = (w > 0.5).float()
    elif kind == "wide":
        w = torch.pow(2.0, 250 * w - 125)
    elif kind == "infinite":
        w[:, :, ::3] = float("inf")
    elif kind == "nan":
        w[:, 0, 1::2] = float("nan")
    elif kind == "signs":
        w -= 0.5
    else:
        w[:] = torch.arange(pages) / 7.0
    for budget, sinks, recent in ((pages // 3, 2, 5), (40, 30, 10), (pages - 1, 0, 1), (pages - 5, 1, 1), (1, 0, 1)):
        geo = geometry(Hkv, Hkv, 64, S, torch.bfloat16, pool, table, lens)
        acc = PageAccounts(budget_pages=budget, sink_pages=sinks, recent_pages=recent, weights=w.to(DEV), **geo)
        acc.evict_pages()
        torch.cuda.synchronize()
        check_evict(acc, table, torch.tensor(lens), w, S, (budget, sinks, recent), geo["page_table"].cpu(), geo["seq_lens"].cpu(), acc.weights.cpu())


def test_the_python_layer_refuses(gpu_lib):
    """Host tensors, other types, shapes and layouts: refused before the library is called."""
    D, S, Hkv, H, lens = 64, 8, 2, 8, [20, 9]
    g = torch.Generator().manual_seed(0)
    table, pool = tables(lens, S, g)
    geo = geometry(H, Hkv, D, S, torch.float32, pool, table, lens)
    cache, acc = QuantisedCache(top_k=4, **geo), PageAccounts(budget_pages=2, **geo)
    k = torch.zeros((pool, Hkv, S, D), device=DEV)
    q = torch.zeros((2, H, D), device=DEV)
    ints = torch.zeros(2, dtype=torch.int32, device=DEV)
    sel = torch.zeros((2, Hkv, 4), dtype=torch.int32, device=DEV)
    count = torch.zeros((2, Hkv), dtype=torch.int32, device=DEV)
    w = torch.zeros_like(acc.weights)
    bad = [lambda: cache.quantise_pages(k.cpu(), k), lambda: cache.quantise_pages(k, k.bfloat16()), lambda: cache.quantise_pages(k[:, :1], k[:, :1]),
           lambda: cache.quantise_pages(k, k[:-1]), lambda: cache.quantise_pages(k.transpose(2, 3).contiguous().transpose(2, 3), k),
           lambda: cache.quantise_pages(k, k, geo["page_table"][:, :1].contiguous()), lambda: cache.quantise_pages(k, k, None, ints.long(), ints, 1),
           lambda: cache.quantise_pages(k, k, None, ints.cpu(), ints, 1), lambda: cache.quantise_pages(k, k, None, ints[:1], ints, 1),
           lambda: cache.restore_pages(k, k.cpu()), lambda: cache.restore_pages(k, k, geo["page_table"].cpu()),
           lambda: cache.paged_decode(q.cpu()), lambda: cache.paged_decode(q.bfloat16()), lambda: cache.paged_decode(q[:1]),
           lambda: cache.paged_decode(q, sel.long(), count), lambda: cache.paged_decode(q, sel, count[:1]), lambda: cache.paged_decode(q, sel.cpu(), count),
           lambda: acc.evict_pages(weights_in=w.cpu()), lambda: acc.evict_pages(weights_in=w.double()), lambda: acc.evict_pages(weights_out=w[:, :1]),
           lambda: acc.evict_pages(page_table_out=geo["page_table"].long()), lambda: acc.evict_pages(seq_lens_out=ints.cpu()),
           lambda: QuantisedCache(records=torch.zeros((pool, 7), dtype=torch.uint8, device=DEV), **geo),
           lambda: PageAccounts(budget_pages=2, weights=w[:, :, 1:], **geo)]
    for i, call in enumerate(bad):
        with pytest.raises(AssertionError):
            call()
            raise RuntimeError(f"call {i} was taken")
    longer = torch.zeros((2, Hkv, 4000), dtype=torch.int32, device=DEV)  # a list that the workspace was not made for
    with pytest.raises(binding.UniqueError) as e:
        cache.paged_decode(q, longer, count)
    assert e.value.code == binding.ERR_WORKSPACE
    with pytest.raises(binding.UniqueError):
        PageAccounts(budget_pages=2, sink_pages=2, recent_pages=1, **geo).evict_pages()


def test_a_step_after_an_eviction_far_below_the_session_s_lower_bound(gpu_lib):
    """The session's bounds on the lengths are those of its start; sequences that eviction has made much shorter are selected and attended to as in a new session."""
    H, Hkv, D, S, lens, budget = 16, 4, 128, 16, [9000, 6400, 8011], 24
    wl = paged(lens, H, Hkv, D, S, torch.bfloat16, 99).to(DEV)
    sess = DecodeSession(wl, track_weights=True, top_k=8)
    sess.update_page_stats()
    sess.weighted_paged_decode()
    acc = PageAccounts(budget_pages=budget, sink_pages=1, recent_pages=3, q_heads=H, kv_heads=Hkv, head_dim=D, page_size=S, dtype=wl.dtype,
                       num_pages=wl.num_phys_pages, page_table=wl.page_table, seq_lens=wl.seq_lens, weights=sess.page_weights)
    acc.evict_pages()
    assert int(wl.seq_lens.max()) <= budget * S
    sess.decode_step(refresh_tail=True)
    sess.dense_paged_decode()
    fresh = DecodeSession(wl, top_k=8)
    fresh.update_page_stats()
    fresh.decode_step(refresh_tail=True)
    fresh.dense_paged_decode()
    torch.cuda.synchronize()
    assert torch.equal(sess.sel_pages, fresh.sel_pages) and torch.equal(sess.sel_count, fresh.sel_count)
    for x, y in ((sess.out, fresh.out), (sess.out_dense, fresh.out_dense)):
        assert (x.float() - y.float()).abs().max() <= 2.0 ** -7 * y.float().abs().max()
    sess.weighted_paged_decode(weights_in=None, weights_out=sess.page_weights)
    torch.cuda.synchronize()
    check_weighted(wl, sess, None, sess.page_weights, 0.0)


@pytest.mark.parametrize("dtype,D,S,Hkv,batch,tokens", [(torch.bfloat16, 128, 16, 8, 40, 4000), (torch.float32, 128, 16, 8, 33, 5000), (torch.bfloat16, 64, 32, 16, 50, 7000)])
def test_batches_of_many_rows_cut_by_their_lengths(gpu_lib, dtype, D, S, Hkv, batch, tokens):
    """With the workspace that is asked for, and with the smaller one of unique_workspace_bytes, which is cut otherwise: the same within rounding, and what a cut
    writes stays in the workspace."""
    G = 2
    lens = [max(0, tokens - 97 * b) for b in range(batch)]
    g = torch.Generator().manual_seed(batch)
    table, pool = tables(lens, S, g)
    rec = random_records(pool, Hkv, S, D, g)
    q = torch.randn((batch, Hkv * G, D), generator=g).to(dtype)
    cache = QuantisedCache(records=rec.to(DEV).view(pool, -1), **geometry(Hkv * G, Hkv, D, S, dtype, pool, table, lens))
    small = gpu_lib.workspace_bytes(cache.desc, 1)
    assert small < cache.workspace.numel()
    guard = torch.full((cache.workspace.numel() + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    for size in (cache.workspace.numel(), small):
        guard.fill_(0xA5)
        cache.workspace = guard[:size]
        cache.paged_decode(q.to(DEV))
        torch.cuda.synchronize()
        assert (guard[size:] == 0xA5).all()
        check_decode(cache, rec, q, table, lens, Hkv, S, D, rows=[(0, 0), (1, Hkv - 1), (batch // 2, 3), (batch - 1, 1)])


@pytest.mark.parametrize("dtype,G,D,batch,tokens", [(torch.bfloat16, 4, 128, 40, 2500), (torch.float32, 2, 64, 50, 4200)])
def test_weighted_batches_of_many_rows(gpu_lib, dtype, G, D, batch, tokens):
    """More rows than compute units, long ones among them: cut by their lengths into a workspace that a guard follows."""
    Hkv = 8
    lens = [max(0, tokens - (tokens // batch + 1) * b) for b in range(batch)]
    wl = paged(lens, Hkv * G, Hkv, D, 16, dtype, 70).to(DEV)
    sess = DecodeSession(wl, track_weights=True, max_seq_len_hint=tokens)
    need = gpu_lib.account_workspace_bytes(sess.desc)
    guard = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    sess.workspace = guard[:need]
    w = torch.rand_like(sess.page_weights)
    before = w.clone()
    sess.weighted_paged_decode(decay=0.5, weights_in=w, weights_out=w)
    torch.cuda.synchronize()
    assert (guard[need:] == 0xA5).all()
    check_weighted(wl, sess, before, w, 0.5, rows=[(0, 0), (1, 7), (batch // 2, 3), (batch - 1, 1)])
    pages = (wl.seq_lens + 15) // 16
    for b in (1, batch - 1):
        assert torch.equal(w[b, :, int(pages[b]):], before[b, :, int(pages[b]):])
    sess.workspace = guard[:need - 256]
    with pytest.raises(binding.UniqueError) as e:
        sess.weighted_paged_decode(decay=0.5, weights_in=w, weights_out=w)
    assert e.value.code == binding.ERR_WORKSPACE


def test_the_python_layer_refuses_repeated_pages_and_flat_lists(gpu_lib):
    """A stride of 0 is the descriptor's word for the default, and a list of pages has a row per KV head: both would have the kernels read elsewhere."""
    D, S, Hkv, H, lens = 64, 8, 2, 8, [20, 9]
    table, pool = tables(lens, S, torch.Generator().manual_seed(0))
    cache = QuantisedCache(top_k=4, **geometry(H, Hkv, D, S, torch.float32, pool, table, lens))
    page = torch.zeros((1, Hkv, S, D), device=DEV).expand(pool, Hkv, S, D)
    head = torch.zeros((pool, 1, S, D), device=DEV).expand(pool, Hkv, S, D)
    q, count = torch.zeros((2, H, D), device=DEV), torch.zeros((2, Hkv), dtype=torch.int32, device=DEV)
    for call in (lambda: cache.quantise_pages(page, page), lambda: cache.quantise_pages(head, head), lambda: cache.restore_pages(page, page),
                 lambda: cache.paged_decode(q, count, count), lambda: cache.paged_decode(q, count.reshape(2, Hkv, 1, 1), count)):
        with pytest.raises(AssertionError):
            call()


def test_accounts_of_a_session_from_one_array_to_another(gpu_lib):
    """The account arrays of a session: its own, one given as the input alone, a pair, and an output alone; none without ``track_weights``."""
    wl = paged([70, 33], 16, 4, 64, 8, torch.bfloat16, 9).to(DEV)
    sess = DecodeSession(wl, top_k=2, track_weights=True)
    given, out = torch.rand_like(sess.page_weights), torch.zeros_like(sess.page_weights)
    sess.weighted_paged_decode()
    share = sess.page_weights.clone()
    sess.weighted_paged_decode(decay=0.5, weights_in=given)
    other = given.clone()
    sess.weighted_paged_decode(decay=0.5, weights_in=other, weights_out=other)
    sess.weighted_paged_decode(decay=0.5, weights_out=out)
    pages = [-(-n // 8) for n in (70, 33)]
    for b, n in enumerate(pages):
        assert torch.equal(sess.page_weights[b, :, :n], other[b, :, :n]) and torch.equal(out[b, :, :n], share[b, :, :n])
        # decay * in + share, rounded once, below 8 (G = 4 and a half)
        assert (other[b, :, :n].double() - given[b, :, :n].double() / 2 - share[b, :, :n].double()).abs().max() <= 8 * 2.0 ** -24
        assert torch.equal(other[b, :, n:], given[b, :, n:])
    with pytest.raises(AssertionError, match="track_weights"):
        DecodeSession(wl, top_k=2).weighted_paged_decode()
