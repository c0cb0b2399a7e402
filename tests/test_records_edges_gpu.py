"""Edges of the calls on 4-bit records, page accounts and eviction on the GPU against plain 64-bit counterparts (records_ref.py)."""
import math

import pytest
import torch

from paper_2605_27740_amd import binding
from paper_2605_27740_amd.session import DecodeSession, PageAccounts, QuantisedCache
from tests import records_ref as R
from tests.test_records_gpu import DEV, DTYPES, check_evict, geometry, paged, say, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("G,D,S", [(1, 128, 16), (2, 64, 8), (4, 128, 16), (4, 64, 32), (8, 128, 32), (8, 64, 8)])
def test_probabilities_of_records_are_32_bit_numbers(gpu_lib, dtype, G, D, S):
    """Two tokens with opposite values and nearly equal weights: what is left of the output is as small as 2^-10 of what it is the
    difference of, so that its own rounding does not hide a probability of few bits.

    Only channel 0 of a query is not zero, so a logit is one product, exact in 32 bits. Relative to the reference, which is 6 above the larger
    one, a logit lies in (-8, 0]: one rounding of 2^-22, ln 2 times that in the exponential, and 2^-23 for the exponential's last bit: 2^-21.7 of
    a probability. The reference is common to probabilities and normaliser; their sums add at most four roundings of the small difference. 2^-21
    of the sum of |p v| covers these; 16 bits of a probability would be off by up to 2^-16 of it."""
    say(f"two tokens {dtype} G={G} D={D} S={S}")
    B, Hkv = 16, 4
    lens = [2] * B
    g = torch.Generator().manual_seed(G + D + S)
    table, pool = tables(lens, S, g)
    code = torch.randint(1, 8, (pool, Hkv, D), generator=g)
    k = torch.zeros((pool, Hkv, S, D), dtype=torch.float64)
    v = torch.zeros_like(k)
    k[:, :, 0, 0], k[:, :, 1, 0] = 6.0, R.LEVELS[torch.randint(0, 7, (pool, Hkv), generator=g)]
    v[:, :, 0] = R.LEVELS[code]
    v[:, :, 0, ::32] = 6.0           # the largest of every block: all scales are 1
    v[:, :, 1] = -v[:, :, 0]
    rec = R.tiles_of(k.flatten(0, 1), v.flatten(0, 1)).view(pool, Hkv, -1)
    q = torch.zeros((B, Hkv * G, D))
    q[:, :, 0] = (1 + torch.rand((B, Hkv * G), generator=g)) * 2.0 ** -10
    q = q.to(dtype)
    cache = QuantisedCache(records=rec.to(DEV).view(pool, -1), **geometry(Hkv * G, Hkv, D, S, dtype, pool, table, lens))
    cache.paged_decode(q.to(DEV))
    torch.cuda.synchronize()
    out = cache.out.cpu().double().view(B, Hkv, G, D)
    page = table[:, 0].long()
    x = q.double().view(B, Hkv, G, D)[..., :1] * k[page][:, :, None, :2, 0] / math.sqrt(D)  # [B, Hkv, G, 2]
    p = torch.softmax(x, -1)
    want = (p[..., :1] - p[..., 1:]) * v[page][:, :, None, 0]
    mass = v[page][:, :, None, 0].abs().expand_as(want)
    tol = 1.01 * torch.finfo(dtype).eps / 2 * want.abs() + 2.0 ** -21 * mass
    worst = float(((out - want).abs() / tol).max())
    assert worst <= 1


def test_evict_in_place_from_many_long_sequences(gpu_lib):
    """More workgroups than the GPU holds at a time share the sequences, nine to the longest: the lengths that a call shortens in place are those
    that all of them work from. Twice, the second time with ids of the first in the list of freed pages."""
    S, Hkv, B, budget, policy = 8, 1, 70, 9000, (4, 16)
    say(f"evict {B} long sequences")
    g = torch.Generator().manual_seed(5)
    for longest in (33_500, 36_000):
        lens = [longest * S - 7 - 64 * b if b % 10 else budget * S - 8 * (b - 1) for b in range(B)]
        table, pool = tables(lens, S, g)
        weights = torch.rand((B, Hkv, table.shape[1]), generator=g)
        geo = geometry(Hkv, Hkv, 64, S, torch.bfloat16, pool, table, lens)
        acc = PageAccounts(budget_pages=budget, sink_pages=policy[0], recent_pages=policy[1], weights=weights.to(DEV), **geo)
        acc.freed_pages.copy_(torch.arange(acc.freed_pages.numel()).view(acc.freed_pages.shape))  # what an earlier call may have left
        acc.freed_count.fill_(-3)
        acc.evict_pages()
        torch.cuda.synchronize()
        acc.freed_pages, acc.freed_count = acc.freed_pages.cpu(), acc.freed_count.cpu()
        check_evict(acc, table, torch.tensor(lens), weights, S, (budget, *policy), geo["page_table"].cpu(), geo["seq_lens"].cpu(), acc.weights.cpu())


@pytest.mark.parametrize("kind", ["equal", "two values", "wide", "infinite", "nan", "signs"])
@pytest.mark.parametrize("pages,Hkv", [(1000, 32), (3900, 8), (8188, 8), (20_000, 2)])
def test_evict_whatever_the_accounts_and_the_heads(gpu_lib, kind, pages, Hkv):
    """Rows whose sums other workgroups have formed, and rows that no workgroup holds; in place and into other arrays."""
    S, B = 8, 2
    say(f"evict {pages} pages, {Hkv} heads, {kind}")
    g = torch.Generator().manual_seed(pages)
    lens = [pages * S - 1, (pages - 77) * S]
    table, pool = tables(lens, S, g)
    w = torch.rand((B, Hkv, pages), generator=g)
    if kind == "equal":
        w[:] = 0.125
    elif kind == "two values":
        w = (w > 0.5).float()
    elif kind == "wide":
        w = torch.pow(2.0, 250 * w - 125)
    elif kind == "infinite":
        w[:, :, 1::3] = float("inf")
    elif kind == "nan":
        w[:, 0, 1::2] = float("nan")
    else:
        w -= 0.5
    for budget, sinks, recent in ((pages // 3, 2, 5), (pages - 3, 1, 1), (pages - 100, 0, 40)):
        geo = geometry(Hkv, Hkv, 64, S, torch.bfloat16, pool, table, lens)
        acc = PageAccounts(budget_pages=budget, sink_pages=sinks, recent_pages=recent, weights=w.to(DEV), **geo)
        args = table, torch.tensor(lens), w, S, (budget, sinks, recent)
        t_out, l_out, w_out = torch.full_like(geo["page_table"], 77), torch.full_like(geo["seq_lens"], 77), torch.full_like(acc.weights, 77.0)
        acc.evict_pages(weights_out=w_out, page_table_out=t_out, seq_lens_out=l_out)
        torch.cuda.synchronize()
        check_evict(acc, *args, t_out.cpu(), l_out.cpu(), w_out.cpu())
        assert torch.equal(geo["page_table"].cpu(), table) and geo["seq_lens"].tolist() == lens
        acc.freed_pages.fill_(5)
        acc.evict_pages()
        torch.cuda.synchronize()
        check_evict(acc, *args, geo["page_table"].cpu(), geo["seq_lens"].cpu(), acc.weights.cpu())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
def test_records_of_values_that_are_denormal_in_the_cache(gpu_lib, dtype, D):
    """Multiples of 2^-130 on either side of the smallest level, 2^-127, whose restored value is a denormal of both types, and of its ties; bytes and values exactly."""
    S, Hkv = 8, 1
    step = torch.arange(S * D, dtype=torch.float64).view(1, Hkv, S, D) % 97
    k = step * 2.0 ** -130 * (1 - 2 * (torch.arange(D) % 2)) + 0.0
    v = (96 - step) * 2.0 ** -130
    v[..., -1, 32:] *= 2.0 ** 8  # blocks of an ordinary exponent beside them
    assert torch.equal(k.to(dtype).double(), k) and torch.equal(v.to(dtype).double(), v)
    want = [R.values(*R.encode(x)) for x in (k, v)]
    assert all((x.abs() == 2.0 ** -127).any() and (x == 0).any() for x in want)
    table = torch.zeros((1, 1), dtype=torch.int32)
    cache = QuantisedCache(**geometry(1, 1, D, S, dtype, 1, table, [S]))
    cache.quantise_pages(k.to(dtype).to(DEV), v.to(dtype).to(DEV))
    ko, vo = (torch.full((1, 1, S, D), -77.0, dtype=dtype, device=DEV) for _ in range(2))
    cache.restore_pages(ko, vo)
    torch.cuda.synchronize()
    for got, x in zip((ko, vo), want):
        wrong = got.cpu().double() != x
        assert not wrong.any(), (int(wrong.sum()), got.cpu().double()[wrong][:4].tolist(), x[wrong][:4].tolist())
    wrong = (cache.records.cpu().view(-1) != R.tiles_of(k.flatten(0, 1), v.flatten(0, 1)).view(-1)).nonzero().flatten().tolist()
    assert wrong == []


def test_evict_reads_given_accounts_and_writes_its_own(gpu_lib):
    """Accounts given as the input alone are read and stay as they are, as in ``DecodeSession.weighted_paged_decode``; given as the output alone they
    take what becomes of the own ones."""
    S, Hkv, budget, lens = 8, 2, 6, [77, 30, 160]
    g = torch.Generator().manual_seed(3)
    table, pool = tables(lens, S, g)
    own, given = (torch.rand((3, Hkv, table.shape[1]), generator=g) for _ in range(2))
    for which in ("in", "out", "both"):
        geo = geometry(Hkv, Hkv, 64, S, torch.bfloat16, pool, table, lens)
        acc = PageAccounts(budget_pages=budget, weights=own.to(DEV), **geo)
        w, other = given.to(DEV), torch.full_like(own, 9.0).to(DEV)
        if which == "in":
            acc.evict_pages(weights_in=w)
            source, result, untouched = given, acc.weights, (w, given)
        elif which == "out":
            acc.evict_pages(weights_out=w)
            source, result, untouched = own, w, (acc.weights, own)
        else:
            acc.evict_pages(weights_in=w, weights_out=other)
            source, result, untouched = given, other, (acc.weights, own)
        torch.cuda.synchronize()
        assert torch.equal(untouched[0].cpu(), untouched[1]), which
        check_evict(acc, table, torch.tensor(lens), source, S, (budget, 0, 1), geo["page_table"].cpu(), geo["seq_lens"].cpu(), result.cpu())


def test_counts_without_lists_are_refused(gpu_lib):
    """In the handle and in the binding; lists without counts, too."""
    D, S, Hkv, H, lens = 64, 8, 2, 8, [20, 9]
    table, pool = tables(lens, S, torch.Generator().manual_seed(0))
    cache = QuantisedCache(top_k=4, **geometry(H, Hkv, D, S, torch.float32, pool, table, lens))
    q, count = torch.zeros((2, H, D), device=DEV), torch.ones((2, Hkv), dtype=torch.int32, device=DEV)
    sel = torch.zeros((2, Hkv, 4), dtype=torch.int32, device=DEV)
    with pytest.raises(AssertionError, match="counts"):
        cache.paged_decode(q, None, count)
    for pages, n in ((None, count), (sel, None)):
        with pytest.raises(binding.UniqueError) as e:
            gpu_lib.quantised_paged_decode(cache.desc, cache.records, q, pages, n, 0.0, cache.out, cache.lse, cache.workspace)
        assert e.value.code == binding.ERR_INVALID_ARG


def test_ranges_without_a_bound_on_their_pages(gpu_lib):
    """All pages of a range are written and read back; with a bound, those that it covers."""
    D, S, Hkv, lens = 64, 8, 2, [100, 3, 61]
    g = torch.Generator().manual_seed(8)
    table, pool = tables(lens, S, g)
    k, v = (torch.randn((pool, Hkv, S, D), generator=g).to(DEV) for _ in range(2))
    begin, end = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([5, 0, 60], [99, 3, 61]))
    want = [R.values(*R.encode(x.cpu())) for x in (k, v)]
    for bound, pages in ((None, [13, 1, 8]), (2, [2, 1, 8]), (0, [0, 0, 0])):
        cache = QuantisedCache(**geometry(Hkv, Hkv, D, S, torch.float32, pool, table, lens))
        cache.quantise_pages(k, v, tok_begin=begin, tok_end=end, **({} if bound is None else dict(max_pages_touched_per_seq=bound)))
        got = [torch.full_like(k, -77.0) for _ in range(2)]
        cache.restore_pages(*got, tok_begin=begin, tok_end=end, **({} if bound is None else dict(max_pages_touched_per_seq=bound)))
        torch.cuda.synchronize()
        mine = torch.zeros((pool, 1, S, 1), dtype=torch.bool)
        for b in range(3):
            for t in range(int(begin[b]), int(end[b])):
                mine[int(table[b, t // S]), 0, t % S] = t // S < pages[b]
        for x, y in zip(got, want):
            assert torch.equal(x.cpu().double(), torch.where(mine, y, torch.full((), -77.0, dtype=torch.float64))), bound


def test_a_session_with_accounts_claims_no_lower_bound_on_its_lengths(gpu_lib):
    """The descriptor's hint has to hold for every later call, also behind an eviction; one that is given is kept."""
    wl = paged([700, 900], 8, 2, 64, 8, torch.bfloat16, 2).to(DEV)
    assert DecodeSession(wl, track_weights=True).desc.min_seq_len_hint == 0
    assert DecodeSession(wl, track_weights=True, min_seq_len_hint=40).desc.min_seq_len_hint == 40
    assert DecodeSession(wl).desc.min_seq_len_hint == 700


def test_evict_from_two_tables(gpu_lib):
    """A pool of records and full-precision pages with a table each: both close up by the same accounts and lengths, which the second call changes."""
    S, Hkv, budget, lens = 8, 2, 6, [77, 30, 1600]
    g = torch.Generator().manual_seed(3)
    (table, pool), (records, _) = (tables(lens, S, g) for _ in range(2))
    w = torch.rand((3, Hkv, table.shape[1]), generator=g)
    geo = geometry(Hkv, Hkv, 64, S, torch.bfloat16, pool, table, lens)
    policy = dict(budget_pages=budget, sink_pages=1, recent_pages=2, weights=w.to(DEV))
    acc = PageAccounts(**policy, **geo)
    other = PageAccounts(**policy, **dict(geo, page_table=records.to(DEV)))
    w_out, l_out = torch.zeros_like(acc.weights), torch.zeros_like(geo["seq_lens"])
    other.evict_pages(weights_out=w_out, seq_lens_out=l_out)
    acc.evict_pages()
    torch.cuda.synchronize()
    args = torch.tensor(lens), w, S, (budget, 1, 2)
    check_evict(other, records, *args, other.page_table.cpu(), l_out.cpu(), w_out.cpu())
    check_evict(acc, table, *args, geo["page_table"].cpu(), geo["seq_lens"].cpu(), acc.weights.cpu())


def test_accounts_that_became_infinite_or_nan_stay_so(gpu_lib):
    """With any decay, for their page alone; from nothing they are finite again."""
    wl = paged([70, 33], 16, 4, 64, 8, torch.bfloat16, 9).to(DEV)
    sess = DecodeSession(wl, top_k=2, track_weights=True)
    for decay in (0.0, 0.5, 1.0):
        w, out = torch.rand_like(sess.page_weights), torch.zeros_like(sess.page_weights)
        w[0, 1, 2], w[1, 0, 1] = float("nan"), float("inf")
        sess.weighted_paged_decode(decay=decay, weights_in=w, weights_out=out)
        lost = torch.zeros_like(w, dtype=torch.bool)
        lost[0, 1, 2] = lost[1, 0, 1] = True
        assert torch.equal(~torch.isfinite(out), lost), decay
        sess.weighted_paged_decode(decay=decay, weights_out=out)
        assert torch.isfinite(out).all()
