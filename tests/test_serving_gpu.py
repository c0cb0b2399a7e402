"""Places for new tokens, their queries, keys and values, and attention over shared prefixes on the GPU against plain counterparts (serving_ref.py)."""
import math
import random

import pytest
import torch

from paper_2605_27740_amd import binding
from paper_2605_27740_amd.session import CacheWriter, PageAccounts, PagePool, PrefixGroups, rotary_frequencies
from tests import serving_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float32]


def say(*a):
    print(*a, flush=True)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------ places

def place_case(seed, B, S, width, most_len, most_new, free_share, *, ended=0.1, evicted=0, shared=True, own_positions=True, spare_rows=5):
    r = random.Random(seed)
    lens = [r.choice([0, 1, S - 1, S, r.randrange(most_len + 1)]) for _ in range(B)]
    lens = [min(n, width * S) for n in lens]
    new = [-r.randrange(1, 9) if r.random() < ended else r.choice([0, 1, 1, S, r.randrange(most_new + 1)]) for _ in range(B)]
    pages = [-(-n // S) for n in lens]
    freed_count = [r.randrange(evicted + 1) for _ in range(B)]
    need = sum(max(0, -(-(n + max(t, 0)) // S) - -(-n // S)) for n, t in zip(lens, new))
    free = int(need * free_share)
    total = sum(pages) + sum(freed_count) + free
    ids = list(range(total))
    r.shuffle(ids)
    take = iter(ids)
    table = [[next(take) for _ in range(p)] + [-1] * (width - p) for p in pages]
    freed = [[next(take) for _ in range(n)] + [-1] * (max(evicted, 1) - n) for n in freed_count]
    stack = list(take)
    c = dict(S=S, table=table, lens=lens, new=new, free=stack + [-7] * (total - len(stack) + 3), free_count=len(stack),
             rows=sum(max(t, 0) for t in new) + spare_rows)
    if shared:
        c["shared"] = [r.choice([0, 0, 2, p]) for p in pages]
    if own_positions:
        c["nxt"] = [n + S * r.randrange(4) for n in lens]
    if evicted:
        c.update(freed=freed, freed_count=freed_count)
    return c, max(total, 1)


def run_place(c, total, *, in_place, rows=None):
    table, lens, nxt, count = i32(c["table"]), i32(c["lens"]), i32(c["nxt"]) if "nxt" in c else None, i32([c["free_count"]])
    free = i32(c["free"])
    rows = c["rows"] if rows is None else rows
    pool = PagePool(q_heads=8, kv_heads=8, head_dim=64, page_size=c["S"], dtype=torch.float32, num_pages=total, page_table=table, seq_lens=lens,
                    max_new_tokens=rows, free_pages=free, free_count=count, shared_pages=i32(c["shared"]) if "shared" in c else None, next_positions=nxt)
    freed = {} if "freed" not in c else dict(freed_pages=i32(c["freed"]), freed_count=i32(c["freed_count"]))
    outs = {}
    if not in_place:
        outs = dict(page_table_out=table.clone(), seq_lens_out=torch.full_like(lens, -9), free_count_out=torch.full_like(count, -9))
        if nxt is not None:
            outs["next_positions_out"] = torch.full_like(nxt, -9)
    pool.place_tokens(i32(c["new"]), **freed, **outs)
    torch.cuda.synchronize()
    table_out, lens_out = (table, lens) if in_place else (outs["page_table_out"], outs["seq_lens_out"])
    nxt_out, count_out = (nxt, count) if in_place else (outs.get("next_positions_out"), outs["free_count_out"])
    if not in_place:
        assert table.tolist() == c["table"] and lens.tolist() == c["lens"] and count.tolist() == [c["free_count"]]
    return dict(table=table_out.tolist(), seq_lens=lens_out.tolist(), next=None if nxt_out is None else nxt_out.tolist(), placed=pool.placed.tolist(),
                token_starts=pool.token_starts.tolist(), positions=pool.positions.tolist(), slots=pool.slots.tolist(),
                stack=free.tolist()[:int(count_out)])


def check_place(c, total, **how):
    got = run_place(c, total, **how)
    want = R.place(**{**c, "rows": how.get("rows", c["rows"]) if how.get("rows") is not None else c["rows"]})
    for key, x in got.items():
        if x is not None:
            assert x == want[key], key


PLACE = [  # B, S, width, longest, most new, share of the needed pages that are free
    (1, 16, 40, 100, 1, 1.0), (1, 8, 3, 20, 30, 1.0), (64, 16, 70, 800, 1, 1.1), (257, 32, 20, 300, 70, 0.7), (1024, 8, 12, 60, 9, 0.9),
    (1025, 16, 9, 60, 40, 0.8), (3000, 8, 30, 100, 20, 1.2), (7, 16, 3000, 9000, 12000, 1.0), (40, 32, 400, 4000, 3000, 0.6), (2100, 16, 5, 64, 3, 0.0)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", PLACE)
def test_places_as_one_after_the_other(gpu_lib, case, in_place):
    """Small and large calls; sequences that end, do not fit their row, or find no pages; lengths 0, 1 and around a page."""
    say(f"place {case} in_place={in_place}")
    for seed, more in ((1, dict()), (2, dict(evicted=3)), (3, dict(ended=0.0, shared=False, own_positions=False)), (4, dict(ended=0.9, evicted=1))):
        c, total = place_case(seed + case[0], *case, **more)
        check_place(c, total, in_place=in_place)


@pytest.mark.parametrize("rows", [0, 1, 50, 8192, 8193])
def test_rows_that_are_not_there(gpu_lib, rows):
    """Fewer rows than new tokens: the last sequences get no place; more: -1 behind the last."""
    say(f"rows {rows}")
    c, total = place_case(5, 60, 16, 40, 200, 30, 2.0)
    check_place(c, total, in_place=False, rows=rows)
    check_place(c, total, in_place=True, rows=rows)


@pytest.mark.parametrize("B", [900, 1024, 5000])
def test_places_of_few_among_many(gpu_lib, B):
    """Long runs of sequences without new tokens between those that have some, and rows of one sequence over many workgroups."""
    for where in ([3, B - 20], [0, 1, 2, 70, 71, 500, B - 1], [B // 2]):
        r = random.Random(B)
        c, total = place_case(B, B, 16, 4, 60, 1, 0.0, ended=0.0, shared=False)
        c["table"] = [row + [-1] * 600 for row in c["table"]]
        c["new"] = [0] * B
        for b in where:
            c["new"][b] = r.choice([1, 9000])
        c["new"][where[0]] = 9000
        need = sum(-(-(n + t) // 16) - -(-n // 16) for n, t in zip(c["lens"], c["new"]))
        c.update(free=list(range(total, total + need)), free_count=need, rows=sum(c["new"]) + 3)
        check_place(c, total + need, in_place=True)


def test_a_stack_that_is_too_small_loses_what_does_not_fit(gpu_lib):
    c, total = place_case(6, 50, 8, 30, 200, 10, 0.5, ended=0.6, evicted=2)
    c["free"] = c["free"][:c["free_count"] + 11]
    for how in (False, True):
        check_place(c, total, in_place=how)


# ------------------------------------------------------------------ queries, keys and values

def append_bound(y, size, dtype):
    """The one rounding, and the work in 32 bits. With u = 2^-24: a sum of 128 squares is off by 128 u, so its root by 64 u, division, root and two
    products 4 u; the angle is off by 2 pi (2^-25 + 2^-33) < 4 u of a radian, sine and cosine by 4 u more, the factor, products and sum by 4 u: 80 u of
    |y_1| + |y_2| in all. Below the smallest normal number of the type a step is absolute."""
    return torch.finfo(dtype).eps / 2 * y.abs() + 80 * 2.0 ** -24 * size * (1 + 2.0 ** -7) + torch.finfo(dtype).tiny


def run_append(dtype, H, Hkv, D, S, rows, *, rotary, interleaved, norm, magnitude, fused, far=0, in_place=False, strided=False, seed=0, scaled=False):
    g = torch.Generator().manual_seed(seed + D + rows)
    pages = rows // S + 7
    x = torch.randn((rows, H + 2 * Hkv, D), generator=g)
    x[..., 3] *= 50
    x = x.to(dtype)
    q, k, v = x.split([H, Hkv, Hkv], 1)
    slots = torch.randperm(pages * S, generator=g)[:rows]
    slots[::5] = -1 - torch.arange(slots[::5].numel())
    slots[3::11] = pages * S + 1  # outside the pool
    positions = (torch.randint(0, 5000, (rows,), generator=g) + far).int()
    shape = (pages, Hkv, 2, S, D) if strided else (pages, Hkv, S, D)
    caches = [torch.full(shape, -3.0, dtype=dtype, device=DEV) for _ in range(2)]
    kc, vc = (caches[0][:, :, 0], caches[0][:, :, 1]) if strided else caches
    w = [(1 + 0.3 * torch.randn((D,), generator=g)).to(dtype) for _ in range(2)] if norm else [None, None]
    f = rotary_frequencies(rotary, base=5e5, **(dict(factor=8.0, trained_len=4096, low_turns=1.0, high_turns=4.0) if scaled else {}))
    writer = CacheWriter(q_heads=H, k_cache=kc, v_cache=vc, q_weight=None if w[0] is None else w[0].to(DEV), k_weight=None if w[1] is None else w[1].to(DEV),
                         eps=1e-5, frequencies=f, magnitude=magnitude, interleaved=interleaved)
    if fused:
        parts = x.to(DEV).split([H, Hkv, Hkv], 1)
    else:
        parts = [p.contiguous().to(DEV) for p in (q, k, v)]
    q_out = parts[0] if in_place else torch.full((rows, H, D), -5.0, dtype=dtype, device=DEV)
    got = writer.append_tokens(*parts, positions.to(DEV), slots.to(DEV), q_out=q_out).cpu()
    torch.cuda.synchronize()
    here = (slots >= 0) & (slots < pages * S)
    (yq, sq), (yk, sk) = (R.heads(t, u, 1e-5, positions, f, magnitude, interleaved) for t, u in ((q, w[0]), (k, w[1])))
    assert torch.equal(got[~here], q[~here] if in_place else torch.full_like(q[~here], -5.0)), "rows without a slot"
    assert ((got[here].double() - yq[here]).abs() <= append_bound(yq, sq, dtype)[here]).all()
    kg, vg = (t.cpu().transpose(1, 2).reshape(pages * S, Hkv, D) for t in (kc, vc))
    mine = slots[here]
    assert ((kg[mine].double() - yk[here]).abs() <= append_bound(yk, sk, dtype)[here]).all()
    assert torch.equal(vg[mine], v[here])
    others = torch.ones(pages * S, dtype=torch.bool)
    others[mine] = False
    assert (kg[others] == -3).all() and (vg[others] == -3).all(), "slots that no row has"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,H,Hkv,S", [(128, 32, 8, 16), (64, 8, 2, 8), (128, 1, 1, 32), (64, 32, 32, 16), (128, 64, 8, 8), (64, 2, 1, 32)])
@pytest.mark.parametrize("rows", [1, 37])
def test_append_every_rotation(gpu_lib, dtype, D, H, Hkv, S, rows):
    for rotary in [r for r in (0, 16, 48, 64, 96, 128) if r <= D]:
        for interleaved in (False, True):
            for norm in (False, True):
                say(f"append {dtype} {(D, H, Hkv, S)} rows={rows} R={rotary} interleaved={interleaved} norm={norm}")
                run_append(dtype, H, Hkv, D, S, rows, rotary=rotary, interleaved=interleaved, norm=norm, magnitude=1.0, fused=rotary % 32 == 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("far", [1 << 20, (1 << 31) - 6000])
def test_append_far_positions_scaled(gpu_lib, dtype, far):
    say(f"append {dtype} far={far}")
    run_append(dtype, 16, 4, 128, 16, 600, rotary=128, interleaved=False, norm=True, magnitude=1.2, fused=True, far=far, scaled=True)
    run_append(dtype, 16, 4, 64, 8, 601, rotary=32, interleaved=True, norm=False, magnitude=0.7, fused=False, far=far, scaled=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_append_in_place_and_into_a_strided_cache(gpu_lib, dtype):
    say(f"append strides {dtype}")
    run_append(dtype, 16, 4, 128, 16, 5000, rotary=64, interleaved=False, norm=True, magnitude=1.0, fused=False, in_place=True)
    run_append(dtype, 8, 8, 64, 32, 333, rotary=64, interleaved=True, norm=True, magnitude=1.0, fused=True, strided=True)


def test_append_without_a_transform_copies(gpu_lib):
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((9, h, 128), generator=g).bfloat16().to(DEV) for h in (8, 2, 2))
    kc, vc = (torch.zeros((4, 2, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    slots = torch.arange(9, device=DEV) + 11
    out = CacheWriter(q_heads=8, k_cache=kc, v_cache=vc).append_tokens(q, k, v, i32(list(range(9))), slots)
    torch.cuda.synchronize()
    assert torch.equal(out, q)
    for cache, x in ((kc, k), (vc, v)):
        assert torch.equal(cache.transpose(1, 2).reshape(32, 2, 128)[11:20], x)


# ------------------------------------------------------------------ shared prefixes

def prefix_case(dtype, H, Hkv, D, S, groups, *, seed=0, loose=0, poison=True, extra_cols=0):
    """groups: (members' own tokens, prefix pages); a negative number of own tokens makes a member so many tokens shorter than its prefix. `loose`
    sequences are in no group."""
    g = torch.Generator().manual_seed(seed + D + S)
    n = sum(len(own) for own, _ in groups)
    B = n + loose
    where = torch.randperm(B, generator=g)
    lens, rows = [0] * B, [[] for _ in range(B)]
    ids = iter(torch.randperm(20 + sum(p + sum(-(-max(t, 0) // S) for t in own) for own, p in groups) + 3 * loose, generator=g).tolist())
    starts, at = [0], 0
    for own, p in groups:
        shared = [next(ids) for _ in range(p)]
        for t in own:
            b = int(where[at])
            lens[b] = max(p * S + t, 0)
            rows[b] = shared + [next(ids) for _ in range(-(-max(t, 0) // S))]
            at += 1
        starts.append(at)
    for b in where[at:].tolist():
        lens[b], rows[b] = 2 * S + 1, [next(ids) for _ in range(3)]
    width = max(len(r) for r in rows) + extra_cols
    table = torch.tensor([r + [-1] * (max(width, 1) - len(r)) for r in rows], dtype=torch.int32)
    pool = max(max(r, default=0) for r in rows) + 2
    k, v = (torch.full((pool, Hkv, S, D), math.nan if poison else 0.0) for _ in range(2))
    for b in range(B):
        for p, ph in enumerate(rows[b]):
            used = S if any(p < q and b in where[s:e].tolist() for (_, q), s, e in zip(groups, starts, starts[1:])) else max(0, min(S, lens[b] - p * S))
            if torch.isnan(k[ph, 0, 0, 0]) or not poison:
                k[ph, :, :used] = torch.randn((Hkv, used, D), generator=g)
                v[ph, :, :used] = torch.randn((Hkv, used, D), generator=g)
    q = torch.randn((B, H, D), generator=g) * 1.5
    return dict(q=q.to(dtype), k=k.to(dtype), v=v.to(dtype), table=table, lens=torch.tensor(lens, dtype=torch.int32), starts=starts, members=where[:n].int(),
                pages=[p for _, p in groups], groups=groups, S=S)


def make_groups(c, H, wide=True, **over):
    """wide: rows of the page table that are long enough (by entries that no sequence reaches) for the batch not to be one of little to read, where every member reads its prefix
    for itself."""
    table = c["table"]
    if wide:
        columns = max((256 << 20) // (len(c["lens"]) * c["k"][0].numel() * 2 * c["k"].element_size()), 768 // c["S"]) + 1
        table = torch.nn.functional.pad(table, (0, max(0, columns - table.shape[1])), value=-1)
    args = dict(q_heads=H, k_cache=c["k"].to(DEV), v_cache=c["v"].to(DEV), page_table=table.to(DEV), seq_lens=c["lens"].to(DEV),
                group_starts=i32(c["starts"]), prefix_pages=i32(c["pages"]), members=torch.cat([c["members"], c["members"].new_zeros(len(c["lens"]))]).to(DEV),
                max_members=max(len(own) for own, _ in c["groups"]), max_prefix_pages=max(c["pages"]))
    args.update(over)
    return PrefixGroups(**args)


def prefix_bounds(c, want, dtype):
    """u = 2^-24. A logit is a sum of D products, off by (D + 2) u of the sum of |q k|, so a weight by twice that relatively (its own and the normaliser's); exponentials and
    their arguments 2^-21 of a weight, sums of n tokens n u. bf16: probabilities and the output are rounded, half a step each."""
    out, lse, terms, reach = want
    n = c["lens"].double()[:, None]
    rel = 2 * (c["q"].shape[-1] + 2) * 2.0 ** -24 * reach + 2.0 ** -20 + 2 * n * 2.0 ** -24
    half = 2.0 ** -8 if dtype is torch.bfloat16 else 0.0
    return (rel + half)[..., None] * terms * (1 + half) + half * out.abs(), rel + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0.0)


def check_prefix(c, got, dtype, want=None):
    out, lse = (x.cpu() for x in got)
    want = want or R.attend(c["q"], c["k"], c["v"], c["table"], c["lens"])
    listed = torch.zeros(len(c["lens"]), dtype=torch.bool)
    listed[c["members"].long()] = True
    tol, tol_lse = prefix_bounds(c, want, dtype)
    some = listed & (c["lens"] > 0)
    assert ((out.double() - want[0]).abs() <= tol)[some].all(), float(((out.double() - want[0]).abs() / tol)[some].max())
    assert ((lse.double() - want[1]).abs() <= tol_lse)[some].all(), float((lse.double() - want[1])[some].abs().max())
    none = listed & (c["lens"] == 0)
    assert (out[none] == 0).all() and torch.isneginf(lse[none]).all()
    return listed


def check_both(c, H, dtype, check=None, **over):
    """Prefixes shared, and read by every member for itself."""
    want = R.attend(c["q"], c["k"], c["v"], c["table"], c["lens"])
    for wide in (True, False):
        (check or check_prefix)(c, make_groups(c, H, wide=wide, **over).paged_decode(c["q"].to(DEV)), dtype, want)


PREFIX = [
    [([5], 3)],
    [([0, 1, 40], 1)],
    [([17] * 9, 20), ([1, 2, 3], 0), ([100], 7)],
    [([3] * 33, 9), ([0] * 2, 33)],
    [([-1, 7, -20, 2], 4), ([-10000, 0], 2)],
    [(list(range(70)), 5)],
    [([11] * 130, 6)],
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,H,Hkv,S", [(128, 8, 2, 16), (64, 8, 8, 8), (128, 8, 1, 32), (64, 4, 2, 16), (128, 4, 1, 8), (64, 8, 1, 32)])
@pytest.mark.parametrize("which", range(len(PREFIX)))
def test_prefix_groups_of_all_kinds(gpu_lib, dtype, D, H, Hkv, S, which):
    """Few and many members, prefixes of no, one and odd numbers of pages, own parts of 0 tokens and more, members that are shorter than their
    prefix or empty, sequences in no group; unwritten slots hold NaN."""
    say(f"prefix {dtype} {(D, H, Hkv, S)} case {which}")
    c = prefix_case(dtype, H, Hkv, D, S, PREFIX[which], seed=which, loose=2, extra_cols=which % 3)
    want = R.attend(c["q"], c["k"], c["v"], c["table"], c["lens"])
    for wide in (True, False):
        groups = make_groups(c, H, wide=wide)
        groups.out.fill_(-7.0)
        groups.lse.fill_(-7.0)
        got = groups.paged_decode(c["q"].to(DEV))
        torch.cuda.synchronize()
        listed = check_prefix(c, got, dtype, want)
        assert (got[0][~listed.to(DEV)] == -7).all() and (got[1][~listed.to(DEV)] == -7).all(), "sequences in no group"


def holes(c, seed):
    """Entries of prefixes and of own pages that are no pages: -1 and ids beyond the pool."""
    r = random.Random(seed)
    pool, S = c["k"].shape[0], c["S"]
    for g, (own, p) in enumerate(c["groups"]):
        rows = c["members"][c["starts"][g]:c["starts"][g + 1]].tolist()
        for i in r.sample(range(p), min(p, max(1, p // 5))):
            c["table"][rows, i] = r.choice([-1, -7, pool, 2 ** 31 - 1])
        for b in rows:
            n = -(-int(c["lens"][b]) // S)
            if n > p and r.random() < 0.7:
                c["table"][b, r.randrange(p, n)] = r.choice([-1, pool + 3])
    return c


def check_holes(c, got, dtype, want=None):
    """A sequence all of whose pages are missing is as an empty one."""
    S, pool = c["S"], c["k"].shape[0]
    lens = c["lens"].clone()
    for b, n in enumerate(lens.tolist()):
        ids = c["table"][b, :-(-n // S)]
        if not bool(((ids >= 0) & (ids < pool)).any()):
            lens[b] = 0
    check_prefix(dict(c, lens=lens), got, dtype, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,H,Hkv,S", [(128, 8, 2, 16), (64, 8, 8, 8), (128, 8, 1, 32)])
@pytest.mark.parametrize("which", range(len(PREFIX)))
def test_prefix_pages_that_are_not_there(gpu_lib, dtype, D, H, Hkv, S, which):
    say(f"holes {dtype} {(D, H, Hkv, S)} case {which}")
    c = holes(prefix_case(dtype, H, Hkv, D, S, PREFIX[which], seed=40 + which, loose=1), which)
    check_both(c, H, dtype, check_holes)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("S,pages", [(16, 511), (16, 513), (8, 1500), (8, 4100), (32, 700)])
def test_prefix_windows_and_long_items(gpu_lib, dtype, S, pages):
    """One KV head and few or many rows: items of many windows of page ids, their last tiles cut; two groups of different lengths."""
    say(f"long {dtype} S={S} pages={pages}")
    for own, H in (([3, 50], 2), ([9] * 20, 8), ([1] * 70, 8)):
        c = prefix_case(dtype, H, 1, 64, S, [(own, pages), ([2, 2], pages // 3)], seed=pages, poison=False)
        check_both(c, H, dtype)
    c = holes(c, 1)
    check_both(c, H, dtype, check_holes)


@pytest.mark.parametrize("own_tokens", [0, 90])
def test_prefix_items_of_the_most_pages(gpu_lib, own_tokens):
    """So many groups that an item may be as long as its page ids reach: 20 prefixes of 2000 pages with 8 heads."""
    c = prefix_case(torch.bfloat16, 8, 8, 64, 8, [([7, 5], 2000)] * 20, seed=3, poison=False)
    want = make_groups(c, 8, max_own_tokens=own_tokens)
    check_prefix(c, want.paged_decode(c["q"].to(DEV)), torch.bfloat16)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,D,S", [(8, 128, 16), (2, 64, 32), (8, 64, 8)])
def test_prefix_that_nobody_fills(gpu_lib, dtype, H, D, S):
    """Samples of one prompt before their first token: the last page of the prefix is not full, and what lies behind its tokens is NaN; then members that all end
    pages before the prefix does, and by different amounts in different blocks of rows."""
    for owns in ([-1] * 3, [-S + 1] * 40, [-3 * S - 5] * 5, [-9 - i for i in range(2 * S)], [-7 * S - i for i in range(70)], [-10 ** 6, -10 ** 6]):
        for pages in (9, 40):
            c = prefix_case(dtype, H, 2, D, S, [(owns, pages)], seed=pages)
            for key in ("k", "v"):
                row = c["table"][c["members"][0].long()].long()[:pages]
                flat = c[key][row].transpose(1, 2).reshape(pages * S, 2, D)
                flat[int(c["lens"].max()):] = math.nan
                c[key][row] = flat.view(pages, S, 2, D).transpose(1, 2)
            check_both(c, H, dtype)


@pytest.mark.parametrize("n,each", [(120, 2), (300, 2), (700, 2), (1030, 1), (600, 3)])
def test_prefix_many_groups(gpu_lib, n, each):
    """Plans of up to 255 sources, up to 1023, and more."""
    say(f"groups {n} of {each}")
    r = random.Random(n)
    c = prefix_case(torch.float32, 2, 1, 64, 8, [([r.randrange(30) for _ in range(each)], r.randrange(4)) for _ in range(n)], seed=n, loose=3, poison=False)
    check_both(c, 2, torch.float32)


@pytest.mark.parametrize("loose", [0, 300, 1100])
def test_prefix_members_that_are_none(gpu_lib, loose):
    """-1 and numbers outside the batch among the members, also as a group's first; without a list; the number of groups' bounds used up."""
    c = prefix_case(torch.bfloat16, 8, 2, 128, 16, [([17] * 5, 9), ([100, 3, 40], 20), ([5, 6], 0)], seed=8, loose=loose)
    listed = c["members"].tolist()
    for at, gone in ((0, -1), (5, len(c["lens"]) + 4), (6, -1), (9, -5)):
        c["members"][at] = gone
    there = [b for b in c["members"].tolist() if 0 <= b < len(c["lens"])]
    gone = sorted(set(listed) - set(there))
    for wide in (True, False):
        groups = make_groups(c, 8, wide=wide)
        groups.out.fill_(-7.0)
        got = groups.paged_decode(c["q"].to(DEV))
        torch.cuda.synchronize()
        assert (got[0].cpu()[gone] == -7).all()
        check_prefix(dict(c, members=torch.tensor(there, dtype=torch.int32)), got, torch.bfloat16)


def test_prefix_without_a_list_of_members(gpu_lib):
    c = prefix_case(torch.bfloat16, 8, 2, 128, 16, [([17] * 5, 9), ([100, 3, 40], 20)], seed=9)
    order = c["members"].long()
    for key in ("q", "table", "lens"):
        c[key] = c[key][order]
    c["members"] = torch.arange(8, dtype=torch.int32)
    check_both(c, 8, torch.bfloat16, members=None)


@pytest.mark.parametrize("loose", [0, 400, 1200])
def test_prefix_starts_that_do_not_ascend_write_nothing(gpu_lib, loose):
    """Refused on the device: the plan sees it, there are no items and no members."""
    c = prefix_case(torch.float32, 8, 2, 64, 16, [([17] * 5, 9), ([100, 3, 40], 20), ([4, 4], 2)], seed=9, loose=loose)
    n = c["starts"][-1]
    for starts, wide in [(x, w) for x in ([0, n, 0, n], [0, 5, 4, n], [n, 0, 0, 0]) for w in (True, False)]:
        groups = make_groups(c, 8, wide=wide, group_starts=i32(starts), max_members=n)
        groups.out.fill_(-7.0)
        groups.lse.fill_(-7.0)
        out, lse = groups.paged_decode(c["q"].to(DEV))
        torch.cuda.synchronize()
        assert (out == -7).all() and (lse == -7).all()


def test_prefix_bounds_hold(gpu_lib):
    """What lies beyond the host's bounds does not count: members, pages of prefixes, own pages."""
    c = prefix_case(torch.float32, 8, 2, 64, 16, [([30, 100, 70, 1], 6), ([200, 90], 3)], seed=4, poison=False)
    first = c["members"][:2].tolist() + c["members"][4:].tolist()
    rest = [b for b in c["members"].tolist() if b not in first]
    for wide in (True, False):
        groups = make_groups(c, 8, wide=wide, max_members=2)
        groups.out.fill_(-7.0)
        out, _ = groups.paged_decode(c["q"].to(DEV))
        assert (out[rest] == -7).all()
        check_prefix(dict(c, members=torch.tensor(first, dtype=torch.int32)), (groups.out, groups.lse), torch.float32)
    # own pages: two of each
    d = dict(c, lens=torch.minimum(c["lens"], torch.tensor([96 + 32 if b in c["members"][:4].tolist() else 48 + 32 for b in range(6)], dtype=torch.int32)))
    for more in ({}, dict(max_prefix_pages=1 << 16)):  # (the latter: prefixes are shared)
        check_prefix(d, make_groups(c, 8, max_own_tokens=32, **more).paged_decode(c["q"].to(DEV)), torch.float32)


def test_prefix_a_member_listed_twice_and_other_scales(gpu_lib):
    c = prefix_case(torch.bfloat16, 8, 2, 128, 16, [([30, 100, 30], 6)], seed=5, loose=3)
    twice = c["members"].tolist() + [c["members"][1].item()]
    want = [x.clone() for x in make_groups(c, 8).paged_decode(c["q"].to(DEV), sm_scale=1.0 / math.sqrt(128))]
    check_both(c, 8, torch.bfloat16, group_starts=i32([0, 4]), members=i32(twice + [0] * 6), max_members=4)
    small = make_groups(c, 8)
    half = dict(c, q=c["q"] * 0.5)  # exact
    got = small.paged_decode(half["q"].to(DEV), sm_scale=2.0 / math.sqrt(128))
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_prefix_strided_caches(gpu_lib, dtype):
    """Keys and values of a page next to each other, and heads apart."""
    c = prefix_case(dtype, 8, 2, 128, 16, [([30, 100, 0], 70), ([5] * 9, 3)], seed=6)
    P, Hkv, S, D = c["k"].shape
    both = torch.full((P, Hkv, 2, S, D), math.nan, dtype=dtype, device=DEV)
    both[:, :, 0], both[:, :, 1] = c["k"].to(DEV), c["v"].to(DEV)
    check_both(c, 8, dtype, k_cache=both[:, :, 0], v_cache=both[:, :, 1])
    apart = [torch.full((P + 1, Hkv, S, D), math.nan, dtype=dtype, device=DEV) for _ in range(2)]
    room = torch.cat([apart[1], apart[0]])  # values before keys
    k, v = room[P + 1:2 * P + 1], room[:P]
    k.copy_(c["k"]), v.copy_(c["v"])
    check_both(c, 8, dtype, k_cache=k, v_cache=v)


def test_prefix_without_lse_and_far_pages(gpu_lib):
    """No lse is wanted; pages beyond 2^31 elements of the cache, 2^32 bytes."""
    c = prefix_case(torch.bfloat16, 8, 2, 128, 16, [([30, 100, 0], 40)], seed=7, poison=False)
    P, Hkv, S, D = c["k"].shape
    pages = (1 << 31) // (Hkv * S * D) + P + 9
    k, v = (torch.empty((pages, Hkv, S, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k[-P:], v[-P:] = c["k"].to(DEV), c["v"].to(DEV)
    table = torch.where(c["table"] < 0, -1, c["table"] + (pages - P))
    groups = make_groups(c, 8, k_cache=k, v_cache=v, page_table=table.to(DEV))
    check_prefix(c, groups.paged_decode(c["q"].to(DEV)), torch.bfloat16)
    want = groups.out.clone()
    groups.out.zero_()
    lib = groups.lib
    lib.shared_prefix_decode(groups.desc, groups.groups, c["q"].to(DEV), 0.0, groups.out, None, groups.workspace)
    torch.cuda.synchronize()
    assert torch.equal(groups.out, want)


# ------------------------------------------------------------------ together

class Server:
    """A batch that decodes: places for the new tokens, heads into the cache, statistics of the touched pages, attention over the prefix that all of its
    sequences share; with a plain copy of everything on the host."""

    def __init__(self, seed, dtype=torch.bfloat16, H=16, Hkv=4, D=128, S=16, B=6, prefix=5, pages=400, rows=64, width=1600):
        self.geo = H, Hkv, D, S, B, prefix
        self.dtype, self.g = dtype, torch.Generator().manual_seed(seed)
        self.r = random.Random(seed)
        self.kc, self.vc = (torch.zeros((pages, Hkv, S, D), dtype=dtype, device=DEV) for _ in range(2))
        ids = list(range(pages))
        self.r.shuffle(ids)
        self.prefix = [ids.pop() for _ in range(prefix)]
        for cache in (self.kc, self.vc):
            cache[self.prefix] = torch.randn((prefix, Hkv, S, D), generator=self.g).to(dtype).to(DEV)
        self.k, self.v = self.kc.cpu(), self.vc.cpu()  # the plain copies
        self.host = dict(S=S, table=[self.prefix + [-1] * (width - prefix) for _ in range(B)], lens=[prefix * S] * B, free=ids, free_count=len(ids),
                         rows=rows, capacity=len(ids), shared=[prefix] * B, nxt=[prefix * S + 1000 * b for b in range(B)])
        h = self.host
        self.table, self.lens, self.nxt, self.shared = i32(h["table"]), i32(h["lens"]), i32(h["nxt"]), i32(h["shared"])
        self.pool = PagePool(q_heads=H, kv_heads=Hkv, head_dim=D, page_size=S, dtype=dtype, num_pages=pages, page_table=self.table, seq_lens=self.lens,
                             max_new_tokens=rows, free_pages=i32(ids), free_count=i32([len(ids)]), shared_pages=self.shared, next_positions=self.nxt)
        self.weights = [(1 + 0.2 * torch.randn((D,), generator=self.g)).to(dtype) for _ in range(2)]
        self.f = rotary_frequencies(D // 2, base=5e5)
        self.writer = CacheWriter(q_heads=H, k_cache=self.kc, v_cache=self.vc, q_weight=self.weights[0].to(DEV), k_weight=self.weights[1].to(DEV),
                                  frequencies=self.f)
        self.groups = PrefixGroups(q_heads=H, k_cache=self.kc, v_cache=self.vc, page_table=self.table, seq_lens=self.lens, group_starts=i32([0, B]),
                                   prefix_pages=i32([prefix]), max_members=B, max_prefix_pages=prefix)
        self.new = torch.zeros((B,), dtype=torch.int32, device=DEV)
        self.x = torch.zeros((rows, H + 2 * Hkv, D), dtype=dtype, device=DEV)
        self.q_out = torch.zeros((rows, H, D), dtype=dtype, device=DEV)
        self.q = torch.zeros((B, H, D), dtype=dtype, device=DEV)
        self.out, self.lse = torch.zeros_like(self.groups.out), torch.zeros_like(self.groups.lse)

    def step(self):
        """What the server launches, and a graph records."""
        H, Hkv = self.geo[:2]
        self.pool.place_tokens(self.new)
        self.writer.append_tokens(*self.x.split([H, Hkv, Hkv], 1), self.pool.positions, self.pool.slots, q_out=self.q_out)
        last = (self.pool.token_starts[1:] - 1).clamp(min=0).long()  # each sequence's last new token asks
        torch.index_select(self.q_out, 0, last, out=self.q)
        self.groups.paged_decode(self.q)

    def inputs(self, new):
        rows = self.x.shape[0]
        self.asked = new
        self.xh = torch.randn(self.x.shape, generator=self.g).to(self.dtype)
        self.new.copy_(i32(new))
        self.x.copy_(self.xh)

    def check(self):
        H, Hkv, D, S, B, prefix = self.geo
        torch.cuda.synchronize()
        h = self.host
        want = R.place(**{**h, "new": self.asked})
        assert self.table.tolist() == want["table"] and self.lens.tolist() == want["seq_lens"] and self.nxt.tolist() == want["next"]
        assert self.pool.slots.tolist() == want["slots"] and self.pool.positions.tolist() == want["positions"] and self.pool.placed.tolist() == want["placed"]
        assert self.pool.free_pages[:int(self.pool.free_count)].tolist() == want["stack"]
        h.update(table=want["table"], lens=want["seq_lens"], nxt=want["next"], free=want["stack"], free_count=len(want["stack"]))
        slots, positions = torch.tensor(want["slots"]), torch.tensor(want["positions"])
        here = slots >= 0
        q, k, v = self.xh.split([H, Hkv, Hkv], 1)
        got_k, got_v = self.kc.cpu(), self.vc.cpu()
        for x, w, got in ((q, self.weights[0], self.q_out.cpu()), (k, self.weights[1], got_k.transpose(1, 2).reshape(-1, Hkv, D)[slots.clamp(min=0)])):
            y, size = R.heads(x, w, 1e-6, positions, self.f, 1.0, False)
            assert ((got.double() - y).abs() <= append_bound(y, size, self.dtype))[here].all()
        # the keys as they were rounded, from here on
        at = slots[here]
        self.k[at // S, :, at % S] = got_k[at // S, :, at % S]
        self.v[at // S, :, at % S] = v[here]
        assert torch.equal(got_k, self.k) and torch.equal(got_v, self.v)
        c = dict(q=self.q.cpu(), k=self.k, v=self.v, table=self.table.cpu(), lens=self.lens.cpu(), members=torch.arange(B))
        check_prefix(c, (self.groups.out, self.groups.lse), self.dtype)


    def admit(self):
        """Sequences that have ended make room for others with the same prefix."""
        S, prefix, h = self.geo[3], self.geo[5], self.host
        for b, n in enumerate(self.asked):
            if n < 0:
                h["table"][b][:prefix] = self.prefix
                h["lens"][b], h["nxt"][b] = prefix * S, prefix * S + 7
                self.table[b, :prefix] = i32(self.prefix)
                self.lens[b], self.nxt[b] = prefix * S, prefix * S + 7


def asked(r, i, B):
    """Tokens of a step: most decode, some bring a few, in some steps one ends."""
    new = [r.choice([1, 1, 1, 5, 0]) for _ in range(B)]
    if i % 5 == 4:
        new[i // 5 % B] = -1  # also the first
    return new


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [40, 1600])
def test_a_server_places_appends_and_attends(gpu_lib, dtype, captured, width):
    """Thirty steps, every one against the host's copy; eager, or one HIP graph replayed with work of other kinds between the replays. Tables of 40 pages: every sequence reads
    the prefix for itself; of 1600: it is shared."""
    s = Server(11, dtype, width=width)
    graph = None
    for i in range(30):
        new = asked(s.r, i, s.geo[4])
        s.inputs(new)
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


def test_two_servers_on_two_streams(gpu_lib):
    """Each behind a long kernel of its own stream, with objects of its own."""
    servers = [Server(21), Server(22, prefix=30, B=9)]
    streams = [torch.cuda.Stream() for _ in servers]
    big = torch.randn((4096, 4096), device=DEV)
    for i in range(3):
        for s in servers:
            s.inputs(asked(s.r, 0, s.geo[4]))
        torch.cuda.synchronize()
        for s, stream in zip(servers, streams):
            with torch.cuda.stream(stream):
                big @ big
                s.step()
        torch.cuda.synchronize()
        for s in servers:
            s.check()


@pytest.mark.parametrize("captured", [False, True])
def test_evicted_pages_are_given_out_again(gpu_lib, captured):
    """Placement and eviction in turn on one table: what an eviction frees goes back at the next placement, no page is lost or held twice, and positions run on."""
    B, S, Hkv, budget, width, pages = 5, 8, 2, 6, 16, 60
    r = random.Random(3)
    table, lens, nxt = torch.full((B, width), -1, dtype=torch.int32, device=DEV), i32([0] * B), i32([0] * B)
    geo = dict(q_heads=4, kv_heads=Hkv, head_dim=64, page_size=S, dtype=torch.float32, num_pages=pages, page_table=table, seq_lens=lens)
    pool = PagePool(max_new_tokens=64, next_positions=nxt, **geo)
    acc = PageAccounts(budget_pages=budget, sink_pages=1, recent_pages=2, **geo)
    new = i32([0] * B)
    host = dict(S=S, table=table.tolist(), lens=[0] * B, nxt=[0] * B, free=list(range(pages)), free_count=pages, rows=64, capacity=pages)

    def step():
        pool.place_tokens(new, acc.freed_pages, acc.freed_count)

    graph = None
    for i in range(60):
        asked = [r.choice([1, 1, 9, 3, 0, -1 if i % 7 == 6 else 1]) for _ in range(B)]
        new.copy_(i32(asked))
        freed, count = acc.freed_pages.tolist(), acc.freed_count.tolist()
        if captured and graph is None and i == 3:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                step()
        if graph is not None:
            graph.replay()
        else:
            step()
        torch.cuda.synchronize()
        want = R.place(**{**host, "new": asked, "freed": freed, "freed_count": count})
        for key, x in (("table", table), ("seq_lens", lens), ("next", nxt), ("placed", pool.placed), ("slots", pool.slots), ("positions", pool.positions)):
            assert x.tolist() == want[key], (i, key)
        assert pool.free_pages[:int(pool.free_count)].tolist() == want["stack"]
        acc.weights.copy_(torch.rand(acc.weights.shape))
        acc.evict_pages()
        torch.cuda.synchronize()
        held = [p for row, n in zip(table.tolist(), lens.tolist()) for p in row[:-(-n // S)]]
        back = [p for row, n in zip(acc.freed_pages.tolist(), acc.freed_count.tolist()) for p in row[:n]]
        assert sorted(held + back + want["stack"]) == list(range(pages)) and max(lens.tolist()) <= budget * S
        host.update(table=table.tolist(), lens=lens.tolist(), nxt=want["next"], free=want["stack"], free_count=len(want["stack"]))
        if i % 10 == 0:
            torch.randn((256, 256), device=DEV).sum().item()


def test_prefix_random_batches(gpu_lib):
    """Shapes, groups and bounds drawn together."""
    for seed in range(40):
        r = random.Random(seed)
        dtype, D, S, Hkv, G = r.choice(DTYPES), r.choice([64, 128]), r.choice([8, 16, 32]), r.choice([1, 2, 4, 8]), r.choice([1, 2, 4, 8])
        groups = [([r.choice([0, 1, r.randrange(300), -r.randrange(3 * S)]) for _ in range(r.choice([1, 1, 2, 3, 20, 60]))], r.choice([0, 1, r.randrange(60), r.randrange(300)]))
                  for _ in range(r.choice([1, 2, 6]))]
        say(f"random {seed}: {dtype} D={D} S={S} Hkv={Hkv} G={G} groups={[(len(o), p) for o, p in groups]}")
        c = prefix_case(dtype, G * Hkv, Hkv, D, S, groups, seed=seed, loose=r.randrange(3), extra_cols=r.randrange(4), poison=r.random() < 0.7)
        most = max(max(o) for o, _ in groups)
        bounds = r.choice([{}, dict(max_own_tokens=max(most, 1)), dict(max_seq_len=max(int(c["lens"].max()), 1)),
                           dict(max_members=len(c["lens"]) + 3, max_prefix_pages=c["table"].shape[1] + 7)])
        check_both(c, G * Hkv, dtype, **bounds)


def test_objects_refuse_what_does_not_fit(gpu_lib):
    """Types, shapes and strides that the calls cannot see."""
    table, lens = torch.full((2, 8), -1, dtype=torch.int32, device=DEV), i32([0, 0])
    geo = dict(q_heads=4, kv_heads=2, head_dim=64, page_size=8, dtype=torch.float32, num_pages=16, page_table=table, seq_lens=lens, max_new_tokens=4)
    with pytest.raises(AssertionError):
        PagePool(free_pages=i32([1, 2]), **geo)
    with pytest.raises(AssertionError):
        PagePool(shared_pages=i32([1]), **geo)
    pool = PagePool(**geo)
    for bad in (i32([1]), torch.tensor([1, 1], device=DEV), torch.tensor([1, 1], dtype=torch.int32)):
        with pytest.raises(AssertionError):
            pool.place_tokens(bad)
    for over in (dict(freed_count=i32([0, 0])), dict(freed_pages=i32([[1], [2]]), freed_count=i32([0])), dict(seq_lens_out=i32([0])), dict(next_positions_out=i32([0, 0])),
                 dict(page_table_out=table[:, :4])):
        with pytest.raises(AssertionError):
            pool.place_tokens(i32([1, 1]), **over)
    k, v = (torch.zeros((16, 2, 8, 64), device=DEV) for _ in range(2))
    for over in (dict(frequencies=torch.ones((32,))), dict(frequencies=torch.ones((33,), dtype=torch.float64)), dict(q_weight=torch.ones((64,), device=DEV)),
                 dict(q_weight=torch.ones((32,), device=DEV), k_weight=torch.ones((64,), device=DEV)), dict(v_cache=v.bfloat16())):
        with pytest.raises(AssertionError):
            CacheWriter(**{**dict(q_heads=4, k_cache=k, v_cache=v), **over})
    writer = CacheWriter(q_heads=4, k_cache=k, v_cache=v)
    good = dict(q=torch.zeros((3, 4, 64), device=DEV), k=torch.zeros((3, 2, 64), device=DEV), v=torch.zeros((3, 2, 64), device=DEV), positions=i32([0, 1, 2]),
                slots=torch.arange(3, device=DEV))
    writer.append_tokens(**good)
    for over in (dict(q=good["q"].bfloat16()), dict(k=good["q"]), dict(slots=i32([0, 1, 2])), dict(positions=good["slots"]), dict(v=good["v"][:2]),
                 dict(q=torch.zeros((3, 64, 4), device=DEV).transpose(1, 2)), dict(q_out=torch.zeros((3, 4, 64))), dict(q=torch.zeros((3, 8, 64), device=DEV)[:, ::2])):
        with pytest.raises(AssertionError):
            writer.append_tokens(**{**good, **over})
    args = dict(q_heads=4, k_cache=k, v_cache=v, page_table=table, seq_lens=lens, group_starts=i32([0, 2]), prefix_pages=i32([1]), max_members=2, max_prefix_pages=1)
    for over in (dict(group_starts=i32([0])), dict(members=i32([0])), dict(prefix_pages=torch.ones((1,), device=DEV, dtype=torch.int64)), dict(seq_lens=i32([0]))):
        with pytest.raises(AssertionError):
            PrefixGroups(**{**args, **over})
    groups = PrefixGroups(**args)
    for bad in (torch.zeros((2, 4, 64), device=DEV).bfloat16(), torch.zeros((1, 4, 64), device=DEV), torch.zeros((4, 2, 64), device=DEV).transpose(0, 1)):
        with pytest.raises(AssertionError):
            groups.paged_decode(bad)
    with pytest.raises(RuntimeError):
        PrefixGroups(**{**args, "max_members": 0})
