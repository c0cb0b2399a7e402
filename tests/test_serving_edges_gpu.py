"""Values of placement, append and attention over shared prefixes where they can go wrong: terms that cancel, sums near their type's end, values that are not finite."""
import math

import pytest
import torch

from paper_2605_27740_amd.session import CacheWriter, PagePool, rotary_frequencies
from tests import serving_ref as R
from tests import test_serving_gpu as G

pytestmark = pytest.mark.gpu
DEV, DTYPES, i32, say = G.DEV, G.DTYPES, G.i32, G.say


# ------------------------------------------------------------------ shared prefixes

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,H,Hkv,S,members", [(128, 8, 1, 16, 3), (128, 8, 1, 16, 20), (64, 8, 2, 8, 5), (64, 8, 1, 32, 40), (128, 2, 2, 32, 50)])
def test_prefix_terms_that_cancel(gpu_lib, dtype, D, H, Hkv, S, members):
    """Two tokens of opposite values whose weights are within some 2^-12 of each other, all others' weights 0: out = v tanh(d / 2) with the difference d of the logits.
    A weight is off by 2^-20 of itself (its argument, below 16, by 2^-21 twice, the exponential by 2^-23), the sums of two by 2^-24, so out by
    2^-19 of |v| and its rounding. Probabilities of 8 bits would be equal and leave 0."""
    say(f"cancel {dtype} {(D, H, Hkv, S)} members={members}")
    pages = 200 // S
    c = G.prefix_case(dtype, H, Hkv, D, S, [([0] * members, pages)], seed=members, poison=False)
    g = torch.Generator().manual_seed(D + S)
    ids = c["table"][c["members"][0].long(), :pages].long()
    pool = c["k"].shape[0]
    half = torch.finfo(dtype).eps / 2
    for i, j in ((0, 1), (3, 30), (7, 40), (33, 70), (66, 190), (150, 199 // S * S - 1)):
        k = torch.zeros((pool, Hkv, S, D))
        k[..., 0] = -2.0 ** 14
        v = torch.randn((pool, Hkv, S, D), generator=g)
        q = torch.zeros((members, H, D))
        q[..., 0] = torch.tensor([1.0, 0.5, 2.0, 1.0])[torch.arange(members * H).view(members, H) % 4]
        value = torch.randn((Hkv, D), generator=g).to(dtype).float()
        for t, logit, sign in ((i, 0.0, -1.0), (j, 2.0 ** -8, 1.0)):
            k[ids[t // S], :, t % S, 0] = logit
            v[ids[t // S], :, t % S] = sign * value
        x = dict(c, q=q.to(dtype), k=k.to(dtype), v=v.to(dtype))
        d = q[..., 0].double() * 2.0 ** -8 / math.sqrt(D)
        of = value.double().repeat_interleave(H // Hkv, 0)
        want = of * torch.tanh(d / 2)[..., None]
        for wide in (True, False):
            out = G.make_groups(x, H, wide=wide).paged_decode(x["q"].to(DEV))[0].cpu().double()
            tol = 2.0 ** -19 * of.abs() * (1 + half) + half * want.abs()
            assert ((out - want).abs() <= tol).all(), (i, j, wide, float(((out - want).abs() / tol).max()))


# ------------------------------------------------------------------ places

@pytest.mark.parametrize("B,rows", [(50, 100), (50, 9000), (1100, 100)])
def test_a_stack_of_2_31_entries(gpu_lib, B, rows):
    """Pages that come back to a nearly full stack whose capacity is the largest there is: those that do not fit are lost, and nothing is written in front of the stack. One launch, two, three."""
    say(f"stack of 2^31 - 1 entries, B={B} rows={rows}")
    most, window, guard = 2 ** 31 - 1, 60, 1024
    c, total = G.place_case(B, B, 8, 30, 200, 1, 0.0, ended=0.7, evicted=3)
    c.update(free=list(range(total, total + window)), free_count=window - 5, rows=rows)
    c["new"] = [min(t, 1) for t in c["new"]]
    want = R.place(**c)
    buf = torch.empty((guard + most,), dtype=torch.int32, device=DEV)
    buf[:guard] = -5
    stack = buf[guard:]
    stack[most - window:] = i32(c["free"])
    table, lens, nxt, count = i32(c["table"]), i32(c["lens"]), i32(c["nxt"]), i32([most - 5])
    pool = PagePool(q_heads=8, kv_heads=8, head_dim=64, page_size=8, dtype=torch.float32, num_pages=total + window, page_table=table, seq_lens=lens, max_new_tokens=rows,
                    free_pages=stack, free_count=count, shared_pages=i32(c["shared"]), next_positions=nxt)
    pool.place_tokens(i32(c["new"]), i32(c["freed"]), i32(c["freed_count"]))
    torch.cuda.synchronize()
    assert (buf[:guard] == -5).all()
    assert table.tolist() == want["table"] and lens.tolist() == want["seq_lens"] and pool.slots.tolist() == want["slots"] and pool.placed.tolist() == want["placed"]
    assert stack[most - window:int(count)].tolist() == want["stack"]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,rows", [(40, 300), (40, 9000), (1100, 9000)])
def test_sequences_without_a_place_stay_as_they_are(gpu_lib, B, rows, in_place):
    """Also those whose length is more than their row holds, or none: theirs was cut to the row's."""
    say(f"stay {B} {rows} {in_place}")
    c, total = G.place_case(B, B, 16, 6, 90, 5, 1.0, ended=0.1, evicted=1)
    lens = list(c["lens"])
    for b, n in ((3, 97), (8, 5000), (17, 2 ** 31 - 1), (21, -4), (30, -2 ** 31)):
        lens[b], c["new"][b] = n, 0 if b in (8, 21, 30) else 2
    c["lens"] = [n if 0 <= n <= 96 else 0 for n in lens]
    c["new"] = [0 if not 0 <= n <= 96 else t for n, t in zip(lens, c["new"])]
    new = [2 if n > 96 and b != 8 else t for b, (n, t) in enumerate(zip(lens, c["new"]))]
    c["rows"] = rows
    table, lens_in, nxt, count = i32(c["table"]), i32(lens), i32(c["nxt"]), i32([c["free_count"]])
    pool = PagePool(q_heads=8, kv_heads=8, head_dim=64, page_size=16, dtype=torch.float32, num_pages=total, page_table=table, seq_lens=lens_in, max_new_tokens=rows,
                    free_pages=i32(c["free"]), free_count=count, shared_pages=i32(c["shared"]), next_positions=nxt)
    outs = {} if in_place else dict(seq_lens_out=torch.full_like(lens_in, -9), next_positions_out=torch.full_like(nxt, -9))
    pool.place_tokens(i32(new), i32(c["freed"]), i32(c["freed_count"]), **outs)
    torch.cuda.synchronize()
    want = R.place(**c)
    got = (lens_in if in_place else outs["seq_lens_out"]).tolist()
    assert got == [n if not 0 <= n <= 96 else w for n, w in zip(lens, want["seq_lens"])]
    assert (nxt if in_place else outs["next_positions_out"]).tolist() == want["next"]
    assert pool.placed.tolist() == want["placed"] and table.tolist() == want["table"] and pool.free_pages[:int(count)].tolist() == want["stack"]


# ------------------------------------------------------------------ queries, keys and values

@pytest.mark.parametrize("D,interleaved", [(128, False), (128, True), (64, False), (64, True)])
@pytest.mark.parametrize("magnitude", [1.0, 1.25])
def test_sine_and_cosine_are_rounded_once(gpu_lib, D, interleaved, magnitude):
    """fp32 heads whose pairs are (1, 0) come out as m (cos a, sin a): half a step from 64 bits. The angle of a position below 2^20 is off by three roundings in 64 bits, 2^-31
    of a radian, and the reference's by one, 2^-33."""
    rows, g = 4000, torch.Generator().manual_seed(D)
    x = torch.zeros((rows, 4, D))
    lo, hi = (slice(0, D, 2), slice(1, D, 2)) if interleaved else (slice(0, D // 2), slice(D // 2, D))
    x[..., lo] = 1.0
    positions = torch.randint(0, 1 << 20, (rows,), generator=g).int()
    positions[:64] = torch.arange(64)
    kc, vc = (torch.zeros((rows // 16, 2, 16, D), device=DEV) for _ in range(2))
    f = rotary_frequencies(D, base=5e5)
    writer = CacheWriter(q_heads=4, k_cache=kc, v_cache=vc, frequencies=f, magnitude=magnitude, interleaved=interleaved)
    q = writer.append_tokens(x.to(DEV), x[:, :2].contiguous().to(DEV), x[:, :2].contiguous().to(DEV), positions.to(DEV), torch.arange(rows, device=DEV))
    torch.cuda.synchronize()
    a = (positions.double()[:, None] * f)[:, None]
    for got in (q.cpu(), kc.cpu().transpose(1, 2).reshape(rows, 2, D)):
        for part, want in ((lo, magnitude * torch.cos(a)), (hi, magnitude * torch.sin(a))):
            off = (got[..., part].double() - want).abs()
            assert (off <= 2.0 ** -24 * want.abs() + magnitude * 2.0 ** -30.5).all(), float((off - 2.0 ** -24 * want.abs()).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,H,Hkv,S", [(128, 8, 2, 16), (64, 8, 1, 8), (128, 4, 4, 32), (64, 2, 2, 16)])
@pytest.mark.parametrize("members", [2, 5, 45])
def test_prefix_values_that_are_not_finite_are_their_own_members(gpu_lib, dtype, D, H, Hkv, S, members):
    """Infinities and NaN among the values of a prefix: members that are shorter get their results as ever, the others have no finite number in those channels, and theirs in all
    other channels. Members end before the prefix does, in its first pages, at a page's end, or are empty; a page in the middle is missing in one case."""
    say(f"not finite {dtype} {(D, H, Hkv, S)} members={members}")
    pages = 1200 // S
    N = pages * S
    lens = [N + 9, N - 700, 0, N, 1, N - 64, N - 65, S, N - 300, 130]
    own = [lens[i % 10] - N - (i // 10 if i % 10 > 3 and lens[i % 10] > 9 else 0) for i in range(members)]
    for seed, hole in ((1, False), (2, True)):
        c = G.prefix_case(dtype, H, Hkv, D, S, [(own, pages), ([3], 1)], seed=seed + members)
        row = c["table"][c["members"][0].long(), :pages].long()
        if hole:
            c["table"][c["members"][:members].long(), 30] = -1
        bad = [(0, 5, math.nan), (64, 7, math.inf), (129, 8, -math.inf), (130, D - 1, math.inf), (131, D - 2, math.nan), (N - 701, 0, math.nan), (N - 700, 33, math.nan),
               (N - 300, 34, -math.inf), (N - 66, 1, math.nan), (N - 40, 2, math.inf), (N - 1, 3, math.nan)]
        if seed == 2:
            bad = bad[-5:]
        clean = dict(c, v=c["v"].clone())
        lost = torch.zeros((len(c["lens"]), H, D), dtype=torch.bool)
        for at, channel, x in bad:
            kv = at % Hkv
            c["v"][row[at // S], kv, at % S, channel] = x
            clean["v"][row[at // S], kv, at % S, channel] = 0.0
            heads = torch.arange(kv * (H // Hkv), (kv + 1) * (H // Hkv))
            if at // S != 30 or not hole:
                for b in c["members"][:members].tolist():
                    if c["lens"][b] > at:
                        lost[b, heads, channel] = True
        want = R.attend(clean["q"], clean["k"], clean["v"], clean["table"], clean["lens"])
        tol, tol_lse = G.prefix_bounds(clean, want, dtype)
        some = c["lens"] > 0
        for wide in (True, False):
            out, lse = (x.cpu() for x in G.make_groups(c, H, wide=wide).paged_decode(c["q"].to(DEV)))
            fine = ((out.double() - want[0]).abs() <= tol) | ~some[:, None, None]
            assert (fine | lost).all(), (seed, wide, (~(fine | lost)).nonzero()[:5].tolist())
            assert not out[lost].isfinite().any(), (seed, wide)
            assert ((lse.double() - want[1]).abs() <= tol_lse)[some].all()
            assert (out[~some] == 0).all() and torch.isneginf(lse[~some]).all()
