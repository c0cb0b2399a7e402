"""The calls around the cache without a GPU: refusals, sizes, frequencies, and the plain counterparts themselves."""
import ctypes as C
import math
import os
import random
import subprocess

import pytest
import torch

from paper_2605_27740_amd import binding
from paper_2605_27740_amd.session import rotary_frequencies
from tests import serving_ref as R
from tests.test_boundary_cpu import good_desc

BAD, UNSUPPORTED, WORKSPACE = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE
A, NWS = 0x10000, 1 << 30


@pytest.fixture(scope="module")
def c():
    return binding.load().c


def placement(**over):
    f = {name: A for name, kind in binding.Placement._fields_ if kind is C.c_void_p}
    f.update(freed_stride=4, free_capacity=9, max_new_tokens=7)
    f.update(over)
    return binding.Placement(**f)


def groups(**over):
    f = dict(starts=A, members=A, prefix_pages=A, num_groups=1, max_members=2, max_prefix_pages=3, max_own_pages=4)
    f.update(over)
    return binding.PrefixGroupsDesc(**f)


def transform(**over):
    f = dict(q_weight=A, k_weight=A, frequencies=A, eps=1e-6, magnitude=1.0, rotary_dim=64, interleaved=0)
    f.update(over)
    return binding.HeadTransform(**f)


SHAPES = [(dict(dtype=2), BAD), (dict(batch=0), BAD), (dict(num_q_heads=30), BAD), (dict(head_dim=96), UNSUPPORTED), (dict(page_size=12), UNSUPPORTED),
          (dict(num_q_heads=24), UNSUPPORTED), (dict(max_seq_len_hint=-1), BAD), (dict(kv_head_stride=1024), BAD)]


@pytest.mark.parametrize("over,code", SHAPES)
def test_descriptors_are_refused(c, over, code):
    d, n = C.byref(good_desc(**over)), C.c_size_t()
    assert c.unique_place_tokens(d, placement(), A, NWS, None) == code
    assert c.unique_place_workspace_bytes(d, 7, C.byref(n)) == code
    assert c.unique_append_tokens(d, 3, A, 4096, A, 1024, A, 1024, A, A, transform(), A, None) == code
    assert c.unique_shared_prefix_decode(d, groups(), A, 0.0, A, None, A, NWS, None) == code
    assert c.unique_shared_prefix_workspace_bytes(d, groups(), C.byref(n)) == code


def test_place_refuses(c):
    f, d = c.unique_place_tokens, C.byref(good_desc())
    n = C.c_size_t()
    assert f(None, placement(), A, NWS, None) == BAD
    assert f(d, None, A, NWS, None) == BAD
    for name in ("new_tokens", "free_pages", "free_count", "free_count_out", "page_table_out", "seq_lens_out", "placed", "token_starts", "positions", "slots",
                 "next_positions", "next_positions_out", "freed_pages", "freed_count"):
        assert f(d, placement(**{name: 0}), A, NWS, None) == BAD, name
    for over in (dict(page_table=0), dict(seq_lens=0)):
        assert f(C.byref(good_desc(**over)), placement(), A, NWS, None) == BAD
    for over in (dict(freed_stride=0), dict(free_capacity=0), dict(max_new_tokens=-1), dict(max_new_tokens=(1 << 24) + 1)):
        assert f(d, placement(**over), A, NWS, None) == BAD, over
    assert f(C.byref(good_desc(batch=1 << 12)), placement(freed_stride=1 << 20), A, NWS, None) == UNSUPPORTED
    assert f(d, placement(), None, NWS, None) == WORKSPACE
    assert f(d, placement(), A + 8, NWS, None) == WORKSPACE
    assert f(d, placement(max_new_tokens=100_000), A, 64, None) == WORKSPACE
    assert c.unique_place_workspace_bytes(d, 7, None) == BAD
    assert c.unique_place_workspace_bytes(None, 7, C.byref(n)) == BAD
    assert c.unique_place_workspace_bytes(d, -1, C.byref(n)) == BAD
    assert c.unique_place_workspace_bytes(C.byref(good_desc(page_table=0, seq_lens=0, k_cache=0)), 100_000, C.byref(n)) == 0
    assert n.value % 256 == 0 and n.value >= 256


def test_append_refuses(c):
    f = c.unique_append_tokens
    good = dict(desc=good_desc(), rows=3, q=A, qs=4096, k=A, ks=1024, v=A, vs=1024, positions=A, slots=A, how=transform(), out=A + (1 << 20))

    def call(**over):
        x = dict(good, **over)
        d = None if x["desc"] is None else C.byref(x["desc"])
        return f(d, x["rows"], x["q"], x["qs"], x["k"], x["ks"], x["v"], x["vs"], x["positions"], x["slots"], x["how"], x["out"], None)

    for name in ("desc", "q", "k", "v", "positions", "slots", "out"):
        assert call(**{name: None}) == BAD, name
    for name in ("q", "k", "v", "out"):
        assert call(**{name: A + 8}) == BAD, name
    for over in (dict(rows=-1), dict(qs=4088), dict(ks=1023), dict(vs=1028), dict(qs=4100), dict(out=A, qs=8192), dict(desc=good_desc(k_cache=0)),
                 dict(desc=good_desc(v_cache=0))):
        assert call(**over) == BAD, over
    for over in (dict(q_weight=0), dict(k_weight=0), dict(q_weight=A + 4), dict(rotary_dim=-16), dict(rotary_dim=24), dict(rotary_dim=144), dict(frequencies=0),
                 dict(frequencies=A + 4), dict(eps=-1.0), dict(eps=math.nan), dict(magnitude=math.nan)):
        assert call(how=transform(**over)) == BAD, over
    assert call(rows=0, q=None, out=None) == 0  # nothing to do


def test_prefix_refuses(c):
    f, d = c.unique_shared_prefix_decode, C.byref(good_desc())
    n = C.c_size_t()
    assert f(None, groups(), A, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, None, A, 0.0, A, None, A, NWS, None) == BAD
    for over in (dict(starts=0), dict(prefix_pages=0), dict(num_groups=0), dict(num_groups=good_desc().batch + 1), dict(max_members=0),
                 dict(max_prefix_pages=-1), dict(max_own_pages=-1)):
        assert f(d, groups(**over), A, 0.0, A, None, A, NWS, None) == BAD, over
    for over in (dict(k_cache=0), dict(v_cache=0), dict(page_table=0), dict(seq_lens=0)):
        assert f(C.byref(good_desc(**over)), groups(), A, 0.0, A, None, A, NWS, None) == BAD, over
    assert f(d, groups(), None, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, groups(), A, 0.0, None, None, A, NWS, None) == BAD
    assert f(d, groups(), A + 2, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, groups(), A, math.nan, A, None, A, NWS, None) == BAD
    assert f(d, groups(), A, 0.0, A, None, None, NWS, None) == WORKSPACE
    assert f(d, groups(), A, 0.0, A, None, A, 1, None) == WORKSPACE
    # bounds by which there would be 2^31 rows of partial results and more
    wide = good_desc(batch=65535, max_pages_per_seq=1 << 20)
    assert f(C.byref(wide), groups(num_groups=65535, max_members=65535, max_prefix_pages=1 << 20), A, 0.0, A, None, A, 1 << 62, None) == UNSUPPORTED
    assert c.unique_shared_prefix_workspace_bytes(C.byref(wide), groups(num_groups=65535, max_members=65535, max_prefix_pages=1 << 20), C.byref(n)) == UNSUPPORTED
    assert c.unique_shared_prefix_workspace_bytes(C.byref(wide), groups(num_groups=65535, max_members=2, max_prefix_pages=100), C.byref(n)) == 0
    assert c.unique_shared_prefix_workspace_bytes(d, groups(), None) == BAD
    assert c.unique_shared_prefix_workspace_bytes(C.byref(good_desc(page_table=0, seq_lens=0, k_cache=0)), groups(starts=0, prefix_pages=0, members=0),
                                                  C.byref(n)) == 0 and n.value > 0


def test_frequencies():
    f = rotary_frequencies(64, base=1e4)
    assert f.dtype is torch.float64 and f.shape == (32,) and f[0] == 1.0
    assert torch.allclose(f, torch.tensor([1e4 ** (-i / 32) for i in range(32)], dtype=torch.float64), rtol=1e-15)
    assert torch.equal(rotary_frequencies(64, base=1e4, factor=4.0), f / 4)
    g = rotary_frequencies(64, base=1e4, factor=4.0, trained_len=4096, low_turns=1.0, high_turns=32.0)
    for a, b in zip(f.tolist(), g.tolist()):
        turns = 4096 * a / (2 * math.pi)
        share = min(1.0, max(0.0, (turns - 1) / 31))
        assert math.isclose(b, a * share + a / 4 * (1 - share), rel_tol=1e-14)
    assert rotary_frequencies(0).numel() == 0


def test_plain_heads_against_complex_numbers():
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn((5, 3, 64), generator=g), torch.randn((64,), generator=g)
    pos, f = torch.arange(5) * 1000, rotary_frequencies(32)
    for interleaved in (False, True):
        y, _ = R.heads(x, w, 1e-3, pos, f, 1.5, interleaved)
        for r in range(5):
            for h in range(3):
                z = x[r, h].double()
                z = z / math.sqrt(float((z * z).sum()) / 64 + 1e-3) * w.double()
                for i in range(16):
                    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + 16)
                    c = complex(z[a], z[b]) * 1.5 * complex(math.cos(float(pos[r] * f[i])), math.sin(float(pos[r] * f[i])))
                    assert abs(c - complex(y[r, h, a], y[r, h, b])) < 1e-12
                assert torch.equal(y[r, h, 32:], z[32:])


def test_plain_places_keep_every_page():
    """No page is lost or given twice, a slot is in its sequence's page, and places follow one another."""
    for seed in range(200):
        r = random.Random(seed)
        S, B, width = r.choice([8, 16]), r.randrange(1, 9), 6
        lens = [r.randrange(width * S + 1) for _ in range(B)]
        new = [r.choice([-1, 0, 1, r.randrange(40)]) for _ in range(B)]
        pages = [-(-n // S) for n in lens]
        ids = list(range(sum(pages) + r.randrange(10)))
        r.shuffle(ids)
        take = iter(ids)
        table = [[next(take) for _ in range(p)] + [-1] * (width - p) for p in pages]
        free = list(take)
        got = R.place(S, table, lens, new, free + [-1] * sum(pages), len(free), 60)
        held = [p for b in range(B) for p in got["table"][b] if p >= 0]
        assert sorted(held + got["stack"]) == sorted(ids)
        for b in range(B):
            assert sum(p >= 0 for p in got["table"][b]) == -(-got["seq_lens"][b] // S)
            assert got["seq_lens"][b] == (0 if new[b] < 0 else lens[b] + got["placed"][b])
            rows = range(got["token_starts"][b], got["token_starts"][b] + got["placed"][b])
            for i, row in enumerate(rows):
                at = lens[b] + i
                assert got["slots"][row] == got["table"][b][at // S] * S + at % S and got["positions"][row] == at


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("rules") / "prefix_rules.so")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-ftrapv", "-shared", "-fPIC", "-o", so, os.path.join(here, "c_abi", "prefix_rules.cpp")], check=True)
    return C.CDLL(so)


def prefix_items(rules, kv_heads, group, elem, S, sizes, prefix, own, max_members, max_prefix, max_own, batch):
    """Sources of a batch as the kernels see them, cut -> shape, sources and their (count, pages each, blocks)."""
    src = [(p if n > 1 else 0, n * group, 0) for n, p in zip(sizes, prefix)]
    at = 0
    for n, p in zip(sizes, prefix):
        src += [(own[at + i] + (p if n == 1 else 0), group, 1) for i in range(n)]
        at += n
    n = len(src)
    arr = [(C.c_int * n)(*col) for col in zip(*src)]
    shape, outs = (C.c_int * 8)(), [(C.c_int * n)() for _ in range(3)]
    assert rules.prefix_items(batch, kv_heads, group, elem, S, len(sizes), max_members, max_prefix, max_own, n, *arr, shape, *outs) == 0
    return dict(zip("rows tile wanted max_items max_rows plans slots most".split(), shape)), src, list(zip(*outs))


def test_prefix_items_fit_their_arrays(rules):
    """Whatever true bounds the host knows: items cover every page once, whole tiles but the last, page ids fit the registers, and items and rows of
    partial results are no more than the workspace has."""
    for seed in range(3000):
        r = random.Random(seed)
        S, group, kv, elem = r.choice([8, 16, 32]), r.choice([1, 2, 4, 8]), r.choice([1, 2, 8, 32]), r.choice([2, 4])
        n = r.choice([1, 1, 2, 5, 40])
        longest, alone = r.choice([0, 1, 30, 3000, 70_000]), r.choice([0, 1, 20, 5000])
        sizes = [r.choice([0, 1, 1, 2, r.randrange(200)]) for _ in range(n)]
        sizes[0] = max(sizes[0], 1)
        prefix = [r.choice([0, longest, r.randrange(longest + 1)]) for _ in sizes]
        own = [r.choice([0, alone, r.randrange(alone + 1)]) for _ in range(sum(sizes))]
        slack = r.choice([0, 0, 3])
        batch = max(sum(sizes), n) + slack
        shape, src, cuts = prefix_items(rules, kv, group, elem, S, sizes, prefix, own, max(sizes) + slack, max(prefix) + slack, max(own) + slack, batch)
        items = rows = 0
        for (pages, live, mine), (count, each, blocks) in zip(src, cuts):
            assert count * each >= pages and (count - 1) * each < max(pages, 1), "every page, no item without pages"
            assert each % shape["tile"] == 0 or count <= 1
            assert mine or count == 0 or each <= shape["most"]
            items += count * blocks
            rows += count * blocks * (group if mine else shape["rows"])
        assert items <= shape["max_items"] and rows <= shape["max_rows"], seed
        if shape["plans"]:
            assert len(src) < 256 and len(sizes) + batch < 256 and shape["max_items"] * kv <= 2 * shape["slots"]


def test_prefix_items_fill_the_chip(rules):
    """Where there is much to read, items are about as many as run at a time."""
    for kv, group, n, pages, own in ((8, 4, 16, 8192, 60), (8, 4, 256, 2048, 20), (8, 8, 10, 1500, 180), (1, 8, 4, 100_000, 10)):
        shape, src, cuts = prefix_items(rules, kv, group, 2, 16, [n], [pages], [own] * n, n, pages, own, n)
        assert shape["slots"] * 7 // 8 <= shape["wanted"] * kv <= shape["slots"]
        assert 0.5 * shape["wanted"] <= sum(n * b for n, _, b in cuts) <= shape["max_items"]


def test_prefix_members_for_themselves(rules):
    """Where there is little to read: chunks cover the most pages that a member may have, every one has some, and they are no more than launches and arrays are made for."""
    out = (C.c_int * 3)()
    for seed in range(3000):
        r = random.Random(seed)
        batch, kv, group, elem, S, D = r.choice([1, 2, 9, 64, 4096]), r.choice([1, 2, 8, 32]), r.choice([1, 4, 8]), r.choice([2, 4]), r.choice([8, 16, 32]), r.choice([64, 128])
        width, prefix, own = r.choice([1, 40, 300, 5000, 1 << 22]), r.choice([0, 1, 30, 400, 10_000]), r.choice([0, 1, 50, 5000])
        page = S * D * 2 * elem
        rules.prefix_alone(batch, kv, group, elem, S, page, width, prefix, own, out)
        chunks, pages, rows = out
        most = max(min(width, prefix + own), 1)
        one = 2 * most * S <= 3 * (128 if elem == 4 else 512)
        assert (chunks > 0) == (most * batch * kv * page <= (256 if one else 160 if elem == 4 else 64) << 20) and (chunks <= 1 or not one), seed
        if chunks:
            assert chunks * pages >= most > (chunks - 1) * pages and rows == batch * chunks * group
            assert chunks == 1 or (chunks * batch * kv <= 1024 and pages * S >= (64 if elem == 4 else 256))
