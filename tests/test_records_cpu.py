"""The calls on 4-bit records, page accounts and eviction without a GPU: refusals, sizes, and the plain 64-bit counterparts themselves."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

from paper_2605_27740_amd import binding
from tests import records_ref as R
from tests.test_boundary_cpu import good_desc

BAD, UNSUPPORTED, WORKSPACE = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED, binding.ERR_WORKSPACE
A, NWS = 0x10000, 1 << 30


@pytest.fixture(scope="module")
def c():
    return binding.load().c


def test_record_bytes(c):
    assert c.unique_page_record_bytes(C.byref(good_desc())) == 8 * (16 * 128 + 2 * 16 * 4)
    assert c.unique_page_record_bytes(C.byref(good_desc(head_dim=64, page_size=8, num_kv_heads=2))) == 2 * 544
    for over in (dict(head_dim=96), dict(page_size=12), dict(num_kv_heads=0)):
        assert c.unique_page_record_bytes(C.byref(good_desc(**over))) == 0
    assert c.unique_page_record_bytes(None) == 0


SHAPES = [(dict(dtype=2), BAD), (dict(batch=0), BAD), (dict(num_q_heads=30), BAD), (dict(head_dim=96), UNSUPPORTED), (dict(page_size=12), UNSUPPORTED),
          (dict(num_q_heads=24), UNSUPPORTED), (dict(page_table=0), BAD), (dict(seq_lens=0), BAD), (dict(max_seq_len_hint=-1), BAD),
          (dict(kv_head_stride=1024), BAD)]


@pytest.mark.parametrize("over,code", SHAPES)
def test_descriptors_are_refused(c, over, code):
    d = C.byref(good_desc(**over))
    n = C.c_size_t()
    assert c.unique_quantise_pages(d, None, None, 0, A, None, 9, None) == code
    assert c.unique_restore_pages(d, None, None, 0, A, None, 9, A, A, None) == code
    assert c.unique_quantised_paged_decode(d, A, A, None, None, 0, 0.0, A, None, A, NWS, None) == code
    assert c.unique_weighted_paged_decode(d, A, 0.0, 1.0, None, A, 64, A, None, A, NWS, None) == code
    assert c.unique_evict_pages(d, 8, 0, 1, A, A, 64, A, A, A, A, 64, A, NWS, None) == code
    if not any(k in over for k in ("page_table", "seq_lens")):  # a size needs no pointers
        assert c.unique_account_workspace_bytes(d, C.byref(n)) == code


def test_quantise_and_restore_refuse(c):
    d = C.byref(good_desc())
    f = c.unique_quantise_pages
    assert f(None, None, None, 0, A, None, 9, None) == BAD
    assert f(C.byref(good_desc(k_cache=0)), None, None, 0, A, None, 9, None) == BAD
    assert f(C.byref(good_desc(v_cache=0)), None, None, 0, A, None, 9, None) == BAD
    assert f(d, None, None, 0, None, None, 9, None) == BAD
    assert f(d, None, None, 0, A + 8, None, 9, None) == BAD
    assert f(d, None, None, 0, A, None, 0, None) == BAD
    assert f(d, A, None, 1, A, None, 9, None) == BAD
    assert f(d, None, A, 1, A, None, 9, None) == BAD
    assert f(d, A, A, -1, A, None, 9, None) == BAD
    g = c.unique_restore_pages
    assert g(None, None, None, 0, A, None, 9, A, A, None) == BAD
    assert g(d, None, None, 0, A, None, 9, None, A, None) == BAD
    assert g(d, None, None, 0, A, None, 9, A, None, None) == BAD
    assert g(d, None, None, 0, A, None, 9, A + 8, A, None) == BAD
    assert g(d, None, None, 0, None, None, 9, A, A, None) == BAD
    assert g(d, None, None, 0, A, None, -1, A, A, None) == BAD
    assert g(d, A, None, 0, A, None, 9, A, A, None) == BAD
    assert binding.load().last_error() != ""


def test_decode_over_records_refuses(c):
    d = C.byref(good_desc(k_cache=0, v_cache=0))
    f = c.unique_quantised_paged_decode
    assert f(None, A, A, None, None, 0, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, None, A, None, None, 0, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, A, None, None, None, 0, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, A, A, None, None, 0, 0.0, None, None, A, NWS, None) == BAD
    assert f(d, A + 8, A, None, None, 0, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, A, A + 4, None, None, 0, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, A, A, A, None, 4, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, A, A, None, A, 4, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, A, A, A, A, 0, 0.0, A, None, A, NWS, None) == BAD
    assert f(d, A, A, None, None, 0, float("nan"), A, None, A, NWS, None) == BAD
    assert f(d, A, A, None, None, 0, 0.0, A, None, None, NWS, None) == WORKSPACE
    assert f(d, A, A, None, None, 0, 0.0, A, None, A + 8, NWS, None) == WORKSPACE
    assert f(d, A, A, None, None, 0, 0.0, A, None, A, 16, None) == WORKSPACE
    assert f(d, A, A, A, A, 4, 0.0, A, None, A, 16, None) == WORKSPACE


def test_workspace_of_the_decode_over_records(c):
    n, old = C.c_size_t(), C.c_size_t()
    f = c.unique_quantised_workspace_bytes
    for over in (dict(), dict(batch=40, max_pages_per_seq=250), dict(batch=1, max_pages_per_seq=9000), dict(dtype=0, batch=64, max_pages_per_seq=300)):
        d = C.byref(good_desc(k_cache=0, v_cache=0, page_table=0, seq_lens=0, **over))
        for k in (0, 1, 64, 700):
            assert f(d, k, C.byref(n)) == 0 and n.value % 256 == 0 and n.value > 0
            few = n.value
        assert f(d, 0, C.byref(old)) == 0 and old.value <= few
    assert f(None, 0, C.byref(n)) == BAD and f(d, -1, C.byref(n)) == BAD and f(d, 0, None) == BAD
    assert f(C.byref(good_desc(head_dim=96)), 0, C.byref(n)) == UNSUPPORTED


def test_weighted_decode_refuses(c):
    d = C.byref(good_desc())
    f = c.unique_weighted_paged_decode
    assert f(C.byref(good_desc(k_cache=0)), A, 0.0, 1.0, None, A, 64, A, None, A, NWS, None) == BAD
    assert f(C.byref(good_desc(v_cache=0)), A, 0.0, 1.0, None, A, 64, A, None, A, NWS, None) == BAD
    assert f(d, None, 0.0, 1.0, None, A, 64, A, None, A, NWS, None) == BAD
    assert f(d, A, 0.0, 1.0, None, None, 64, A, None, A, NWS, None) == BAD
    assert f(d, A, 0.0, 1.0, None, A, 64, None, None, A, NWS, None) == BAD
    assert f(d, A + 4, 0.0, 1.0, None, A, 64, A, None, A, NWS, None) == BAD
    for decay in (-0.1, 1.1, float("nan")):
        assert f(d, A, 0.0, decay, None, A, 64, A, None, A, NWS, None) == BAD
    assert f(d, A, float("nan"), 1.0, None, A, 64, A, None, A, NWS, None) == BAD
    assert f(d, A, 0.0, 1.0, None, A, 63, A, None, A, NWS, None) == BAD
    assert f(d, A, 0.0, 1.0, None, A, 64, A, None, None, NWS, None) == WORKSPACE
    n = C.c_size_t()
    assert c.unique_account_workspace_bytes(d, C.byref(n)) == 0 and n.value % 256 == 0
    assert c.unique_account_workspace_bytes(C.byref(good_desc(k_cache=0, page_table=0, seq_lens=0)), C.byref(n)) == 0
    assert c.unique_account_workspace_bytes(d, None) == BAD and c.unique_account_workspace_bytes(None, C.byref(n)) == BAD
    assert f(d, A, 0.0, 1.0, None, A, 64, A, None, A, 256, None) == WORKSPACE


def test_evict_refuses(c):
    d = C.byref(good_desc(k_cache=0, v_cache=0))
    f = c.unique_evict_pages
    good = [8, 2, 1, A, A, 64, A, A, A, A, 64, A, NWS, None]
    for at in (3, 4, 6, 7, 8, 9):
        assert f(d, *[None if i == at else v for i, v in enumerate(good)]) == BAD
    for budget, sinks, recent in ((8, -1, 1), (8, 0, 0), (8, 5, 4), (0, 0, 1), (2 ** 31 - 1, 2 ** 31 - 1, 1)):
        assert f(d, budget, sinks, recent, *good[3:]) == BAD
    assert f(d, *good[:5], 63, *good[6:]) == BAD                  # weight_stride below the pages
    assert f(d, *good[:10], 55, *good[11:]) == BAD                # 64 - 8 pages may be freed
    assert f(d, 100, *good[1:10], 0, *good[11:]) == BAD
    assert f(d, *good[:11], None, NWS, None) == WORKSPACE
    assert f(d, *good[:11], A + 8, NWS, None) == WORKSPACE
    assert f(d, *good[:12], 256, None) == WORKSPACE


@pytest.mark.parametrize("heads,size", [(1, 1), (16, 16), (32, 32), (3, 0), (12, 0), (64, 0)])
def test_record_bytes_of_the_supported_numbers_of_heads(c, heads, size):
    assert c.unique_page_record_bytes(C.byref(good_desc(num_kv_heads=heads, num_q_heads=heads))) == size * (16 * 128 + 2 * 16 * 4)


def test_host_tensors_are_refused():
    """The Python layer takes device tensors only: nothing reaches the library with a host address."""
    from paper_2605_27740_amd.session import PageAccounts, QuantisedCache
    geo = dict(q_heads=8, kv_heads=2, head_dim=64, page_size=8, dtype=torch.float32, num_pages=4, page_table=torch.zeros((1, 4), dtype=torch.int32),
               seq_lens=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(AssertionError, match="on the GPU"):
        QuantisedCache(**geo)
    with pytest.raises(AssertionError, match="on the GPU"):
        PageAccounts(budget_pages=2, **geo)


def test_the_number_format():
    x = torch.zeros(64)
    x[:16] = torch.tensor([6.0, 5.0, 5.01, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, 0.26, -0.75, -5.0, -3.5, 0.0, -0.2, 7.9])
    code, scale = R.encode(x)
    assert code[:16].tolist() == [7, 6, 7, 6, 4, 4, 2, 2, 0, 1, 10, 14, 14, 0, 8, 7] and scale.tolist() == [127, 1]
    assert R.values(code, scale)[:5].tolist() == [6, 4, 6, 4, 2]
    x[40] = float("inf")
    assert R.encode(x)[1].tolist() == [127, 255]
    assert R.encode(torch.full((32,), 3.0e38))[1].tolist() == [252] and R.encode(torch.full((32,), 1e-44))[1].tolist() == [1]


@pytest.mark.parametrize("S,D", [(8, 64), (16, 128), (32, 64), (32, 128)])
def test_the_layout_is_a_permutation_and_its_own_inverse(S, D):
    at = [R.k_byte(S, D, t, ch) for t in range(S) for ch in range(0, D, 2)] + [R.v_byte(S, D, t, ch) for t in range(S) for ch in range(0, D, 2)]
    assert sorted(at) == list(range(S * D))
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn((2, S, D), generator=g), torch.randn((2, S, D), generator=g)
    tiles = R.tiles_of(k, v)
    one = torch.zeros((R.tile_bytes(S, D),), dtype=torch.uint8)
    for t in range(S):
        (kc, ks), (vc, vs) = R.encode(k[1, t]), R.encode(v[1, t])
        R.write_token(one, S, D, t, kc, ks, vc, vs)
    assert torch.equal(one, tiles[1])
    for x, y in zip(R.values_of(tiles, S, D), (k, v)):
        assert torch.equal(x, R.values(*R.encode(y)))


def test_evict_counterpart():
    table = torch.arange(10).view(1, 10).int()
    w = torch.tensor([[[0.0, 5, 1, 1, 9, 1, 2, 0, 0, 0]]])
    (keep, freed, n), = R.evict(table, torch.tensor([73]), w, 8, 5, 1, 2)   # ten pages, the last of one token
    assert keep == [0, 1, 4, 8, 9] and freed == [2, 3, 5, 6, 7] and n == 73 - 40
    assert R.evict(table, torch.tensor([40]), w, 8, 5, 1, 2) == [(list(range(5)), [], 40)]


# ------------------------------------------------------------------ the layout and the cuts that the library compiles

@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    here = os.path.dirname(os.path.abspath(__file__))
    so = str(tmp_path_factory.mktemp("rules") / "record_rules.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-ftrapv", "-shared", "-fPIC", "-o", so, os.path.join(here, "c_abi", "record_rules.cpp")], check=True)
    return C.CDLL(so)


@pytest.mark.parametrize("S", [8, 16, 32])
@pytest.mark.parametrize("D", [64, 128])
def test_layout_of_the_library(rules, S, D):
    assert rules.tile_bytes(S, D) == R.tile_bytes(S, D) and rules.tile_bytes(S, D) % 16 == 0
    assert [rules.tile_part(S, D, i) for i in range(4)] == [0, S * D // 2, S * D, S * D + S * (D // 32)]
    for t in range(S):
        for u in range(16):
            assert rules.v_at(S, D, t, u) == R.v_byte(S, D, t, u * (D // 16))
    # what a lane of the attention takes at once: D/16 channels of four tokens, consecutive and aligned
    for t in range(0, S, 4):
        for u in range(16):
            at = rules.v_at(S, D, t, u)
            assert at % (D // 8) == 0 and [rules.v_at(S, D, t + i, u) for i in range(4)] == [at + i * (D // 32) for i in range(4)]


def test_cuts_of_batches_of_records(rules):
    """Whatever the lengths: the chunks fit the launch and the launch's partial results, and no sequence with pages is without one."""
    rng = random.Random(5)
    seen = 0
    for _ in range(3000):
        heads, batch, most, page = rng.choice([1, 2, 4, 8, 16, 32]), rng.randint(1, 64), int(2 ** rng.uniform(1, 17)), rng.choice([544, 1088, 2176, 4352])
        if not rules.balances(batch, heads, most, page):
            continue
        seen += 1
        lens = [rng.choice([0, 1, most, rng.randint(0, most), int(most ** rng.random())]) for _ in range(batch)]
        if rng.random() < 0.2:
            lens = [most] * batch
        out, chunks = (C.c_int * 2)(), (C.c_int * batch)()
        rules.cut(batch, heads, most, page, rng.randint(0, 1), (C.c_int * batch)(*lens), out, chunks)
        assert out[1] <= out[0] and out[1] >= 2 * batch * heads
        assert sum(chunks) * heads <= out[0]
        assert all((n > 0) == (k > 0) and k <= max(n, 1) for n, k in zip(lens, chunks))
    assert seen > 500


def test_plans_of_lists_of_records(rules):
    """A plan never needs more partial results than a workspace of unique_workspace_bytes holds, and covers the list."""
    rng = random.Random(6)
    for _ in range(3000):
        batch, heads, length, pages = rng.randint(1, 600), rng.choice([1, 2, 4, 8, 16, 32]), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 15))
        out = (C.c_int * 4)()
        rules.list_plan(batch, heads, length, pages, rng.choice([8, 16, 32]), rng.choice([64, 128]), out)
        assert out[0] * out[1] >= length > out[0] * (out[1] - 1) and out[1] <= out[3] and out[2] <= batch
