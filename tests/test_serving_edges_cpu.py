"""Arithmetic of the calls around the cache near the ends of its types, without a GPU."""
import ctypes as C
import os
import random
import subprocess

import pytest
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("rules") / "place_rules.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-ftrapv", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "c_abi", "place_rules.cpp")], check=True)
    lib = C.CDLL(so)
    lib.stack_place.argtypes = [C.c_int, C.c_longlong, C.c_int]
    return lib


def test_places_on_a_stack_of_any_size(places):
    """Stacks of up to 2^31 - 1 entries, as many evicted pages and as many of ended sequences: what does not fit is lost, and no place lies in front of the stack. (Sums in 32
    bits would wrap.) An overflow ends the process."""
    r = random.Random(1)
    some = lambda most: r.choice([0, 1, most // 2, most - 1, most, r.randrange(most + 1)])  # noqa: E731
    for _ in range(20_000):
        capacity = r.choice([1, 7, 1 << 20, 1 << 30, MOST - 3, MOST, r.randrange(1, MOST + 1)])
        size, freed_all, own_before, mine = min(some(MOST), capacity), some(MOST), some(MOST), some(MOST)
        at = places.stack_place(size, freed_all + own_before, capacity)
        assert at == min(size + freed_all + own_before, capacity)
        for i in {0, 1, max(mine - 1, 0), mine, max(capacity - at - 1, 0), capacity - at}:
            assert bool(places.stack_has(at, i, capacity)) == (size + freed_all + own_before + i < capacity)


def test_shapes_that_are_meant_to_share_their_prefixes_do(tmp_path_factory):
    """What the GPU tests of shared prefixes in large pools ask for is not served by every member reading for itself, and the bounds pass what is read past the caches."""
    from tests import test_serving_paths_gpu as P
    so = str(tmp_path_factory.mktemp("rules") / "prefix_rules.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-ftrapv", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "c_abi", "prefix_rules.cpp")], check=True)
    rules, out = C.CDLL(so), (C.c_int * 3)()
    seen = set()
    for dtype, H, Hkv, D, S, members in P.SHARED:
        elem = torch.finfo(dtype).bits // 8
        for B in (members, members + 2):
            columns, page = P.columns_of(B, dtype, Hkv, D, S), S * D * 2 * elem
            for prefix in (1000 // S, 40):
                rules.prefix_alone(B, Hkv, H // Hkv, elem, S, page, columns, prefix, columns, out)
                assert out[0] == 0 and columns * B * page * Hkv > P.STREAM
        seen.add((elem, D, members * (H // Hkv) > 64))
    assert {(2, 128, False), (2, 128, True), (2, 64, False), (2, 64, True), (4, 128, False), (4, 64, True)} <= seen
    with open(os.path.join(HERE, "..", "paper_2605_27740_amd", "csrc", "kernels.hpp")) as f:
        assert "kStreamNtBytes = 96ll << 20" in f.read()
