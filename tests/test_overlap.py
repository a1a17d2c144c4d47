"""Whether strided tensors have a byte in common, replayed on the CPU from the calls' own header (overlap.h), against the sets of
their bytes."""
import ctypes
import itertools
import os
import random
import subprocess

import pytest


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    here = os.path.dirname(os.path.abspath(__file__))
    lib = str(tmp_path_factory.mktemp("overlap") / "replay.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-static-libubsan", "-shared", "-fPIC", "-I", os.path.join(here, "..", "paper_2506_01215_amd", "csrc"),
                    os.path.join(here, "overlap_replay.cpp"), "-o", lib], check=True)
    replay = ctypes.CDLL(lib)

    def pack(at, size, extent, walks):
        walks = list(walks) + [(1, 0)] * (3 - len(walks))
        return (ctypes.c_int64 * 9)(at, size, extent, *itertools.chain(*walks))

    class Calls:
        meet = staticmethod(lambda a, b: bool(replay.overlap_meet(pack(*a), pack(*b))))
        empty = staticmethod(lambda a: bool(replay.overlap_empty(pack(*a))))
    return Calls


def covered(at, size, extent, walks):
    starts = {at}
    for n, step in walks:
        starts = {s + i * step * size for s in starts for i in range(n)}
    return {s + i for s in starts for i in range(extent * size)}


def test_as_the_sets_of_bytes(overlap):
    rnd = random.Random(1)
    found = 0
    for _ in range(6000):
        areas = []
        for _ in range(2):
            size, extent = rnd.choice([1, 2, 4]), rnd.randint(1, 5)
            walks = [(rnd.randint(1, 4), rnd.choice([0, 1, 3, 4, 6, 12, 24, 25, 48, rnd.randint(0, 60)])) for _ in range(rnd.randint(0, 3))]
            areas.append((1000 + rnd.randint(0, 120), size, extent, walks))
        want = bool(covered(*areas[0]) & covered(*areas[1]))
        found += want
        assert overlap.meet(*areas) == want and overlap.meet(*areas[::-1]) == want, areas
    assert 1000 < found < 5000


def test_parts_of_one_buffer(overlap):
    """As attention's tensors lie in one buffer: side by side in every row, halves of a pool's pages, and one element too far."""
    S, hq, hkv, d = 65536, 32, 8, 128
    row = (hq + 2 * hkv) * d
    q, k = (1 << 20, 2, d, [(S, row), (hq, d)]), ((1 << 20) + hq * d * 2, 2, d, [(S, row), (hkv, d)])
    assert not overlap.meet(q, k)
    assert overlap.meet((q[0], 2, d + 1, q[3]), k)
    pages, page_len = 100000, 16
    half = hkv * page_len * d
    a, b = ((x, 2, d, [(pages, 2 * half), (hkv, page_len * d), (page_len, d)]) for x in (1 << 20, (1 << 20) + 2 * half))
    assert not overlap.meet(a, b) and overlap.meet(a, a)
    assert overlap.meet(a, ((1 << 20) + 2 * half - 16, *b[1:])) and overlap.meet(a, (b[0] + 2 * half - 2, *b[1:]))
    inside = (1 << 20) + 4 * half * 777 + 2 * half                       # between page 777's rows and the next page's
    assert not overlap.meet(a, (inside, 2, half, [])) and overlap.meet(a, (inside, 2, half + 1, [])) and overlap.meet(a, (inside - 2, 2, half, []))


def test_nothing_and_the_ends_of_addresses(overlap):
    a = (4096, 2, 64, [(3, 64)])
    for nothing in ((0, 2, 64, []), (4096, 2, 0, []), (4096, 2, 64, [(0, 64)]), (4096, 4, 64, [(2, 1 << 61)]), (4096, 4, 64, [(1 << 31, 1 << 40)])):
        assert overlap.empty(nothing) and not overlap.meet(a, nothing)
    assert overlap.meet(a, (4096 + 383, 1, 1, [])) and not overlap.meet(a, (4096 + 384, 1, 1, [])) and not overlap.meet(a, (4095, 1, 1, []))
    assert overlap.meet(a, (4096, 4, 1, [(1, 1 << 61)]))                 # a step that is never taken


def test_a_search_ends(overlap):
    """Thousands of pieces between one another with different steps: some answer, soon."""
    a, b = (1 << 20, 1, 1, [(1 << 22, 6), (2, 1)]), ((1 << 20) + 2, 1, 1, [(1 << 22, 9)])
    for _ in range(100):
        overlap.meet(a, b)
