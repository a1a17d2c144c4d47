"""Which batches of packed prompts have their keys shared out (prompt_share_rows, asked before the form of prompt_choose), replayed on
the CPU from the kernels' own header and compared with the workspace that the library asks for."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

import test_gpu_prompt_attend
from paper_2506_01215_amd import binding
from test_prompt_plan import load_plan

UNITS = torch.cuda.get_device_properties(0).multi_processor_count if torch.cuda.is_available() else 256
MOST_SHARES = 512


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return load_plan(tmp_path_factory)


@pytest.fixture(scope="module")
def share(tmp_path_factory):
    here = os.path.dirname(os.path.abspath(__file__))
    lib = str(tmp_path_factory.mktemp("prompt_share") / "replay.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-static-libubsan", "-shared", "-fPIC", "-I", os.path.join(here, "..", "paper_2506_01215_amd", "csrc"),
                    os.path.join(here, "prompt_share_replay.cpp"), "-o", lib], check=True)
    replay = ctypes.CDLL(lib)

    def rows(d, G, Hkv, n_seq, n_q, n_k, units=UNITS):
        """Rows of a block (0: not shared out), keys of a tile, groups of waves, least keys of a share, shares of a compute unit."""
        out = [ctypes.c_int() for _ in range(4)]
        return (replay.plan_share(d, G, Hkv, n_seq, n_q, n_k, units, *map(ctypes.byref, out)), *(x.value for x in out))

    return rows


def workspace(d, G, Hkv, n_seq, n_q, n_k, dtype=1):
    desc = binding.PromptDesc(struct_size=ctypes.sizeof(binding.PromptDesc), dtype=dtype, n_q_heads=G * Hkv, n_kv_heads=Hkv, head_dim=d,
                              n_seq=n_seq, n_q_rows=n_q, n_k_rows=n_k, scale=0.1, reserved=0, q_head_stride=d, q_row_stride=G * Hkv * d,
                              k_head_stride=d, k_row_stride=Hkv * d, v_head_stride=d, v_row_stride=Hkv * d, o_head_stride=d,
                              o_row_stride=G * Hkv * d)
    return binding.prompt_workspace_bytes(desc)


def any_sizes(rnd, most_rows=30):
    return (rnd.choice([64, 128]), rnd.choice([1, 3, 8, 64]), rnd.choice([1, 2, 8, 128]), rnd.choice([1, rnd.randint(2, 64), rnd.randint(1, 65536)]),
            int(2 ** rnd.uniform(0, rnd.choice([6, most_rows]))) or 1, int(2 ** rnd.uniform(0, 30)) - 1)


@pytest.mark.parametrize("args,rows", [
    # a row or a few behind many keys, as measured (prompt_plan.h): a block's own chain would take longer
    ((64, 2, 1, 1, 1, 3001), 16), ((128, 1, 8, 8, 75, 24075), 16), ((128, 4, 1, 1, 3, 16003), 16),
    ((128, 4, 8, 4, 64, 32064), 128),      # of several sequences the longest is taken to have 1.3 times the mean: 21 rows of 4 heads, 84
    # rows enough to fill the chip, short keys, more sequences than a wave has lanes
    ((128, 7, 8, 8, 364, 128364), 0), ((128, 4, 8, 1, 16384, 16384), 0), ((64, 3, 8, 7, 900, 900), 0), ((128, 4, 1, 65, 65, 300000), 0),
])
def test_batches_that_are_shared_out(share, args, rows):
    assert share(*args)[0] == rows


def test_any_sizes(share):
    """The whole range of arguments: no overflow, no division by nothing, a block that there is a kernel for, and places (tile by
    tile, 8 more for each item) that 32 bits hold even where broken boundaries give all rows and keys to each of 64 sequences."""
    rnd = random.Random(2)
    seen = set()
    for _ in range(6000):
        args = any_sizes(rnd)
        d, G, Hkv, n_seq, n_q, n_k = args
        rows, keys, groups, least, workgroups = share(*args, rnd.choice([1, 32, 256, 304]))
        seen.add(rows)
        assert rows in (0, 16, 32, 64, 128)
        if rows:
            assert n_seq <= 64 and keys == (32 if rows <= 32 else 64) and least >= keys and workgroups in (1, 2) and groups in (1, 2, 4, 8)
            assert 64 * -(-n_q * G // rows) * Hkv * (-(-n_k // keys) + 8) < 1 << 31
    assert seen == {0, 16, 32, 64, 128}


def test_the_library_asks_for_that_workspace(share):
    rnd = random.Random(3)
    shared = 0
    for _ in range(1500):
        args = any_sizes(rnd, 14)
        d, G, Hkv, n_seq, n_q, n_k = args
        if n_q * G * Hkv / 16 + Hkv * n_seq > 8388607 or Hkv * n_k >= 1 << 30 or max(G, 1) * Hkv * d >= 1 << 24:
            continue
        rows, _, _, _, workgroups = share(*args)
        want = 2 * min(workgroups * UNITS, MOST_SHARES) * min(rows, n_q * G) * (4 * d + 8) if rows else 0
        assert workspace(*args) == want, args
        shared += rows > 0
    assert shared > 100


def test_fp32_places_stay_within_32_bits():
    rnd = random.Random(4)
    shared = 0
    for _ in range(3000):
        d = rnd.choice([4, 32, 64, 96, 256])
        _, G, Hkv, n_seq, n_q, n_k = any_sizes(rnd, 20)
        if n_q * G * Hkv / 16 + Hkv * n_seq > 8388607 or Hkv * n_k >= 1 << 30:
            continue
        if workspace(d, G, Hkv, n_seq, n_q, n_k, dtype=0):
            shared += 1
            assert n_seq <= 64 and 64 * -(-n_q * G // 16) * Hkv * (-(-n_k // 16) + 8) < 1 << 31
    assert shared > 100


def test_the_tests_of_whole_forms_are_of_whole_forms(share, plan):
    """The batches by which the GPU tests cover the forms of prompt_choose are not shared out, with keys in front or without, and every
    form is among them."""
    cases = next(m for m in test_gpu_prompt_attend.test_every_form.pytestmark if m.name == "parametrize").args[1]
    forms = set()
    for d, hq, hkv, n, total, form in cases:
        forms.add((d, *form))
        for front in (0, 37):
            args = (d, hq // hkv, hkv, n, total, total + front * n)
            if front and (total > 9000 or plan(*args) != form):
                continue
            assert share(*args)[0] == 0 and workspace(*args) == 0, args
    assert forms == {(64, 256, 1), (64, 128, 1), (64, 32, 4), (64, 16, 8), (128, 128, 1), (128, 128, 2), (128, 32, 4), (128, 16, 8)}
