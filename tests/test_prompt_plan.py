"""The choice of the packed prompts' form, replayed on the CPU from the kernels' own header (prompt_plan.h)."""
import ctypes
import os
import random
import subprocess

import pytest


def load_plan(tmp_path_factory):
    here = os.path.dirname(os.path.abspath(__file__))
    lib = str(tmp_path_factory.mktemp("prompt_plan") / "replay.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-static-libubsan", "-shared", "-fPIC", "-I", os.path.join(here, "..", "paper_2506_01215_amd", "csrc"),
                    os.path.join(here, "prompt_plan_replay.cpp"), "-o", lib], check=True)
    replay = ctypes.CDLL(lib)

    def form(d, G, Hkv, n_seq, n_q, n_k, units=256):
        rows, groups = ctypes.c_int(), ctypes.c_int()
        replay.plan_form(d, G, Hkv, n_seq, n_q, n_k, units, ctypes.byref(rows), ctypes.byref(groups))
        return rows.value, groups.value

    replay.plan_estimate.restype = ctypes.c_double
    form.estimate = replay.plan_estimate
    return form


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return load_plan(tmp_path_factory)


@pytest.mark.parametrize("args,form", [
    # measured fastest, by more than a tenth: see the header
    ((64, 2, 4, 32, 14586, 30586), (128, 1)), ((64, 3, 1, 4, 2445, 2445), (32, 4)), ((64, 2, 1, 1, 1, 3001), (16, 8)),
    ((64, 4, 8, 50, 3131, 3131), (128, 1)), ((64, 8, 1, 1, 1541, 1641), (32, 4)), ((64, 1, 8, 1, 16384, 16384), (256, 1)),
    ((128, 7, 8, 50, 2859, 2859), (128, 1)), ((128, 8, 1, 1, 6673, 6673), (128, 2)), ((128, 1, 4, 1, 2674, 2674), (32, 4)),
    ((128, 1, 8, 8, 75, 24075), (16, 8)), ((128, 1, 1, 1, 10071, 10071), (32, 4)), ((128, 4, 1, 1, 425, 925), (16, 8)),
])
def test_measured_batches_take_their_form(plan, args, form):
    assert plan(*args) == form


def test_any_sizes_have_a_form(plan):
    """The whole range of arguments: no overflow, no division by nothing, a form that exists for the head_dim."""
    rnd = random.Random(1)
    for _ in range(3000):
        d = rnd.choice([64, 128])
        n_q = int(2 ** rnd.uniform(0, 30)) - 1 or 1
        args = (d, rnd.choice([1, 3, 8, 64]), rnd.choice([1, 2, 8, 128]), rnd.randint(1, 65536), n_q, int(2 ** rnd.uniform(0, 30)) - 1)
        assert plan(*args, rnd.choice([1, 32, 256, 304])) in {64: [(256, 1), (128, 1), (32, 4), (16, 8)], 128: [(128, 1), (128, 2), (32, 4), (16, 8)]}[d]
        for i in range(4):
            t = plan.estimate(i, *args, 256)
            assert 0 < t < 1e18
