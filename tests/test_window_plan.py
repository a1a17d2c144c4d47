"""The choice of the form that window prompts take, replayed on the CPU from the kernels' own header (window_plan.h)."""
import ctypes
import os
import random
import subprocess

import pytest


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    here = os.path.dirname(os.path.abspath(__file__))
    lib = str(tmp_path_factory.mktemp("window_plan") / "replay.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
                    "-static-libubsan", "-shared", "-fPIC", "-I", os.path.join(here, "..", "paper_2506_01215_amd", "csrc"),
                    os.path.join(here, "window_plan_replay.cpp"), "-o", lib], check=True)
    replay = ctypes.CDLL(lib)

    def form(d, G, Hkv, n_seq, n_q, n_k, window, n_sink, units=256):
        rows, groups = ctypes.c_int(), ctypes.c_int()
        replay.plan_form(d, G, Hkv, n_seq, n_q, n_k, window, n_sink, units, ctypes.byref(rows), ctypes.byref(groups))
        return rows.value, groups.value

    replay.plan_estimate.restype = ctypes.c_double
    form.estimate = replay.plan_estimate
    return form


FORMS = {64: [(128, 1), (32, 4), (16, 8)], 128: [(128, 1), (128, 2), (32, 4), (16, 8)]}


@pytest.mark.parametrize("args,form", [
    # measured fastest, by more than a tenth
    ((64, 7, 2, 2, 525, 525, 2, 4), (32, 4)), ((64, 8, 1, 20, 356, 356, 187, 1), (16, 8)), ((128, 3, 8, 4, 157, 157, 157, 1), (16, 8)),
    ((128, 1, 4, 1, 925, 925, 32, 4), (16, 8)), ((128, 1, 1, 1, 10000, 10000, 4000, 0), (32, 4)),
])
def test_measured_batches_take_their_form(plan, args, form):
    assert plan(*args) == form


def test_every_form_is_taken_by_a_tested_size(plan):
    """Sizes of test_gpu_window_attend.py."""
    sizes = [(64, 4, 8, 1, 1200, 1200, 300, 0), (64, 8, 2, 1, 900, 900, 511, 65), (64, 4, 2, 1, 100, 100, 7, 2), (128, 4, 2, 1, 2100, 2100, 300, 100),
             (128, 4, 8, 1, 700, 700, 200, 256), (128, 2, 1, 1, 6164, 6164, 12, 64), (128, 8, 2, 3, 1800, 1800, 833, 5), (128, 8, 2, 4, 266, 266, 8, 64),
             (128, 4, 2, 1, 60, 60, 33, 5)]
    for d in (64, 128):
        assert {plan(*s) for s in sizes if s[0] == d} == set(FORMS[d])


def test_any_sizes_have_a_form(plan):
    """The whole range of arguments: no overflow, no division by nothing, a form that exists for the head_dim."""
    rnd = random.Random(1)
    for _ in range(3000):
        d = rnd.choice([64, 128])
        n_q, n_k = int(2 ** rnd.uniform(0, 27)) - 1 or 1, int(2 ** rnd.uniform(0, 30)) - 1
        window, sinks = min(int(2 ** rnd.uniform(0, 31)), max(n_k, 1)), min(int(2 ** rnd.uniform(0, 31)) - 1, n_k)
        args = (d, rnd.choice([1, 3, 8, 64]), rnd.choice([1, 2, 8, 128]), rnd.randint(1, 65536), n_q, n_k, window, sinks)
        assert plan(*args, rnd.choice([1, 32, 256, 304])) in FORMS[d]
        for i in range(len(FORMS[d])):
            assert 0 < plan.estimate(i, *args, 256) < 1e18


def test_a_wider_window_takes_longer(plan):
    for d in (64, 128):
        for form in range(len(FORMS[d])):
            times = [plan.estimate(form, d, 4, 8, 5, 8000, 9000, w, 16, 256) for w in (1, 64, 500, 2000, 9000)]
            assert times == sorted(times)
