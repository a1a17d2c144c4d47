"""Outputs of the calls on sliding windows and on caches in pages that have bytes in common with an input or with another output are
refused on the host (no GPU is needed: no call here gets past its checks)."""
import ctypes

import pytest

from paper_2506_01215_amd import binding
from test_paged_abi import evict, lib, paged, window

MB = 1 << 20
ROOM = 1 << 40                                           # of the workspace, which is never touched


def call(name, desc, at, ws=900 * MB):
    return getattr(lib(), f"reform_{name}")(ctypes.byref(desc), *at, ws, ROOM, None)


def places(names, **moved):
    """Addresses 16 MB apart, further than any of the tensors reaches."""
    at = {n: (i + 1) * 16 * MB for i, n in enumerate(names)}
    at.update({n: (at[x] if isinstance(x, str) else at[x[0]] + x[1]) for n, x in moved.items()})
    return [at[n] for n in names]


WINDOW = ["q", "k", "v", "cu_q", "cu_k", "out", "lse"]               # q, out: 8 heads x 100 rows x 256 bytes, k, v: 2 of them


@pytest.mark.parametrize("name,where", [
    ("out", ("q", 256)), ("out", ("q", 204544)), ("out", ("q", -204544)), ("out", ("k", 51184)), ("out", ("v", -16)), ("out", ("cu_q", -1024)),
    ("out", ("cu_k", 0)), ("lse", ("q", 8)), ("lse", ("q", -3196)), ("lse", ("k", 51196)), ("lse", ("cu_q", 8)), ("lse", ("cu_k", -3196)),
    ("lse", ("out", 204796)), ("lse", ("out", 4)),
])
def test_window_outputs(name, where):
    assert call("window_attend", window(), places(WINDOW, **{name: where})) == 1


PAGED = ["q", "k", "v", "table", "lens", "score", "out", "lse"]


@pytest.mark.parametrize("name,where", [
    ("out", ("q", 16)), ("out", ("q", 6128)), ("out", ("q", -6128)), ("out", ("k", 500 * 8192 - 16)), ("out", ("v", 8192)), ("out", ("table", 4784)),
    ("out", ("lens", 0)), ("lse", ("q", 6140)), ("lse", ("out", 6140)), ("lse", ("score", 4)), ("lse", ("score", 4 * (12800 * 2 + 6400 * 2) - 4)),
    ("lse", ("table", 4796)), ("lse", ("lens", 8)), ("lse", ("v", 4)), ("score", ("lse", 92)), ("score", ("lse", -4)), ("score", ("q", 6140)), ("score", ("out", -25600)),
    ("score", ("k", 4)), ("score", ("table", -4)), ("score", ("lens", -4)),
])
def test_paged_outputs(name, where):
    assert call("paged_attend", paged(want_score=1), places(PAGED, **{name: where})) == 1


EVICT = ["k", "v", "score", "pos", "table", "lens", "kept", "new_len"]


@pytest.mark.parametrize("name,where", [
    ("v", ("k", 4096)), ("v", ("k", 256)), ("score", ("k", 4)), ("score", ("v", 500 * 8192 - 4)), ("pos", ("score", 4)), ("pos", ("score", 4 * 6396)),
    ("pos", ("v", 0)), ("kept", ("score", 4)), ("kept", ("pos", -4)), ("kept", ("lens", -4)), ("kept", ("table", 4)), ("kept", ("k", 16)),
    ("new_len", ("lens", 8)), ("new_len", ("lens", -8)), ("new_len", ("kept", 3 * 2 * 4096 * 4 - 4)), ("new_len", ("score", 400)), ("new_len", ("table", 4)),
])
def test_evict_outputs(name, where):
    assert call("paged_evict", evict(), places(EVICT, **{name: where})) == 1


def test_a_missing_workspace_comes_first():
    """As a program sees it that asks for the size last."""
    d = paged(want_score=1)
    at = places(PAGED, out=("q", 16))
    assert lib().reform_paged_attend(ctypes.byref(d), *at, None, 0, None) == 3
    assert binding.paged_workspace_bytes(d) > 0
