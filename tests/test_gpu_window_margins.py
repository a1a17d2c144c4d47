"""GPU: reform_window_attend writes the rows of its sequences and nothing else, whatever the boundaries say."""
import pytest
import torch

import paged_reference as ref
import serving_reference as sref
from paper_2506_01215_amd import binding
from serving_checks import check_attention

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KEPT = 5.0
BF, F = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def clamped(cu, n):
    """[start, rows] of the sequences as the call takes them: boundaries moved into [0, n], a descending pair is empty."""
    cu = [min(max(x, 0), n) for x in cu]
    return [(a, max(b - a, 0)) for a, b in zip(cu, cu[1:])]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (16, 2, 128)])
@pytest.mark.parametrize("cu_q,cu_k", [
    ([0, 40, 20, 20], [0, 40, 60, 100]), ([-5, 50, 50, 60], [90, 10, 200, 100]), ([100, 0, 100, 1 << 30], [0, 100, 0, 100]), ([7, 7, 60, 93], [0, 3, 50, 90]),
    ([-(1 << 31), 30, (1 << 31) - 1], [-(1 << 31), 60, (1 << 31) - 1]), ([3, 50, 80], [20, 30, 30]),
])
def test_only_rows_of_sequences_are_written(hq, hkv, d, cu_q, cu_k, dtype):
    """Outputs inside larger buffers, whose other elements stay; keys outside the sequences are NaN and not looked at."""
    n, window, sinks, margin = 100, 7, 2, 37
    g = torch.Generator().manual_seed(len(cu_q) + d)
    q, k, v = (sref.randn(g, h, n, d, dtype=dtype) for h in (hq, hkv, hkv))
    seqs, keys = clamped(cu_q, n), clamped(cu_k, n)
    nobody = torch.ones(n, dtype=torch.bool)
    for i, m in keys:
        nobody[i:i + m] = False
    k[:, nobody], v[:, nobody] = float("nan"), float("nan")
    room = torch.full((hq + 2, n + 2 * margin, d), KEPT, dtype=dtype, device=DEV)
    lse_room = torch.full((hq * n + 2 * margin,), KEPT, device=DEV)
    out, lse = room[1:-1, margin:-margin], lse_room[margin:-margin].view(hq, n)
    print(f"[window margins] {hq}/{hkv} d={d} {dtype} cu_q={cu_q} cu_k={cu_k}", flush=True)
    binding.reform_window_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(cu_q), d ** -0.5, window, n_sink=sinks, cu_k=i32(cu_k), out=out, lse=lse)
    written = torch.zeros(n, dtype=torch.bool)
    for (i, m), (j, m_k) in zip(seqs, keys):
        assert not bool(written[i:i + m].any())                          # the sets above give a row to one sequence
        written[i:i + m] = True
        if m == 0:
            continue
        want, want_lse, a, err = ref.window_attend(q[:, i:i + m], k[:, j:j + m_k], v[:, j:j + m_k], [m], [m_k], d ** -0.5, window, sinks)
        check_attention(out[:, i:i + m], lse[:, i:i + m], want, want_lse, a, err, max(m_k, 1), dtype)
    assert bool((out.cpu()[:, ~written] == KEPT).all()) and bool((lse.cpu()[:, ~written] == KEPT).all())
    room[1:-1, margin:-margin] = KEPT
    assert bool((room == KEPT).all()) and bool((lse_room[:margin] == KEPT).all()) and bool((lse_room[-margin:] == KEPT).all())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (8, 2, 128)])
def test_no_workspace_is_needed(hq, hkv, d, dtype):
    """Few rows behind many keys, whose keys reform_prompt_attend shares out and wants room for: the query gives 0, what is passed is not
    looked at, and a window of all keys gives that call's results up to rounding."""
    nq, nk = 3, 3000
    g = torch.Generator().manual_seed(d)
    q, k, v = (sref.randn(g, h, n, d, dtype=dtype) for h, n in ((hq, nq), (hkv, nk), (hkv, nk)))
    dev = [x.to(DEV) for x in (q, k, v)]
    cu_q, cu_k = i32([0, nq]), i32([0, nk])
    desc = binding.window_desc(*dev, torch.empty_like(dev[0]), cu_q, d ** -0.5, nk)
    prompt = binding.prompt_desc(*dev, torch.empty_like(dev[0]), cu_q, d ** -0.5)
    assert binding.window_workspace_bytes(desc) == 0 and binding.prompt_workspace_bytes(prompt) > 0
    want, want_lse, a, err = ref.window_attend(q, k, v, [nq], [nk], d ** -0.5, nk, 0)
    for ws in (None, torch.empty(1, dtype=torch.uint8, device=DEV)):
        out, lse = binding.reform_window_attend(*dev, cu_q, d ** -0.5, nk, cu_k=cu_k, workspace=ws)
        check_attention(out, lse, want, want_lse, a, err, nk, dtype)
    out, lse = binding.reform_prompt_attend(*dev, cu_q, d ** -0.5, cu_k=cu_k)
    check_attention(out, lse, want, want_lse, a, err, nk, dtype)
