"""GPU: scores of reform_paged_attend where the heads of a KV group have logits far from one another's, as models whose keys have a
bias have: no head's reference may meet another head's logits."""
import random

import pytest
import torch

import paged_reference as ref
import serving_reference as sref
from paper_2506_01215_amd import binding
from test_gpu_paged_attend import BF, DEV, F, check_score, i32

pytestmark = pytest.mark.gpu


def shifted(g, S, hq, hkv, pages, page_len, d, dtype, shifts):
    """q, k, v: the logits of head r of each group lie shifts[r] higher by element 0, which all keys have alike."""
    q, k, v = sref.randn(g, S, hq, d), sref.randn(g, pages, hkv, page_len, d), sref.randn(g, pages, hkv, page_len, d, dtype=dtype)
    k[..., 0] = 8.0
    q[..., 0] = torch.tensor(shifts * hkv) / 8.0 / d ** -0.5
    return q.to(dtype), k.to(dtype), v


def run_shifted(shifts, hkv, lens, dtype, accumulate, d=64, page_len=16, window=0, sinks=0):
    G, S = len(shifts), len(lens)
    g = torch.Generator().manual_seed(G + d)
    table, pages = ref.make_table(random.Random(G), lens, page_len)
    q, k, v = shifted(g, S, hkv * G, hkv, pages, page_len, d, dtype, shifts)
    print(f"[paged heads] {hkv * G}/{hkv} d={d} {dtype} lens={lens} window={window}/{sinks} added={accumulate}", flush=True)
    before = torch.rand(S, hkv, len(table[0]) * page_len, generator=g)
    score = before.to(DEV)
    out, lse = binding.reform_paged_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(table), i32(lens), d ** -0.5, window=window, n_sink=sinks,
                                           score=score, accumulate=accumulate)
    want, want_lse, a, err, scores = ref.paged_attend(q, k, v, table, lens, d ** -0.5, window, sinks)
    for b in range(S):
        ref.check_single(out[b], lse[b], want[b], want_lse[b], a[b], err[b], max(1, lens[b]), dtype, f"sequence {b}")
    check_score(score, before, scores, lens, G, accumulate)


def patterns(G):
    """The last head above and below the others, the first one, and every second one."""
    for at in ({G - 1}, {0}, set(range(1, G, 2))):
        for x in (150.0, -150.0):
            yield [x if r in at else 0.0 for r in range(G)]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("G", [1, 2, 3, 5, 6, 66])
def test_heads_far_apart_over_shared_out_caches(G, accumulate, dtype):
    """Caches in pieces of several workgroups, others that one finishes, one that sees nothing."""
    hkv = 1 if G > 16 else 2
    for shifts in patterns(G):
        run_shifted(shifts, hkv, [1700, 40, 0, 1100, 7] if G > 16 else [5000, 40, 0, 1200, 7], dtype, accumulate)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("G", [2, 3, 66])
def test_heads_far_apart_over_whole_caches_and_windows(G, accumulate, dtype):
    hkv = 1 if G > 16 else 2
    for shifts in patterns(G):
        run_shifted(shifts, hkv, [170, 40, 0, 7], dtype, accumulate)                                     # one workgroup to a cache
        run_shifted(shifts, hkv, [3000, 40, 2999], dtype, accumulate, d=128, page_len=20, window=1500, sinks=33)


@pytest.mark.parametrize("dtype", [BF, F])
def test_scores_of_heads_far_apart_can_be_evicted_by(dtype):
    """What is added up over tokens stays finite, and the eviction keeps the keys that the 64-bit scores would keep."""
    lens, page_len, budget = [2600, 1900], 16, 1000
    g = torch.Generator().manual_seed(4)
    table, pages = ref.make_table(random.Random(4), lens, page_len)
    q, k, v = shifted(g, 2, 4, 2, pages, page_len, 64, dtype, [0.0, 150.0])
    dev_k, dev_v, dev_table, dev_lens = k.to(DEV), v.to(DEV), i32(table), i32(lens)
    score = torch.zeros(2, 2, len(table[0]) * page_len, device=DEV)
    for _ in range(3):
        binding.reform_paged_attend(q.to(DEV), dev_k, dev_v, dev_table, dev_lens, 0.125, score=score, accumulate=True)
    held = score.cpu()
    assert bool(torch.isfinite(held).all())
    kept = torch.zeros(2, 2, budget, dtype=torch.int32, device=DEV)
    binding.reform_paged_evict(dev_k, dev_v, score, dev_table, dev_lens, budget, n_sink=4, n_recent=16, kept_idx=kept)
    for b, n in enumerate(lens):
        for h in range(2):
            assert kept[b, h].tolist() == ref.evict(held[b, h], n, budget, 4, 16)
