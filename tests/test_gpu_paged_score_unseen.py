"""GPU: scores of reform_paged_attend beside keys that are not finite: what is not seen gets 0, or keeps what it has, all the same."""
import math
import random

import pytest
import torch

import paged_reference as ref
import serving_reference as sref
from paper_2506_01215_amd import binding
from test_gpu_paged_attend import BF, DEV, F, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("lens,page_len", [([200, 150], 16), ([200, 150], 10), ([4000, 2500], 16), ([4000, 2500], 10)])
@pytest.mark.parametrize("hq", [4, 40])
def test_keys_that_are_not_seen_beside_ones_that_are_not_finite(hq, lens, page_len, accumulate, dtype):
    """A window and first keys that end inside a tile, a page that is not there, and NaN and infinity in keys that are seen."""
    hkv, d, window, sinks = 2, 64, 50 if lens[0] < 1000 else 1500, 3
    table, pages = ref.make_table(random.Random(1), lens, page_len)
    gone = (lens[0] - 30) // page_len
    table[0][gone] = -1
    g = torch.Generator().manual_seed(8)
    k, v = (sref.randn(g, pages, hkv, page_len, d, dtype=dtype) for _ in range(2))
    q = sref.randn(g, 2, hq, d, dtype=dtype).to(DEV)
    before = torch.rand(2, hkv, len(table[0]) * page_len, generator=g).to(DEV)

    def call():
        score = before.clone()
        binding.reform_paged_attend(q, k.to(DEV), v.to(DEV), i32(table), i32(lens), 0.125, window=window, n_sink=sinks, score=score, accumulate=accumulate)
        return score

    clean = call()
    for j, x in ((lens[0] - 1, math.nan), (lens[0] - 2, math.inf)):
        k[table[0][j // page_len], 1, j % page_len] = x
    got = call()
    assert torch.equal(got[1], clean[1]) and torch.equal(got[0, 0], clean[0, 0])
    j = torch.arange(lens[0])
    seen = ((j >= lens[0] - window) | (j < sinks)) & (j // page_len != gone)
    seen = seen.to(DEV)
    assert torch.equal(got[0, 1, :lens[0]][~seen], before[0, 1, :lens[0]][~seen] if accumulate else torch.zeros(int((~seen).sum()), device=DEV))
    assert bool(torch.isnan(got[0, 1, :lens[0]][seen]).all())
    assert torch.equal(got[0, 1, lens[0]:], before[0, 1, lens[0]:])
