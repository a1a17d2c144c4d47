"""GPU: tensors that lie between one another in one buffer, without a byte in common, are taken as they are: the same bits as apart."""
import random

import pytest
import torch

import paged_reference as ref
import serving_reference as sref
from paper_2506_01215_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", [BF, F])
def test_window_output_beside_its_inputs(dtype):
    """[rows][q, k, v and output heads][elements], and head by head."""
    n, hq, hkv, d = 131, 6, 2, 64
    g = torch.Generator().manual_seed(1)
    x = sref.randn(g, n, 2 * hq + 2 * hkv, d, dtype=dtype).to(DEV)
    cu = i32([0, 40, n])
    for rows in (x, x.transpose(0, 1).contiguous().transpose(0, 1)):
        q, k, v, out = rows.transpose(0, 1).split([hq, hkv, hkv, hq])
        want, want_lse = binding.reform_window_attend(q.clone(), k.clone(), v.clone(), cu, 0.125, 17, n_sink=3)
        got, lse = binding.reform_window_attend(q, k, v, cu, 0.125, 17, n_sink=3, out=out)
        assert torch.equal(got, want) and torch.equal(lse, want_lse) and got.data_ptr() == out.data_ptr()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("layout", ["pages [2][heads][rows]", "rows [2][heads]", "elements [2]"])
def test_paged_caches_in_one_pool(layout, dtype):
    """K and V in one pool, q beside out, scores beside positions, old lengths beside new ones, through a token and an eviction."""
    S, hq, hkv, d, page_len, lens, budget = 3, 8, 2, 64, 16, [300, 40, 170], 100
    rnd, g = random.Random(2), torch.Generator().manual_seed(2)
    table, pages = ref.make_table(rnd, lens, page_len)
    cap = len(table[0]) * page_len
    kv = [sref.randn(g, pages, hkv, page_len, d, dtype=dtype).to(DEV) for _ in range(2)]
    if layout.startswith("pages"):
        pool = torch.stack(kv, 1)
        k, v = pool[:, 0], pool[:, 1]
    elif layout.startswith("rows"):
        pool = torch.stack(kv).permute(1, 3, 0, 2, 4).contiguous()
        k, v = pool[:, :, 0].transpose(1, 2), pool[:, :, 1].transpose(1, 2)
    else:
        pool = torch.cat(kv, -1)
        k, v = pool[..., :d], pool[..., d:]
    table = i32(table)
    both = sref.randn(g, S, 2 * hq, d, dtype=dtype).to(DEV)
    q, out = both[:, :hq], both[:, hq:]
    words = torch.zeros(S, hkv, 2, cap, device=DEV)
    score, pos = words[:, :, 0], words.view(torch.int32)[:, :, 1]
    pos.copy_(torch.arange(cap, device=DEV))
    length = i32([lens, [0] * S])

    apart = dict(k=kv[0], v=kv[1], score=torch.zeros(S, hkv, cap, device=DEV), pos=pos.contiguous())
    want = binding.reform_paged_attend(q.clone(), apart["k"], apart["v"], table, i32(lens), 0.125, score=apart["score"])
    got = binding.reform_paged_attend(q, k, v, table, length[0], 0.125, score=score, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(score, apart["score"])
    want = binding.reform_paged_evict(apart["k"], apart["v"], apart["score"], table, i32(lens), budget, n_sink=2, n_recent=10, pos=apart["pos"])
    got = binding.reform_paged_evict(k, v, score, table, length[0], budget, n_sink=2, n_recent=10, pos=pos, new_len=length[1])
    assert torch.equal(got, want) and length.tolist() == [lens, [min(n, budget) for n in lens]]
    for x, y in ((k, apart["k"]), (v, apart["v"]), (score, apart["score"]), (pos, apart["pos"])):
        assert torch.equal(x, y)
