"""GPU: the calls on sliding windows and on caches in pages where elements lie further than 2^31 from a tensor's first one: the result
has to be that of the same call on dense tensors, bit for bit (strides choose no form).  And a cache so long that its last rows
do, with keys of zeros, whose result is known."""
import random

import pytest
import torch

import paged_reference as ref
import serving_reference as sref
from paper_2506_01215_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
FAR = 1 << 31


@pytest.fixture(autouse=True)
def give_back():
    """Some 10 to 30 GB a test: not kept for the tests that follow."""
    yield
    torch.cuda.empty_cache()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def apart(x, step):
    """x [n, ...] on the GPU, its first dimension's entries `step` elements apart, what lies between never initialised."""
    n, inner = x.shape[0], x[0].numel()
    assert step >= inner and step % 16 == 0 and (n - 1) * step > FAR
    rest = x[0].contiguous().stride()
    view = torch.empty((n - 1) * step + inner, dtype=x.dtype, device=DEV).as_strided(x.shape, (step, *rest))
    for i in range(n):
        view[i].copy_(x[i])
    return view


def far_step(n):
    return -(-FAR // (n - 3) // 16) * 16 + 16


@pytest.mark.parametrize("dtype,d,page_len,lens", [(BF, 128, 16, [500, 90]), (BF, 64, 20, [333, 700]), (F, 64, 16, [300, 150]), (BF, 128, 64, [9000, 20])])
@pytest.mark.parametrize("window", [0, 100])
def test_tokens_over_far_pages(dtype, d, page_len, lens, window):
    g = torch.Generator().manual_seed(1)
    table, pages = ref.make_table(random.Random(1), lens, page_len)
    k, v = (sref.randn(g, pages, 2, page_len, d, dtype=dtype).to(DEV) for _ in range(2))
    q = sref.randn(g, len(lens), 8, d, dtype=dtype).to(DEV)
    cols = len(table[0]) * page_len
    score = torch.rand(len(lens) * 2, cols, device=DEV)
    want_score = score.view(len(lens), 2, cols).clone()
    want = binding.reform_paged_attend(q, k, v, i32(table), i32(lens), 0.1, window=window, n_sink=5, score=want_score, accumulate=True)
    far_score = torch.empty(3 * (1 << 30) + cols, device=DEV).as_strided((len(lens), 2, cols), (2 << 30, 1 << 30, 1))
    far_score.copy_(score.view(len(lens), 2, cols))
    step = far_step(pages)
    got = binding.reform_paged_attend(q, apart(k, step), apart(v, step), i32(table), i32(lens), 0.1, window=window, n_sink=5, score=far_score, accumulate=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(far_score, want_score)


@pytest.mark.parametrize("dtype,d,page_len,lens,budget", [(BF, 128, 16, [500, 90], 300), (F, 64, 20, [333, 301], 300), (BF, 64, 64, [4300], 4096)])
def test_evictions_in_far_pages(dtype, d, page_len, lens, budget):
    g = torch.Generator().manual_seed(2)
    table, pages = ref.make_table(random.Random(2), lens, page_len)
    k, v = (sref.randn(g, pages, 2, page_len, d, dtype=dtype).to(DEV) for _ in range(2))
    cols = len(table[0]) * page_len
    score, pos = torch.rand(len(lens), 2, cols, device=DEV), torch.randint(0, 1 << 30, (len(lens), 2, cols), device=DEV, dtype=torch.int32)
    strides = (2 << 30, 1 << 30, 1)
    far = [torch.empty((2 * len(lens) - 1) * (1 << 30) + cols, dtype=x.dtype, device=DEV).as_strided(x.shape, strides) for x in (score, pos)]
    for x, y in zip(far, (score, pos)):
        x.copy_(y)
    step = far_step(pages)
    fk, fv = apart(k, step), apart(v, step)
    binding.reform_paged_evict(k, v, score, i32(table), i32(lens), budget, n_sink=4, n_recent=20, pos=pos)
    binding.reform_paged_evict(fk, fv, far[0], i32(table), i32(lens), budget, n_sink=4, n_recent=20, pos=far[1])
    for x, y in ((fk, k), (fv, v), (far[0], score), (far[1], pos)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("hq,hkv,d,lens,window,sinks,dtype", [(32, 8, 64, [300], 100, 10, BF), (16, 2, 64, [300], 200, 0, BF), (8, 2, 64, [150], 7, 2, BF),
                                                              (8, 2, 128, [600], 300, 100, BF), (16, 2, 128, [70, 66, 65, 65], 8, 64, BF),
                                                              (8, 2, 128, [150], 33, 5, BF), (16, 2, 128, [700, 600, 500], 833, 5, BF), (4, 2, 64, [200], 50, 5, F)])
def test_windows_over_far_rows(hq, hkv, d, lens, window, sinks, dtype):
    g = torch.Generator().manual_seed(3)
    n = sum(lens)
    cu = i32([sum(lens[:i]) for i in range(len(lens) + 1)])
    x = [sref.randn(g, n, h, d, dtype=dtype).to(DEV) for h in (hq, hkv, hkv)]
    want = binding.reform_window_attend(*(t.transpose(0, 1) for t in x), cu, 0.1, window, n_sink=sinks)
    step = far_step(n)
    assert step < 1 << 24
    out = apart(torch.zeros_like(x[0]), step).transpose(0, 1)
    got = binding.reform_window_attend(*(apart(t, step).transpose(0, 1) for t in x), cu, 0.1, window, n_sink=sinks, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_cache_beyond_32_bits():
    """2^25 + 64 keys of 64 elements: all alike, so every weight is 1 / n, and sums of them are exact in 32 bits."""
    n, d, page_len = (1 << 25) + 64, 64, 4096
    pages = -(-n // page_len)
    k = torch.zeros(pages, 1, page_len, d, dtype=BF, device=DEV)
    v = torch.zeros_like(k)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(4)).to(DEV)
    for j, x in ((0, 1.0), (n // 2, 2.0), (n - 1, 4.0)):
        v[order[j // page_len], 0, j % page_len, j % d] = x * 2.0 ** 25
    v[order[n // page_len], 0, n % page_len:] = float("nan")             # behind the last key
    q = torch.randn(1, 2, d, device=DEV).to(BF)
    score = torch.zeros(1, 1, pages * page_len, device=DEV)
    out, lse = binding.reform_paged_attend(q, k, v, order.int()[None], i32([n]), 0.125, score=score)
    want = torch.zeros(d, dtype=torch.float64)
    for j, x in ((0, 1.0), (n // 2, 2.0), (n - 1, 4.0)):
        want[j % d] += x * 2.0 ** 25 / n
    assert bool(((out[0].cpu().double() - want).abs() <= (2.0 ** -8 + 8 * sref.U24) * want).all())
    assert bool(((lse.cpu().double() - torch.tensor(float(n)).double().log()).abs() <= 20 * 4 * sref.U24).all())
    assert bool(((score[0, 0, :n].double() * n / 2 - 1).abs() <= 8 * sref.U24).all()) and bool((score[0, 0, n:] == 0).all())
    new_len = binding.reform_paged_evict(k, v, score, order.int()[None], i32([n]), n - 64)       # all scores alike: the last keys go
    assert new_len.item() == n - 64
    assert float(v[order[n // 2 // page_len], 0, n // 2 % page_len, n // 2 % d]) == 2.0 ** 26
