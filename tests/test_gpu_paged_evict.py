"""GPU: reform_paged_evict against an exhaustive sort, byte for byte: pages of any length, batches in which some outgrew their
budget, ties, protected keys, pages that are not there, strides, graphs."""
import random

import pytest
import torch

import paged_reference as ref
from paper_2506_01215_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def expected(k, v, score, pos, table, lens, budget, n_sink, n_recent):
    """The definition, head by head, on copies."""
    k, v, score, pos = k.clone(), v.clone(), score.clone(), pos.clone()
    pages, hkv, page_len, _ = k.shape
    kept = torch.full((len(lens), hkv, budget), -7, dtype=torch.int32)
    for b, n in enumerate(lens):
        for h in range(hkv):
            keep = ref.evict(score[b, h], n, budget, n_sink, n_recent)
            kept[b, h, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
            if n <= budget:
                continue
            for x in (k, v):
                moved = []
                for j in keep:
                    at = table[b][j // page_len]
                    moved.append(x[at, h, j % page_len].clone() if 0 <= at < pages else None)
                for r, row in enumerate(moved):
                    at = table[b][r // page_len]
                    if row is not None and 0 <= at < pages:
                        x[at, h, r % page_len] = row
            at = torch.tensor(keep)
            score[b, h, :budget], pos[b, h, :budget] = score[b, h, at].clone(), pos[b, h, at].clone()
    return k, v, score, pos, kept


def scores_of(kind, g, shape):
    if kind == "spread":
        return torch.randn(shape, generator=g).mul(2).exp()
    if kind == "ties":
        return torch.randint(0, 5, shape, generator=g).float()
    if kind == "equal":
        return torch.full(shape, 0.25)
    if kind == "signs":                                                  # both zeros are alike, negative ones come last
        return torch.randint(-3, 3, shape, generator=g).float() * torch.where(torch.rand(shape, generator=g) < 0.3, -0.0, 1.0)
    if kind == "subnormal":                                              # zeros of both signs and numbers below the smallest normal one
        return torch.randint(-9, 200, shape, generator=g, dtype=torch.int32).clamp_min(-1).mul(3).float() * 2.0 ** -149 \
            * torch.where(torch.rand(shape, generator=g) < 0.3, -0.0, 1.0)
    return torch.rand(shape, generator=g) * 1e-30 + 1.0 * (torch.rand(shape, generator=g) < 0.1)      # far apart


def run_case(hkv, d, lens, page_len, budget, n_sink, n_recent, dtype, seed, kind="spread", holes=(), columns=None, with_pos=True, with_kept=True):
    rnd = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    table, pages = ref.make_table(rnd, lens, page_len, columns=columns)
    for n, (b, i) in enumerate(holes):
        table[b][i] = [-1, pages, 1 << 30][n % 3]
    k, v = (torch.randn(pages, hkv, page_len, d, generator=g).to(dtype) for _ in range(2))
    cols = len(table[0]) * page_len
    score = scores_of(kind, g, (len(lens), hkv, cols))
    pos = torch.randint(0, 1 << 30, (len(lens), hkv, cols), generator=g, dtype=torch.int32)
    print(f"[evict] hkv={hkv} d={d} {dtype} page={page_len} lens={lens[:6]} budget={budget} {n_sink}+{n_recent} {kind}", flush=True)
    want = expected(k, v, score, pos, table, lens, budget, n_sink, n_recent)
    dk, dv, ds, dp = (x.to(DEV) for x in (k, v, score, pos))
    kept = torch.full((len(lens), hkv, budget), -7, dtype=torch.int32, device=DEV)
    new_len = binding.reform_paged_evict(dk, dv, ds, i32(table), i32(lens), budget, n_sink=n_sink, n_recent=n_recent,
                                         pos=dp if with_pos else None, kept_idx=kept if with_kept else None)
    torch.cuda.synchronize()
    assert new_len.tolist() == [min(n, budget) for n in lens]
    got = (dk, dv, ds) + ((dp,) if with_pos else ()) + ((kept,) if with_kept else ())
    names = ("k", "v", "score") + (("pos",) if with_pos else ()) + (("kept",) if with_kept else ())
    wants = dict(zip(("k", "v", "score", "pos", "kept"), want))
    for name, x in zip(names, got):
        y = wants[name]
        assert torch.equal(x.cpu(), y), f"{name}: {int((x.cpu() != y).sum())} of {y.numel()} differ"


@pytest.mark.parametrize("hkv,d,lens,page_len,budget,n_sink,n_recent,dtype", [
    (1, 64, [2], 16, 1, 0, 0, BF), (2, 128, [100, 30, 0, 65], 16, 64, 0, 0, BF), (2, 64, [300, 301, 299], 32, 299, 4, 20, BF),
    (8, 128, [1200, 700, 1025], 64, 1000, 16, 256, BF), (1, 128, [5000], 16, 4097, 4, 64, BF), (3, 64, [130], 1, 70, 1, 1, BF),
    (2, 64, [257, 400], 20, 256, 256, 0, BF), (2, 64, [257, 400], 20, 256, 0, 256, BF), (2, 64, [257, 400], 7, 256, 100, 156, BF),
    (4, 64, [384, 300, 257, 120], 16, 256, 4, 128, F), (2, 4, [90], 16, 33, 2, 3, F), (2, 256, [200, 40], 10, 150, 0, 9, F),
    (1, 24, [100], 16, 50, 0, 0, BF), (1, 1024, [80], 16, 60, 0, 5, F),
])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "signs", "apart"])
def test_budgets(hkv, d, lens, page_len, budget, n_sink, n_recent, dtype, kind):
    run_case(hkv, d, lens, page_len, budget, n_sink, n_recent, dtype, seed=budget + d, kind=kind)


@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_long_rows(kind):
    """More candidates than LDS holds, and a budget close to all and to nothing."""
    run_case(1, 64, [40000], 64, 39000, 4, 100, BF, seed=1, kind=kind)
    run_case(1, 64, [40000], 64, 50, 4, 10, BF, seed=2, kind=kind)
    run_case(2, 64, [9000, 8999, 20], 128, 8998, 0, 1, BF, seed=3, kind=kind)


def test_outputs_that_are_not_wanted():
    run_case(2, 64, [100, 70], 16, 60, 4, 4, BF, seed=1, with_pos=False)
    run_case(2, 64, [100, 70], 16, 60, 4, 4, BF, seed=2, with_kept=False)
    run_case(2, 64, [100, 70], 16, 60, 4, 4, BF, seed=3, with_pos=False, with_kept=False, columns=40)


def test_nobody_outgrew():
    run_case(2, 64, [10, 0, 64], 16, 64, 4, 4, BF, seed=1)
    run_case(2, 64, [10, 0, 64], 16, 64, 4, 4, BF, seed=1, columns=20)


@pytest.mark.parametrize("page_len", [16, 9])
def test_pages_that_are_not_there(page_len):
    """Rows that would come from there or go there stay as they are; everything else moves."""
    run_case(2, 64, [200, 150], page_len, 100, 2, 10, BF, seed=page_len, holes=[(0, 1), (0, 7), (1, 3), (1, 0)])


def test_many_sequences():
    rnd = random.Random(4)
    run_case(1, 64, [rnd.randint(0, 90) for _ in range(100)], 16, 40, 3, 7, BF, seed=5)


@pytest.mark.parametrize("dtype", [BF, F])
def test_strides(dtype):
    """A pool [pages, rows, heads, elements], scores with room between heads, a table inside a wider one."""
    rnd, g = random.Random(6), torch.Generator().manual_seed(6)
    lens, page_len, hkv, d, budget = [90, 40], 16, 2, 64, 50
    table, pages = ref.make_table(rnd, lens, page_len)
    raw = [torch.randn(pages, page_len, hkv + 1, d, generator=g).to(dtype) for _ in range(2)]
    cols = len(table[0]) * page_len
    score, pos = torch.rand(2, hkv, cols + 9, generator=g), torch.randint(0, 99, (2, hkv, cols + 9), generator=g, dtype=torch.int32)
    k, v = (x[:, :, :hkv].transpose(1, 2) for x in raw)
    want = expected(k, v, score[..., :cols], pos[..., :cols], table, lens, budget, 2, 5)
    dev = [x.to(DEV) for x in raw]
    dk, dv = (x[:, :, :hkv].transpose(1, 2) for x in dev)
    ds, dp = score.to(DEV), pos.to(DEV)
    wide = i32([[77] * 3 + row for row in table])
    binding.reform_paged_evict(dk, dv, ds[..., :cols], wide[:, 3:], i32(lens), budget, n_sink=2, n_recent=5, pos=dp[..., :cols])
    for x, y in ((dk, want[0]), (dv, want[1]), (ds[..., :cols], want[2]), (dp[..., :cols], want[3])):
        assert torch.equal(x.cpu(), y)
    for x, y in zip(dev, raw):                                           # the head beside is nobody's
        assert torch.equal(x[:, :, hkv].cpu(), y[:, :, hkv])
    assert torch.equal(ds[..., cols:].cpu(), score[..., cols:])


def test_lengths_outside_are_moved_in():
    g = torch.Generator().manual_seed(7)
    table = [[0, 1, 2, 3], [4, 5, 6, 7]]
    k, v = (torch.randn(8, 1, 16, 64, generator=g).to(BF) for _ in range(2))
    score, pos = torch.rand(2, 1, 64, generator=g), torch.zeros(2, 1, 64, dtype=torch.int32)
    want = expected(k, v, score, pos, table, [0, 50], 30, 0, 0)
    dk, dv, ds = (x.to(DEV) for x in (k, v, score))
    new_len = binding.reform_paged_evict(dk, dv, ds, i32(table), i32([-9, 1 << 30]), 30, max_len=50)
    assert new_len.tolist() == [0, 30]
    assert torch.equal(dk.cpu(), want[0]) and torch.equal(ds.cpu(), want[2])


def test_scores_that_are_not_numbers_stay_inside():
    """Which keys stay is then open; that nothing else is touched, and that all ends, is not."""
    g = torch.Generator().manual_seed(8)
    table, pages = [[3, 1, 0, 5, 2]], 7
    k, v = (torch.randn(pages, 2, 16, 64, generator=g).to(BF).to(DEV) for _ in range(2))
    before = k.clone()
    for bad in (float("nan"), -float("nan"), float("inf"), -float("inf")):
        score = torch.rand(1, 2, 80, device=DEV)
        score[0, 0, ::3] = bad
        kept = torch.full((1, 2, 40), -7, dtype=torch.int32, device=DEV)
        binding.reform_paged_evict(k, v, score, i32(table), i32([80]), 40, kept_idx=kept)
        x = kept[0, 0].tolist()
        assert x == sorted(set(x)) and 0 <= x[0] and x[-1] < 80
        assert torch.equal(k[[4, 6]], before[[4, 6]])


def test_graph_follows_lengths_and_scores():
    g = torch.Generator().manual_seed(9)
    k, v = (torch.randn(40, 2, 16, 64, generator=g).to(BF).to(DEV) for _ in range(2))
    table, lens = i32(torch.randperm(40, generator=g).view(2, -1).tolist()), i32([320, 100])
    score = torch.rand(2, 2, 320, device=DEV)
    new_len = torch.zeros(2, dtype=torch.int32, device=DEV)
    ws = torch.empty(binding.paged_evict_workspace_bytes(binding.paged_evict_desc(k, v, score, table, 128, 4, 32)) + 256, dtype=torch.uint8, device=DEV)
    call = lambda a, b, s, n: binding.reform_paged_evict(a, b, s, table, lens, 128, n_sink=4, n_recent=32, new_len=n, workspace=ws)  # noqa: E731
    call(k, v, score, new_len)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(k, v, score, new_len)
    for n in ([320, 129], [128, 127], [0, 320], [200, 300]):
        lens.copy_(i32(n))
        table.copy_(i32(torch.randperm(40, generator=g).view(2, -1).tolist()))
        score.copy_(torch.rand(score.shape, device=DEV))
        k.copy_(torch.randn(k.shape, device=DEV))
        eager = k.clone(), v.clone(), score.clone()
        graph.replay()
        torch.cuda.synchronize()
        want_len = call(*eager, torch.zeros_like(new_len))
        assert torch.equal(k, eager[0]) and torch.equal(v, eager[1]) and torch.equal(score, eager[2]) and torch.equal(new_len, want_len)


@pytest.mark.parametrize("lens,budget,n_sink,n_recent", [
    ([4300], 4096, 4, 64),                  # few rows go: segments move at once
    ([9000, 4200, 100], 4096, 0, 0),        # more go than is staged, beside one where few do
    ([16500, 16385], 16384, 300, 200), ([8193], 8192, 8000, 0), ([8193], 8192, 0, 8000),
])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal"])
@pytest.mark.parametrize("page_len", [16, 50])
def test_rows_in_segments(lens, budget, n_sink, n_recent, kind, page_len):
    run_case(1, 64, lens, page_len, budget, n_sink, n_recent, BF, seed=budget, kind=kind)
    run_case(2, 4, lens, page_len, budget, n_sink, n_recent, F, seed=budget, kind=kind, columns=max(lens) // page_len + 9)


def test_segments_and_pages_that_are_not_there():
    run_case(1, 64, [4300], 64, 4096, 4, 64, BF, seed=1, holes=[(0, 31), (0, 32), (0, 16), (0, 48), (0, 66)])


def test_the_first_rows_go():
    """Every segment's last rows come from the next one's."""
    rnd, g = random.Random(1), torch.Generator().manual_seed(1)
    n, budget, page_len = 4500, 4096, 32
    table, pages = ref.make_table(rnd, [n], page_len)
    k, v = (torch.randn(pages, 1, page_len, 64, generator=g).to(BF) for _ in range(2))
    score = torch.arange(len(table[0]) * page_len).float()[None, None].clone()
    pos = torch.arange(score.shape[2], dtype=torch.int32)[None, None].clone()
    want = expected(k, v, score, pos, table, [n], budget, 0, 0)
    dk, dv, ds, dp = (x.to(DEV) for x in (k, v, score, pos))
    binding.reform_paged_evict(dk, dv, ds, i32(table), i32([n]), budget, pos=dp)
    for x, y in zip((dk, dv, ds, dp), want):
        assert torch.equal(x.cpu(), y)


@pytest.mark.parametrize("lens,budget", [([384, 300], 256), ([9000], 8200), ([40000], 39000), ([36000], 700)])
def test_subnormal_scores(lens, budget):
    run_case(1, 64, lens, 64, budget, 4, 10, BF, seed=budget, kind="subnormal")


@pytest.mark.parametrize("kind", ["equal", "signs", "apart"])
def test_long_rows_of_other_scores(kind):
    """Rows that are read anew in every pass: runs of candidates that end inside 512 and inside 64."""
    for n, budget in ((32900 + 14, 32000), (33800, 33700), (50001, 25000)):
        run_case(1, 64, [n], 64, budget, 4, 10, BF, seed=n, kind=kind)


@pytest.mark.parametrize("columns", [None, 640])
@pytest.mark.parametrize("budget,gone", [(2048, (1, 73, 128, 300)), (2050, (500, 1024, 1025, 1026)), (777, (1, 97, 388, 389)), (4097, (64, 2048, 2049, 4500)), (256, (3, 64, 129))])
def test_segments_by_the_keys_that_go(budget, gone, columns):
    """An item's segments follow from how many of its keys go, whatever its neighbours' do and the table has room for."""
    for kind in ("spread", "ties"):
        run_case(1, 64, [budget + n for n in gone], 16, budget, 4, 10, BF, seed=budget, kind=kind, columns=columns)
