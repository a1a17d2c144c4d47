"""GPU: reform_paged_attend against the 64-bit definition: pages of any length, windows, scores written and added, pages that are
not there, padding, lengths outside, strides, shared pages, graphs."""
import math
import random

import pytest
import torch

import paged_reference as ref
import serving_reference as sref
from paper_2506_01215_amd import binding
from serving_checks import finite

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KEPT = 5.0
BF, F = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make_pool(g, pages, hkv, page_len, d, dtype):
    return [sref.randn(g, pages, hkv, page_len, d, dtype=dtype) for _ in range(2)]


def spoil(k, v, table, lens):
    """What lies behind a sequence's last key, and on pages of nobody, is never looked at."""
    page_len = k.shape[2]
    used = {}
    for row, n in zip(table, lens):
        for i in range(-(-n // page_len)):
            used[row[i]] = max(used.get(row[i], 0), min(page_len, n - i * page_len))
    for page in range(k.shape[0]):
        k[page, :, used.get(page, 0):] = math.nan
        v[page, :, used.get(page, 0):] = math.nan


def check_score(got, before, scores, lens, G, accumulate):
    got = got.double().cpu()
    for b, n in enumerate(lens):
        want, off, seen = scores[b]
        have = before[b, :, :n].double().clone()
        if n:
            have[:, n - 1] = 0.0
        if not accumulate:
            have[:] = 0.0
        want = have + want
        finite(got[b, :, :n], f"score of sequence {b}")
        bound = off * 1.01 + (G + 1) * sref.U24 * want.abs() + 1e-30
        bad = (got[b, :, :n] - want).abs() > bound
        assert not bool(bad.any()), f"sequence {b}: {int(bad.sum())} of {bad.numel()} scores off, worst {float(((got[b, :, :n] - want).abs() / bound).max()):.2f}"
        if n:
            assert torch.equal(got[b, :, :n][:, ~seen], want[:, ~seen])
        assert torch.equal(got[b, :, n:], before[b, :, n:].double())     # entries behind the last key stay


def run_case(hq, hkv, d, lens, page_len, dtype, seed, window=0, sinks=0, score=None, sharp=1.0, columns=None, max_len=None, holes=()):
    """score: None, False (written) or True (added).  holes: (sequence, page place) whose table entry is out of the pool."""
    rnd = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    S = len(lens)
    table, pages = ref.make_table(rnd, lens, page_len, columns=columns)
    k, v = make_pool(g, pages, hkv, page_len, d, dtype)
    spoil(k, v, table, lens)
    for n, (b, i) in enumerate(holes):
        table[b][i] = [-1, pages, 1 << 30, -(1 << 31)][n % 4]
    q = (sref.randn(g, S, hq, d) * sharp).to(dtype)
    print(f"[paged] {hq}/{hkv} d={d} {dtype} page={page_len} lens={lens[:6]} window={window}/{sinks} score={score}", flush=True)
    before = torch.rand((S, hkv, max(len(table[0]) * page_len, 1)), generator=g) if score is not None else None
    sc = None if before is None else before.to(DEV)
    out, lse = torch.full((S, hq, d), KEPT, dtype=dtype, device=DEV), torch.full((S, hq), KEPT, device=DEV)
    got, got_lse = binding.reform_paged_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(table), i32(lens), d ** -0.5, window=window, n_sink=sinks,
                                               score=sc, accumulate=bool(score), out=out, lse=lse, max_len=max_len)
    want, want_lse, a, err, scores = ref.paged_attend(q, k, v, table, lens, d ** -0.5, window, sinks)
    for b in range(S):
        ref.check_single(got[b], got_lse[b], want[b], want_lse[b], a[b], err[b], max(1, lens[b]), dtype, f"sequence {b}")
    if score is not None:
        check_score(sc, before, scores, lens, hq // hkv, score)
    return got, got_lse


@pytest.mark.parametrize("hq,hkv,d,lens,dtype", [
    (4, 4, 64, [1], BF), (32, 8, 128, [1, 31, 32, 33, 0, 300], BF), (8, 2, 128, [5000, 3, 2000], BF), (8, 8, 64, [4000], BF),
    (16, 1, 64, [700, 90], BF), (24, 8, 64, [17, 400, 64], BF), (14, 2, 64, [129, 511], BF), (40, 2, 128, [300, 20], BF),
    (64, 1, 64, [1500], BF), (6, 3, 128, [0, 0], BF),
    (4, 4, 64, [1, 500], F), (8, 2, 128, [300, 20, 0], F), (6, 2, 36, [90, 700], F), (2, 1, 256, [1000, 5], F), (40, 2, 100, [40, 17], F),
])
@pytest.mark.parametrize("page_len", [16, 64, 1, 20, 1000])
@pytest.mark.parametrize("score", [None, False])
def test_pages(hq, hkv, d, lens, dtype, page_len, score):
    run_case(hq, hkv, d, lens, page_len, dtype, seed=d + len(lens) + page_len, score=score)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (17, 3), (64, 64), (500, 33), (1000, 40), (5000, 7)])
@pytest.mark.parametrize("page_len", [16, 24])
def test_windows(dtype, d, window, sinks, page_len):
    run_case(8, 2, d, [900, 1, 33, 64, 0, 517, 1400], page_len, dtype, seed=window + sinks, window=window, sinks=sinks, score=window % 2 == 0)


@pytest.mark.parametrize("dtype,d,hq,hkv", [(BF, 128, 8, 2), (BF, 64, 14, 2), (F, 64, 4, 4), (F, 40, 40, 2), (BF, 128, 40, 2)])
def test_scores_are_added_and_the_new_key_has_none(dtype, d, hq, hkv):
    run_case(hq, hkv, d, [700, 1, 0, 64, 2300], 32, dtype, seed=hq, score=True)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F, 64)])
@pytest.mark.parametrize("page_len", [16, 64, 7])
def test_pages_that_are_not_there(dtype, d, page_len):
    """Given back or broken entries: their keys are not seen, also where none is left."""
    lens = [300, 20, 7, 500]
    holes = [(0, 0), (0, 2), (0, 1), (0, 3)] + [(2, i) for i in range(-(-7 // page_len))] + [(3, (499) // page_len), (1, 0)]
    run_case(8, 2, d, lens, page_len, dtype, seed=page_len, score=False, holes=holes)
    run_case(8, 2, d, lens, page_len, dtype, seed=page_len, score=True, holes=holes, window=100, sinks=20)


@pytest.mark.parametrize("dtype,d,hq,hkv", [(BF, 128, 8, 2), (BF, 64, 16, 2), (F, 64, 8, 2)])
def test_long_and_ragged(dtype, d, hq, hkv):
    """Shares begin and end inside sequences; more sequences than a wave has lanes."""
    rnd = random.Random(1)
    run_case(hq, hkv, d, [9000, 100, 7777, 1], 64, dtype, seed=2, score=True)
    lens = [rnd.choice([0, 1, 64, rnd.randint(0, 90), rnd.randint(0, 1200)]) for _ in range(90)]
    run_case(hq, hkv, d, lens, 16, dtype, seed=3, score=False)
    run_case(4, 1, d, lens[:70], 16, dtype, seed=4, window=40, sinks=5, score=True)
    run_case(4, 1, d, [20000], 128, dtype, seed=5, window=15000, sinks=1000, score=True)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F, 64)])
def test_more_items_than_shares(dtype, d):
    """Hundreds of sequences, a few of them long: shares hold many items, and pieces are found by the shares' ends."""
    rnd = random.Random(9)
    lens = [rnd.choice([0, 1, 5, rnd.randint(0, 60)]) for _ in range(290)]
    for i in (0, 77, 78, 150, 289):
        lens[i] = rnd.randint(2600, 3000)
    run_case(4, 2, d, lens, 32, dtype, seed=6, score=True)
    run_case(2, 2, d, lens, 16, dtype, seed=7)


def test_table_wider_than_the_sequences():
    """The plan goes by what the lengths may be, the result by what they are."""
    run_case(8, 2, 128, [50, 0, 3], 16, BF, seed=1, columns=900, score=True)
    run_case(8, 2, 64, [50, 0, 300], 16, BF, seed=1, columns=900, max_len=310, score=False)
    run_case(8, 2, 64, [50, 0, 300], 16, F, seed=1, columns=900, score=True)


@pytest.mark.parametrize("d,page_len", [(128, 16), (128, 20), (64, 16), (64, 20)])
@pytest.mark.parametrize("window", [0, 3000])
def test_calls_that_may_read_much(d, page_len, window):
    """Tables that have room for 64 MB of keys and values: read past the caches' usual order."""
    columns = 9000 // page_len * 128 // d * 4
    run_case(8, 2, d, [6000, 1, 0, 333, 2700], page_len, BF, seed=d, columns=columns, window=window, sinks=7 if window else 0, score=True)
    run_case(14, 2, d, [17, 4000], page_len, BF, seed=d + 1, columns=3 * columns, window=2 * window, score=None)


@pytest.mark.parametrize("dtype", [BF, F])
def test_lengths_outside_are_moved_in(dtype):
    g = torch.Generator().manual_seed(3)
    k, v = make_pool(g, 12, 2, 16, 64, dtype)
    q = sref.randn(g, 3, 4, 64, dtype=dtype)
    table = [[0, 1, 2, 3], [4, 5, 6, 7], [8, 9, 10, 11]]
    out, lse = binding.reform_paged_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(table), i32([-5, 1 << 30, 30]), 0.125, max_len=50)
    want, wl, a, err, _ = ref.paged_attend(q, k, v, table, [0, 50, 30], 0.125)
    ref.check_single(out, lse, want, wl, a, err, 64, dtype)


def test_sharp_logits():
    run_case(8, 2, 128, [2000, 100], 16, BF, seed=5, sharp=15.0, score=True)
    run_case(4, 2, 64, [300], 16, F, seed=5, sharp=15.0, score=False)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("page_len", [16, 10])
def test_strides_and_shared_pages(dtype, page_len):
    """A pool [pages, rows, heads, elements] with room between rows, a table that is a slice of a wider one, q and out inside
    wider tensors, scores with room between heads, a preamble that sequences share."""
    S, hq, hkv, d, n = 3, 6, 2, 64, [70, 45, 64]
    g = torch.Generator().manual_seed(6)
    pages = 30
    raw = [sref.randn(g, pages, page_len, hkv + 1, d, dtype=dtype) for _ in range(2)]
    pool = [x[:, :, :hkv].transpose(1, 2) for x in raw]
    dev = [x.to(DEV)[:, :, :hkv].transpose(1, 2) for x in raw]
    rnd = random.Random(2)
    own = list(range(4, pages))
    rnd.shuffle(own)
    table = [[0, 1, 2] + own[8 * b:8 * b + 8] for b in range(S)]         # the first three pages are everybody's
    wide = i32([[99] * 5 + row for row in table])
    q = sref.randn(g, hq + 2, S, d, dtype=dtype)
    out = torch.zeros(S, hq, 2 * d, dtype=dtype, device=DEV)[..., :d]
    before = torch.rand(S, hkv, 200, generator=g)
    sc = before.to(DEV)
    got, lse = binding.reform_paged_attend(q.to(DEV)[:hq].transpose(0, 1), *dev, wide[:, 5:], i32(n), 0.125, score=sc[..., :80], accumulate=True, out=out)
    want, wl, a, err, scores = ref.paged_attend(q[:hq].transpose(0, 1), *pool, table, n, 0.125)
    ref.check_single(got, lse, want, wl, a, err, 80, dtype)
    check_score(sc, before, scores, n, hq // hkv, True)


@pytest.mark.parametrize("dtype", [BF, F])
def test_values_that_are_not_finite_stay_in_their_place(dtype):
    """In keys that are not seen (behind the window) they change nothing; in a seen key, only their sequence and head."""
    lens = [200, 150]
    table, pages = ref.make_table(random.Random(1), lens, 16)
    g = torch.Generator().manual_seed(8)
    k, v = make_pool(g, pages, 2, 16, 64, dtype)
    q = sref.randn(g, 2, 4, 64, dtype=dtype).to(DEV)
    call = lambda: binding.reform_paged_attend(q, k.to(DEV), v.to(DEV), i32(table), i32(lens), 0.125, window=50, n_sink=3)  # noqa: E731
    clean = call()
    for j in (3, 100, 149):                                              # behind the window, and between it and the first keys
        k[table[0][j // 16], :, j % 16], v[table[0][j // 16], :, j % 16] = math.nan, math.inf
    got = call()
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    v[table[0][160 // 16], 1, 0] = math.nan
    got = call()
    assert torch.equal(got[0][1], clean[0][1]) and torch.equal(got[0][0, :2], clean[0][0, :2])
    assert bool(torch.isnan(got[0][0, 2:]).all())


def test_nothing_to_see_at_all():
    """No pages in the pool, no columns in the table: zeros and -inf."""
    q = torch.randn(2, 4, 64, device=DEV).to(BF)
    none = torch.zeros(0, 2, 16, 64, dtype=BF, device=DEV)
    for table in (i32([[0, 1], [5, -1]]), torch.zeros(2, 0, dtype=torch.int32, device=DEV)):
        out, lse = binding.reform_paged_attend(q, none, none, table, i32([20, 3]), 0.125)
        assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    out, lse = binding.reform_paged_attend(q[:0], none, none, torch.zeros(0, 3, dtype=torch.int32, device=DEV), i32([]), 0.125)
    assert out.shape[0] == 0


@pytest.mark.parametrize("shared", [False, True])
def test_graph_follows_lengths_and_table(shared):
    g = torch.Generator().manual_seed(9)
    page_len, cap = 16, 4800 if shared else 480
    pages = 2 * cap // page_len
    k, v = (x.to(DEV) for x in make_pool(g, pages, 2, page_len, 128, BF))
    q = sref.randn(g, 2, 8, 128, dtype=BF).to(DEV)
    table, lens = i32(torch.randperm(pages, generator=g).view(2, -1).tolist()), i32([cap, 100])
    score = torch.zeros(2, 2, cap, device=DEV)
    out, lse = torch.zeros_like(q), torch.zeros(2, 8, device=DEV)
    ws = torch.empty(binding.paged_workspace_bytes(binding.paged_desc(q, k, v, out, table, 0.1, score=score, accumulate=True)) + 256,
                     dtype=torch.uint8, device=DEV)
    call = lambda s, o, l: binding.reform_paged_attend(q, k, v, table, lens, 0.1, score=s, accumulate=True, out=o, lse=l, workspace=ws)  # noqa: E731
    call(score, out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(score, out, lse)
    for n in ([cap, 100], [1, cap], [0, 0], [333, 17]):
        lens.copy_(i32(n))
        table.copy_(i32(torch.randperm(pages, generator=g).view(2, -1).tolist()))
        q.copy_(torch.randn(q.shape, device=DEV))
        score.copy_(torch.rand(score.shape, device=DEV))
        eager = score.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        want = call(eager, torch.zeros_like(q), torch.zeros_like(lse))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(score, eager)


def test_two_streams_and_repeats():
    """Two calls at once with workspaces of their own, each the same bits as alone."""
    g = torch.Generator().manual_seed(10)
    table, pages = ref.make_table(random.Random(1), [6000, 30, 2500], 16)
    k, v = (x.to(DEV) for x in make_pool(g, pages, 2, 16, 64, BF))
    table, lens = i32(table), i32([6000, 30, 2500])
    qs = [sref.randn(g, 3, 8, 64, dtype=BF).to(DEV) for _ in range(2)]
    alone = [binding.reform_paged_attend(q, k, v, table, lens, 0.125, score=torch.zeros(3, 2, 6000, device=DEV)) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    scores = [torch.zeros(3, 2, 6000, device=DEV) for _ in qs]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [binding.reform_paged_attend(q, k, v, table, lens, 0.125, score=s, stream=st) for q, s, st in zip(qs, scores, streams)]
        torch.cuda.synchronize()
        for (a, b), (c, d) in zip(alone, got):
            assert torch.equal(a, c) and torch.equal(b, d)
