"""GPU: the attention calls where elements lie further than 2^31 from a tensor's first one, in every form.

Prompts: rows of q, k, v and out so far apart that the last ones do; the result has to be that of the same call on dense tensors, bit
for bit (strides choose no form), and a dense one is held against the 64-bit definition.  Trees: sequences that far apart, and
caches so long that their last rows are; there all keys but a few are zero, so that the result is known."""
import math
import random

import pytest
import torch

import serving_checks
import serving_reference as ref
from paper_2506_01215_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
FAR = 1 << 31


@pytest.fixture(autouse=True)
def give_back():
    """Some 16 to 35 GB a test: not kept for the tests that follow."""
    yield
    torch.cuda.empty_cache()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def starts(lens):
    got = [0]
    for n in lens:
        got.append(got[-1] + n)
    return got


def apart(x, row_stride, fill=True):
    """x [heads, rows, d] on the GPU, token-major with rows `row_stride` elements apart; what lies between is never initialised."""
    h, n, d = x.shape
    assert row_stride >= h * d and (n - 1) * row_stride + h * d > FAR
    view = torch.empty((n - 1) * row_stride + h * d, dtype=x.dtype, device=DEV).as_strided((h, n, d), (d, row_stride, 1))
    if fill:
        for i in range(0, n, 64):                                            # a view of few elements at a time
            view[:, i:i + 64].copy_(x[:, i:i + 64])
    return view


@pytest.mark.parametrize("d,hq,hkv,q_lens,k_lens,dtype,shared", [
    # every whole form, by the same batches as the tests of the forms: rows of a block, groups of waves
    (64, 2, 2, [300, 150, 250], None, BF, False), (64, 7, 1, [900], None, BF, False), (64, 24, 8, [140, 3, 200, 157, 200], None, BF, False),
    (64, 8, 1, [12000], None, BF, False), (128, 6, 2, [100, 1, 170, 0, 229, 100, 100], None, BF, False), (128, 3, 1, [1000], None, BF, False),
    (128, 16, 2, [300, 400, 200, 300], None, BF, False), (128, 12, 4, [125] * 40, None, BF, False), (64, 4, 2, [700, 300], None, F, False),
    # and every shared one: blocks of 16, 32, 64 and 128 rows
    (128, 8, 2, [3, 40], [9000, 70], BF, True), (128, 32, 8, [6, 5, 7, 6], [5000, 4000, 6000, 5200], BF, True),
    (128, 32, 8, [16], [11000], BF, True), (128, 32, 8, [30, 3, 0, 31], [8000, 5, 9000, 15000], BF, True), (64, 4, 4, [1] * 3, [9000, 33, 8000], BF, True),
    (64, 32, 8, [6, 5, 7, 6], [6500, 64, 13000, 6500], BF, True), (64, 32, 8, [12, 10, 14, 12], [7000, 7000, 7000, 7031], BF, True),
    (64, 16, 4, [30, 20], [32001, 33000], BF, True), (64, 4, 2, [3, 20], [3000, 5], F, True),
])
def test_prompts_with_rows_far_apart(d, hq, hkv, q_lens, k_lens, dtype, shared):
    nq, nk = sum(q_lens), sum(k_lens or q_lens)
    g = torch.Generator().manual_seed(nq + d)
    q, k, v = (ref.randn(g, h, n, d, dtype=dtype) for h, n in ((hq, nq), (hkv, nk), (hkv, nk)))
    dense = [x.to(DEV) for x in (q, k, v)]
    cu_q, cu_k, scale = i32(starts(q_lens)), i32(starts(k_lens)) if k_lens else None, d ** -0.5
    print(f"[far prompts] {hq}/{hkv} d={d} {dtype} q={q_lens[:6]} k={k_lens}", flush=True)
    need = binding.prompt_workspace_bytes(binding.prompt_desc(*dense, dense[0], cu_q, scale))
    assert (need > 0) == shared
    out, lse = binding.reform_prompt_attend(*dense, cu_q, scale, cu_k=cu_k)
    for h in sorted({0, hq - 1}):
        one = slice(h * hkv // hq, h * hkv // hq + 1)
        want = ref.prompt_attend(q[h:h + 1], k[one], v[one], q_lens, k_lens or q_lens, scale)
        serving_checks.check_attention(out[h:h + 1], lse[h:h + 1], *want, max(k_lens or q_lens), dtype, f"head {h}")
    stride = lambda n: FAR // (n - 1) // 64 * 64 + 64  # noqa: E731
    far_q, far_out = apart(dense[0], stride(nq)), apart(dense[0], stride(nq), fill=False)
    far_out.zero_()
    far_k, far_v = (dense[i] if stride(nk) >= 1 << 24 else apart(dense[i], stride(nk)) for i in (1, 2))
    got, got_lse = binding.reform_prompt_attend(far_q, far_k, far_v, cu_q, scale, cu_k=cu_k, out=far_out)
    assert torch.equal(got, out) and torch.equal(got_lse, lse)


@pytest.mark.parametrize("d,hq,hkv,q_lens,dtype", [(64, 6, 2, [130, 70], BF), (128, 4, 1, [200], BF), (64, 2, 1, [140], F)])
def test_the_largest_row_stride(d, hq, hkv, q_lens, dtype):
    """Keys at the largest stride that is taken: 63 rows of a tile are 63 (2^24 - 64) elements apart."""
    n, widest = sum(q_lens), (1 << 24) - 64
    g = torch.Generator().manual_seed(d)
    q, k, v = (ref.randn(g, h, n, d, dtype=dtype).to(DEV) for h in (hq, hkv, hkv))
    cu = i32(starts(q_lens))
    out, lse = binding.reform_prompt_attend(q, k, v, cu, 0.1)
    got, got_lse = binding.reform_prompt_attend(q, apart(k, widest), apart(v, widest), cu, 0.1)
    assert torch.equal(got, out) and torch.equal(got_lse, lse)


def far_sequences(x, step, rows=None):
    """x [S, heads, n, d]: sequences `step` elements apart on the GPU, the n rows in front of room for `rows`."""
    S, h, n, d = x.shape
    rows = n if rows is None else rows
    assert step >= h * rows * d and (S - 1) * step + h * rows * d > FAR
    view = torch.empty((S - 1) * step + h * rows * d, dtype=x.dtype, device=DEV).as_strided((S, h, rows, d), (step, rows * d, d, 1))
    for b in range(S):
        view[b, :, :n].copy_(x[b])
    return view


def far_trees(hq, hkv, d, T, lens, counts, cap, have, dtype, seed):
    S = len(lens)
    step = FAR // (S - 1) // 64 * 64 + 64
    rnd = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    q, k, v = ref.randn(g, S, hq, T, d, dtype=dtype), *(ref.randn(g, S, hkv, have, d, dtype=dtype) for _ in range(2))
    parents = [ref.random_parents(rnd, T) for _ in range(S)]
    dq, out, dk, dv = far_sequences(q, step), far_sequences(torch.zeros_like(q), step), far_sequences(k, step, cap), far_sequences(v, step, cap)
    print(f"[far trees] {hq}/{hkv} d={d} T={T} {dtype} S={S} cap={cap}", flush=True)
    need = binding.tree_workspace_bytes(binding.tree_desc(dq, dk, dv, out, 0.1))
    got, lse = binding.reform_tree_attend(dq, dk, dv, i32(lens), d ** -0.5, parent=i32(parents), node_count=i32(counts), out=out)
    want = ref.tree_attend(q, k, v, lens, parents, counts, d ** -0.5)
    for b in range(S):
        m = counts[b]
        if m:
            serving_checks.check_attention(got[b, :, :m], lse[b, :, :m], *(x[b, :, :m] for x in want), lens[b] + m, dtype, f"sequence {b}")
        assert not bool(got[b, :, m:].any())
    return need


# one KV head: 12, 32, 64, 120, 180 and 256 rows, each in a block of its own where caches are long
FORMS = [(1, 4, 64, 3, BF), (1, 4, 64, 8, BF), (1, 4, 64, 16, BF), (1, 4, 64, 30, BF), (1, 4, 64, 45, BF), (1, 4, 64, 64, BF),
         (1, 4, 128, 3, BF), (1, 4, 128, 8, BF), (1, 4, 128, 16, BF), (1, 4, 128, 30, BF), (1, 4, 128, 45, BF), (1, 4, 128, 64, BF), (1, 2, 64, 5, F)]


@pytest.mark.parametrize("hkv,hq,d,T,dtype", FORMS)
def test_trees_of_sequences_far_apart(hkv, hq, d, T, dtype):
    """q, out and the caches of three sequences more than 2^30 elements apart, shared out, in every form."""
    need = far_trees(hq, hkv, d, T, [2900, 0, 77], [T, T, T - 1], 2000000, 3000, dtype, T + d)
    if dtype == BF:
        rows, units = T * hq // hkv, torch.cuda.get_device_properties(0).multi_processor_count
        block = next(x for x in (16, 32, 64, 128, 192, 256) if rows <= x)
        assert need == 2 * min((2 if block == 128 or (block <= 32 and d == 64) else 1) * units, 512) * min(rows, block) * (4 * d + 8)
    assert need > 0


@pytest.mark.parametrize("hq,hkv,d,T,n,top,dtype", [
    (8, 8, 64, 16, 60, 300, BF), (8, 2, 128, 8, 250, 70, BF), (16, 8, 64, 30, 80, 90, BF), (8, 2, 128, 28, 200, 30, BF), (16, 4, 64, 60, 130, 64, BF),
    (16, 4, 128, 60, 110, 100, BF), (21, 3, 64, 64, 100, 70, BF), (12, 4, 128, 50, 120, 90, BF), (16, 4, 64, 48, 130, 130, BF), (2, 2, 64, 3, 60, 50, F),
])
def test_short_trees_far_apart(hq, hkv, d, T, n, top, dtype):
    """The same for the forms that take a short cache whole."""
    rnd = random.Random(n)
    lens = [rnd.choice([0, 1, top, rnd.randint(0, top)]) for _ in range(n)]
    assert far_trees(hq, hkv, d, T, lens, [rnd.choice([T, T, rnd.randint(0, T)]) for _ in range(n)], top + T, top + T, dtype, n) == 0


@pytest.mark.parametrize("hkv,hq,d,T,dtype", FORMS)
def test_trees_over_caches_longer_than_31_bits(hkv, hq, d, T, dtype):
    """One cache whose rows reach beyond 2^31 elements.  All logits are 0 but those of a row in front, one behind 2^31 elements and the
    drafted tokens', which are 32; V is 0 elsewhere."""
    rows = FAR // d + 5000
    L = rows - T
    k, v = (torch.zeros((1, hkv, rows, d), dtype=dtype, device=DEV) for _ in range(2))
    q = torch.zeros((1, hq, T, d), dtype=dtype, device=DEV)
    q[..., 0] = 32.0 * d ** 0.5 / 16.0
    first, last = 3, L - 70
    assert last * d > FAR
    at = [first, last, *range(L, rows)]
    value = {first: 1.0, last: 2.0, **{L + i: 4.0 + i for i in range(T)}}
    for j in at:
        k[0, 0, j, 0] = 16.0
        v[0, 0, j] = value[j]
    parents = ref.random_parents(random.Random(T), T)
    print(f"[long trees] {hq}/{hkv} d={d} T={T} {dtype}", flush=True)
    out, lse = binding.reform_tree_attend(q, k, v, i32([L]), d ** -0.5, parent=i32([parents]))
    # a logit is formed from one exact product, times scale log2 e: an exponent of some 46 with three roundings, 3 * 46 * 2^-24 < 2^-16 of
    # it; a bf16 probability is rounded once more, and so is the result
    u = ref.half_step(dtype)
    logit = float(q[0, 0, 0, 0]) * 16.0 * d ** -0.5
    for i in range(T):
        seen = [first, last, *(L + j for j in ref.line_of(parents, i))]
        total = len(seen) * math.exp(logit) + (L + len(ref.line_of(parents, i)) - len(seen))
        want = sum(value[j] for j in seen) * math.exp(logit) / total
        bound = want * (2 * u + 2.0 ** -16)
        assert bool(((out[0, :, i].double() - want).abs() <= bound).all()), i
        assert bool(((lse[0, :, i].double() - math.log(total)).abs() <= 46 * 4 * 2.0 ** -24 + 2.0 ** -16).all()), i
