"""GPU: reform_tree_attend against the 64-bit definition: trees, chains and single tokens over caches of any
lengths, split over workgroups and not, padded batches, broken parents and lengths, strides."""
import math
import random

import pytest
import torch

import serving_reference as ref
from paper_2506_01215_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KEPT = 5.0
BF, F = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def run_case(hq, hkv, d, T, lens, dtype, seed, chain=False, counts=None, spare=3, parents=None, sharp=1.0, max_len=None):
    rnd = random.Random(seed)
    g = torch.Generator().manual_seed(seed)
    S, cap = len(lens), max(lens) + T + spare
    q = (ref.randn(g, S, hq, T, d) * sharp).to(dtype)
    k, v = (ref.randn(g, S, hkv, cap, d, dtype=dtype) for _ in range(2))
    if parents is None and not chain:
        parents = [ref.random_parents(rnd, T) for _ in range(S)]
    used = [T] * S if counts is None else [min(max(c, 0), T) for c in counts]
    for b in range(S):           # what lies behind the last row is never looked at
        k[b, :, lens[b] + used[b]:] = math.nan
        v[b, :, lens[b] + used[b]:] = math.nan
    print(f"[tree] {hq}/{hkv} d={d} T={T} {dtype} lens={lens[:6]} chain={chain} counts={counts}", flush=True)
    out = torch.full((S, hq, T, d), KEPT, dtype=dtype, device=DEV)
    lse = torch.full((S, hq, T), KEPT, device=DEV)
    got, got_lse = binding.reform_tree_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(lens), d ** -0.5,
                                              parent=None if chain else i32(parents), max_cache_len=max_len,
                                              node_count=None if counts is None else i32(counts), out=out, lse=lse)
    want, want_lse, a, err = ref.tree_attend(q, k, v, lens, None if chain else parents, used, d ** -0.5)
    for b in range(S):
        m = used[b]
        if m:
            ref.check_attention(got[b, :, :m], got_lse[b, :, :m], want[b, :, :m], want_lse[b, :, :m], a[b, :, :m], err[b, :, :m],
                                lens[b] + m, dtype, f"sequence {b}")
        assert bool((got[b, :, m:] == KEPT).all()) and bool((got_lse[b, :, m:] == KEPT).all()), b
    return got, got_lse


@pytest.mark.parametrize("hq,hkv,d,T,lens,dtype", [
    (4, 4, 64, 1, [0], BF),                                    # a first token sees itself
    (32, 8, 128, 1, [1, 31, 32, 33, 0, 300], BF),
    (8, 2, 128, 1, [5000, 3, 2000], BF),                       # shared out
    (8, 8, 64, 1, [4000], BF), (16, 1, 64, 1, [700, 90], BF),
    (8, 2, 64, 5, [100, 0, 1000, 31], BF),                     # 20 rows: two row blocks of a wave
    (8, 2, 128, 8, [3000, 17], BF), (4, 1, 128, 16, [257, 2000], BF),     # 64 rows
    (8, 2, 64, 17, [600, 1], BF), (12, 4, 128, 40, [900, 64, 0], BF),     # 68 and 120 rows
    (8, 2, 128, 64, [1000, 0, 63], BF), (4, 1, 64, 33, [2500], BF),       # 256 and 132 rows
    (16, 2, 128, 64, [700, 40], BF), (14, 2, 64, 50, [300], BF),          # 512 and 350 rows: two row blocks
    (8, 2, 64, 32, [3000, 0, 1500], BF), (8, 2, 128, 30, [2500], BF),     # the same blocks shared out
    (16, 2, 128, 64, [3000, 40], BF), (14, 2, 64, 50, [2000, 1999], BF),
    (4, 2, 128, 15, [2100, 5], BF), (6, 2, 64, 21, [1300], BF),
    (4, 4, 64, 1, [0, 500], F), (8, 2, 128, 7, [300, 20, 0], F), (6, 2, 36, 64, [90, 700], F),
    (2, 1, 256, 3, [1000, 5], F), (8, 1, 100, 20, [40], F),
])
def test_trees(hq, hkv, d, T, lens, dtype):
    run_case(hq, hkv, d, T, lens, dtype, seed=T + d + len(lens))


@pytest.mark.parametrize("T,d,dtype", [(1, 128, BF), (4, 64, BF), (64, 128, BF), (9, 64, F)])
def test_chains(T, d, dtype):
    run_case(8, 2, d, T, [333, 0, 65], dtype, seed=T, chain=True)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F, 64)])
def test_padded_batches(dtype, d):
    """Fewer nodes than room, none at all, counts outside; idle sequences beside long ones."""
    run_case(8, 2, d, 12, [50, 700, 0, 900, 33, 1500], dtype, seed=3, counts=[12, 5, 0, 99, -4, 1])
    run_case(4, 1, d, 3, [0, 10, 20], dtype, seed=4, counts=[0, 0, 0])


def test_many_sequences_and_shares_that_cross_them():
    """More sequences than a wave has lanes, lengths far apart: shares begin and end inside items."""
    rnd = random.Random(2)
    lens = [rnd.choice([0, 1, 64, rnd.randint(0, 90), rnd.randint(0, 1200)]) for _ in range(90)]
    run_case(4, 2, 64, 3, lens, BF, seed=7, counts=[rnd.randint(0, 3) for _ in lens])
    run_case(2, 1, 32, 2, lens[:70], F, seed=8)


def test_broken_parents_are_roots():
    T = 10
    parents = [[0, 1, 5, -3, 99, 2, 5, -(1 << 31), (1 << 31) - 1, 8]] * 2
    run_case(4, 2, 64, T, [40, 0], BF, seed=1, parents=parents)


def test_lengths_outside_are_moved_in():
    g = torch.Generator().manual_seed(3)
    q, k, v = ref.randn(g, 3, 4, 2, 64, dtype=BF), ref.randn(g, 3, 2, 50, 64, dtype=BF), ref.randn(g, 3, 2, 50, 64, dtype=BF)
    out, lse = binding.reform_tree_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32([-5, 1 << 30, 30]), 0.125, max_cache_len=40)
    want, wl, a, err = ref.tree_attend(q, k, v, [0, 40, 30], None, [2] * 3, 0.125)
    ref.check_attention(out, lse, want, wl, a, err, 42, BF)


def test_sharp_logits():
    run_case(8, 2, 128, 6, [2000, 100], BF, seed=5, sharp=15.0)
    run_case(8, 2, 64, 64, [900], BF, seed=5, sharp=15.0)
    run_case(4, 2, 64, 6, [300], F, seed=5, sharp=15.0)


def test_strides_and_shared_cache():
    """q and out node-major, caches with room between the heads, one cache that all sequences share (stride 0)."""
    S, hq, hkv, T, d, cap, L = 3, 4, 2, 5, 64, 90, 70
    g = torch.Generator().manual_seed(6)
    q = ref.randn(g, S, T, hq, d, dtype=BF)
    k, v = ref.randn(g, hkv, cap + 7, d, dtype=BF), ref.randn(g, hkv, cap + 7, d, dtype=BF)
    kd, vd = (x.to(DEV)[:, :cap].unsqueeze(0).expand(S, hkv, cap, d) for x in (k, v))
    out = torch.zeros((S, T, hq, d), dtype=BF, device=DEV).transpose(1, 2)
    got, lse = binding.reform_tree_attend(q.to(DEV).transpose(1, 2), kd, vd, i32([L] * S), 0.125, out=out)
    want, wl, a, err = ref.tree_attend(q.transpose(1, 2), k[None, :, :cap].expand(S, -1, -1, -1), v[None, :, :cap].expand(S, -1, -1, -1),
                                       [L] * S, None, [T] * S, 0.125)
    ref.check_attention(got, lse, want, wl, a, err, L + T, BF)


def test_long_cache_offsets_beyond_32_bits():
    """Two caches of 1.1 million rows, 8 heads each: 2.25 GB a cache, the second one beyond 2^31 elements' bytes.  Few keys matter: the
    rest are zero, so their logits are 0 and the result is known."""
    S, hkv, cap, d = 2, 8, 1100000, 128
    k = torch.zeros((S, hkv, cap, d), dtype=BF, device=DEV)
    v = torch.zeros((S, hkv, cap, d), dtype=BF, device=DEV)
    L = cap - 1
    q = torch.zeros((S, hkv, 1, d), dtype=BF, device=DEV)
    q[..., 0] = 16.0
    for b in range(S):
        for h in range(hkv):
            k[b, h, L - 5, 0] = 16.0                           # logit 16 * 16 * scale = 32
            v[b, h, L - 5] = float(b * hkv + h + 1)
    out, lse = binding.reform_tree_attend(q, k, v, i32([L] * S), 0.125)
    weight = math.exp(32.0) / (math.exp(32.0) + L)
    for b in range(S):
        for h in range(hkv):
            want = weight * (b * hkv + h + 1)
            assert float((out[b, h].double() - want).abs().max()) <= want * 2.0 ** -7
    assert float((lse.double() - math.log(math.exp(32.0) + L)).abs().max()) <= 1e-4


def test_workspace_is_needed_and_results_repeat():
    g = torch.Generator().manual_seed(7)
    S, hq, hkv, T, d, cap = 4, 8, 2, 3, 128, 3000
    q, k, v = ref.randn(g, S, hq, T, d, dtype=BF).to(DEV), ref.randn(g, S, hkv, cap, d, dtype=BF).to(DEV), ref.randn(g, S, hkv, cap, d, dtype=BF).to(DEV)
    lens = i32([2990, 100, 1500, 0])
    need = binding.tree_workspace_bytes(binding.tree_desc(q, k, v, q, 0.1))
    assert need > 0
    first = binding.reform_tree_attend(q, k, v, lens, 0.1)
    ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device=DEV)        # NaN everywhere: nothing stale is read
    again = binding.reform_tree_attend(q, k, v, lens, 0.1, workspace=ws)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    with pytest.raises(binding.ReformError, match="WORKSPACE"):
        binding.reform_tree_attend(q, k, v, lens, 0.1, workspace=ws[:need // 2])


@pytest.mark.parametrize("hq,hkv,d,T,n,dtype", [
    (4, 2, 64, 1, 300, BF), (8, 2, 128, 6, 280, BF), (8, 2, 64, 20, 270, BF),     # 2, 24 and 80 rows, 560 and more items
    (16, 2, 128, 40, 130, BF), (2, 2, 64, 3, 300, F),                             # 320 rows: two row blocks; fp32
])
def test_more_sequences_than_shares(hq, hkv, d, T, n, dtype):
    """More items than the caches are shared out to workgroups: most are finished by one, and those that a share's end
    cuts are put together; padded ones among them."""
    rnd = random.Random(n + T)
    lens = [rnd.choice([0, 1, 33, rnd.randint(0, 60), rnd.randint(0, 200)]) for _ in range(n)]
    lens[3], lens[n // 2], lens[-1] = 1500, 1100, 900
    counts = [rnd.choice([T, T, rnd.randint(0, T)]) for _ in lens]
    run_case(hq, hkv, d, T, lens, dtype, seed=n, counts=counts)


def test_many_short_caches():
    """One workgroup to a sequence and head, more sequences than a wave has lanes."""
    rnd = random.Random(5)
    lens = [rnd.choice([0, 1, 64, rnd.randint(0, 90)]) for _ in range(200)]
    run_case(4, 2, 64, 2, lens, BF, seed=5, counts=[rnd.randint(0, 2) for _ in lens])
    run_case(2, 2, 16, 2, lens, F, seed=5)


@pytest.mark.parametrize("hq,hkv,d,T,lens,block", [
    (4, 4, 128, 11, [3000, 0, 40], 16), (8, 2, 64, 4, [700, 3000, 1, 0], 16), (8, 2, 64, 7, [63, 2000, 500, 5], 32),
    (16, 4, 128, 8, [1, 2500], 32), (6, 2, 64, 11, [100, 0, 1000, 31], 64), (16, 4, 128, 16, [3000, 17], 64),
    (8, 2, 128, 9, [257, 2000, 3, 64], 64), (8, 8, 64, 64, [1300], 64), (8, 2, 64, 17, [600, 1, 64, 128], 128), (12, 4, 128, 40, [900, 64, 0], 128),
    (4, 2, 128, 64, [63, 1999, 0, 20], 128), (28, 4, 64, 10, [1, 300], 128), (8, 2, 128, 64, [1000, 0, 63, 65], 256),
    (16, 4, 64, 33, [2500, 0], 192), (16, 4, 128, 48, [3000, 64, 0], 192), (12, 4, 64, 64, [63, 1300], 192), (24, 8, 128, 43, [1, 2000], 192),
    (28, 4, 64, 50, [300, 1], 128), (32, 4, 128, 64, [700, 40], 256), (28, 4, 128, 23, [1, 3000], 256),
])
def test_every_form_shared_out(hq, hkv, d, T, lens, block):
    """Short caches in a large capacity, which is what the host chooses by: each form, with lengths where its tiles and shares end.  The
    workspace's size tells the rows of a block."""
    cap, rows, units = 40000, T * hq // hkv, torch.cuda.get_device_properties(0).multi_processor_count if torch.cuda.is_available() else 256
    side = -(-rows // block)
    shares = min((2 if block == 128 or (block <= 32 and d == 64) else 1) * units // side, 512)
    desc = binding.tree_desc(*(torch.empty(s, dtype=BF, device="meta") for s in
                               ((len(lens), hq, T, d), (len(lens), hkv, cap, d), (len(lens), hkv, cap, d), (len(lens), hq, T, d))), 0.1)
    assert binding.tree_workspace_bytes(desc) == 2 * shares * side * min(rows, block) * (4 * d + 8)
    run_case(hq, hkv, d, T, lens, BF, seed=block + T, spare=cap - max(lens) - T)
    run_case(hq, hkv, d, T, lens, BF, seed=block + T + 1, spare=cap - max(lens) - T, chain=True, counts=[max(T - 3 * i - 1, 0) for i in range(len(lens))])


@pytest.mark.parametrize("hq,hkv,d,T,n,top", [
    (8, 8, 64, 16, 60, 300), (8, 2, 128, 8, 250, 70), (16, 8, 64, 30, 80, 90), (8, 2, 128, 28, 200, 30), (16, 4, 64, 60, 130, 64),
    (16, 4, 128, 60, 110, 100), (21, 3, 64, 64, 100, 70), (12, 4, 128, 50, 120, 90), (16, 4, 64, 48, 130, 130),
])
def test_every_form_whole(hq, hkv, d, T, n, top):
    """Many short caches: one workgroup to each sequence, KV head and row block, in every form."""
    rnd = random.Random(T)
    lens = [rnd.choice([0, 1, top, rnd.randint(0, top)]) for _ in range(n)]
    q, kv = torch.empty((n, hq, T, d), dtype=BF, device="meta"), torch.empty((n, hkv, top + T, d), dtype=BF, device="meta")
    assert binding.tree_workspace_bytes(binding.tree_desc(q, kv, kv, q, 0.1)) == 0
    run_case(hq, hkv, d, T, lens, BF, seed=T + n, spare=0, counts=[rnd.choice([T, T, rnd.randint(0, T)]) for _ in lens])


def test_many_heads_of_one_group():
    """2560 rows of one KV head: up to 160 row blocks to a sequence."""
    run_case(64, 1, 64, 40, [500, 3], BF, seed=64)
    run_case(64, 1, 128, 40, [300], BF, seed=65, spare=40000)
    run_case(48, 1, 32, 9, [700, 0], F, seed=66)
