"""GPU: reform_prompt_attend against the 64-bit definition: packed sequences of any lengths, one token to long ones,
keys before the first query row, rows that see nothing, odd heads, strides, values far apart."""
import math
import random

import pytest
import torch

import serving_reference as ref
from paper_2506_01215_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KEPT = 5.0           # what rows of no sequence hold before and after


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def starts(lens):
    got = [0]
    for n in lens:
        got.append(got[-1] + n)
    return got


def run_case(hq, hkv, d, q_lens, k_lens, dtype, seed, spare=0, layout="heads", sharp=1.0):
    g = torch.Generator().manual_seed(seed)
    nq, nk = sum(q_lens) + spare, sum(k_lens) + spare
    q, k, v = ref.randn(g, hq, nq, d), ref.randn(g, hkv, nk, d), ref.randn(g, hkv, nk, d)
    q, k, v = (q * sharp).to(dtype), k.to(dtype), v.to(dtype)
    scale = d ** -0.5
    print(f"[prompt] {hq}/{hkv} d={d} {dtype} q={q_lens[:8]} k={k_lens[:8]} spare={spare} {layout}", flush=True)
    if layout == "tokens":       # token-major, as a projection leaves them, with room between the rows
        put = lambda x: torch.cat([x, x], -1).transpose(0, 1).contiguous().to(DEV)[..., :d].transpose(0, 1)  # noqa: E731
    else:
        put = lambda x: x.to(DEV)  # noqa: E731
    qd, kd, vd = put(q), put(k), put(v)
    out = torch.full((nq, hq, d), KEPT, dtype=dtype, device=DEV).transpose(0, 1) if layout == "tokens" \
        else torch.full((hq, nq, d), KEPT, dtype=dtype, device=DEV)
    lse = torch.full((hq, nq), KEPT, device=DEV)
    same = list(q_lens) == list(k_lens)
    got, got_lse = binding.reform_prompt_attend(qd, kd, vd, i32(starts(q_lens)), scale, cu_k=None if same else i32(starts(k_lens)),
                                                out=out, lse=lse)
    want, want_lse, a, err = ref.prompt_attend(q, k, v, q_lens, k_lens, scale)
    rows = sum(q_lens)
    ref.check_attention(got[:, :rows], got_lse[:, :rows], want[:, :rows], want_lse[:, :rows], a[:, :rows], err[:, :rows],
                        max(k_lens), dtype, "prompt")
    if spare:
        assert bool((got[:, rows:] == KEPT).all()) and bool((got_lse[:, rows:] == KEPT).all())
    return got, got_lse


BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("hq,hkv,d,q_lens,dtype", [
    (1, 1, 64, [1], BF), (4, 4, 128, [1, 1, 1], BF), (8, 2, 64, [0, 5, 0, 1, 64, 0], BF),
    (8, 2, 128, [33, 31, 32, 64, 65, 63, 7], BF), (32, 8, 128, [130], BF), (14, 2, 64, [257, 3, 100], BF),
    (3, 1, 128, [300, 1, 77], BF), (24, 8, 64, [129, 64, 200], BF), (5, 5, 128, [500], BF), (16, 1, 64, [90, 91], BF),
    (1, 1, 64, [1], F), (4, 4, 64, [128, 301, 256], F), (6, 2, 128, [17, 0, 90], F), (2, 1, 256, [40, 3], F), (8, 2, 36, [50, 16], F),
    (3, 3, 100, [33], F), (4, 1, 4, [20], F), (2, 2, 200, [65], F),
])
def test_prompts(hq, hkv, d, q_lens, dtype):
    run_case(hq, hkv, d, q_lens, q_lens, dtype, seed=sum(q_lens) + d)


@pytest.mark.parametrize("hq,hkv,d,q_lens,k_lens,dtype", [
    (8, 2, 128, [1, 40, 64, 7], [300, 41, 64, 500], BF),
    (4, 2, 64, [100, 3], [164, 1000], BF),
    (8, 2, 128, [20, 70, 5, 30], [0, 30, 5, 1], BF),         # fewer keys than rows: the first rows see nothing
    (8, 4, 64, [300], [200], BF),
    (4, 2, 64, [20, 70, 5], [0, 30, 50], F),
    (2, 1, 96, [9, 1], [300, 77], F),
])
def test_keys_before_and_rows_without_keys(hq, hkv, d, q_lens, k_lens, dtype):
    run_case(hq, hkv, d, q_lens, k_lens, dtype, seed=d, spare=11)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    from test_prompt_plan import load_plan
    return load_plan(tmp_path_factory)


@pytest.mark.parametrize("d,hq,hkv,n,total,form", [
    (64, 2, 2, 3, 700, (16, 8)), (64, 7, 1, 1, 900, (32, 4)), (64, 24, 8, 5, 700, (128, 1)), (64, 6, 2, 9, 700, (32, 4)),
    (64, 12, 4, 40, 6000, (128, 1)), (64, 7, 7, 60, 9000, (128, 1)), (64, 8, 1, 1, 12000, (256, 1)), (64, 30, 2, 1, 12000, (256, 1)),
    (128, 6, 2, 7, 700, (32, 4)), (128, 3, 1, 1, 1000, (16, 8)), (128, 7, 1, 2, 3000, (32, 4)), (128, 16, 2, 4, 1200, (128, 2)),
    (128, 14, 2, 3, 3000, (128, 2)), (128, 12, 4, 40, 5000, (128, 1)), (128, 7, 7, 90, 7000, (128, 1)),
])
def test_every_form(plan, d, hq, hkv, n, total, form):
    """Ragged batches that take each of the forms (the plan's own header says so), with and without keys in front; the
    reference on three of the heads."""
    rnd = random.Random(total + d)
    cuts = sorted(rnd.sample(range(1, total), n - 1))
    lens = [b - a for a, b in zip([0] + cuts, cuts + [total])]
    assert plan(d, hq // hkv, hkv, n, total, total) == form
    g = torch.Generator().manual_seed(total)
    for front in (0, 37):
        k_lens = [x + front for x in lens]
        nk = sum(k_lens)
        if front and (total > 9000 or plan(d, hq // hkv, hkv, n, total, nk) != form):
            continue
        q = torch.randn((hq, total, d), generator=g).bfloat16()
        k, v = (torch.randn((hkv, nk, d), generator=g).bfloat16() for _ in range(2))
        print(f"[prompt form] {form} {hq}/{hkv} d={d} n={n} total={total} front={front}", flush=True)
        out, lse = binding.reform_prompt_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(starts(lens)), d ** -0.5,
                                                cu_k=i32(starts(k_lens)) if front else None)
        for h in sorted({0, hq // 2, hq - 1}):
            kv = slice(h * hkv // hq, h * hkv // hq + 1)
            want, wl, a, err = ref.prompt_attend(q[h:h + 1], k[kv], v[kv], lens, k_lens, d ** -0.5)
            ref.check_attention(out[h:h + 1], lse[h:h + 1], want, wl, a, err, max(k_lens), BF, f"head {h}")


def test_token_major_strides():
    run_case(8, 2, 128, [65, 3, 200], [65, 3, 200], BF, seed=1, layout="tokens")
    run_case(4, 1, 64, [1300, 1200], [1300, 1200], BF, seed=1, layout="tokens", spare=2)
    run_case(4, 2, 64, [65, 3], [65, 30], F, seed=2, layout="tokens", spare=5)


def test_sharp_logits_rescale():
    """Logits of some hundred: the reference maximum is outgrown again and again."""
    run_case(4, 2, 128, [400, 90], [400, 90], BF, seed=3, sharp=12.0)
    run_case(2, 1, 64, [3000], [3000], BF, seed=3, sharp=20.0)
    run_case(2, 1, 64, [300], [300], F, seed=3, sharp=12.0)


def test_more_sequences_than_a_wave_has_lanes():
    lens = [(i * 7) % 23 for i in range(150)]
    run_case(4, 2, 64, lens, lens, BF, seed=6)
    run_case(2, 1, 64, lens[:70], [n + 5 for n in lens[:70]], F, seed=6)


def test_boundaries_outside_are_moved_in():
    """Device-side boundaries that point outside the tensors, descend or overlap in the keys: nothing outside is
    touched, and what they mean after being moved in is computed."""
    g = torch.Generator().manual_seed(4)
    q, k, v = (ref.randn(g, 2, 100, 64, dtype=BF) for _ in range(3))
    cu = [-7, 30, 30, 20, 60, 1 << 30]
    out, lse = binding.reform_prompt_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(cu), 0.125, out=torch.full((2, 100, 64), KEPT, dtype=BF, device=DEV))
    # the sequences that remain: [0, 30), [20, 60), [60, 100); rows 20..30 belong to two of them, either result stands
    for lo, hi, own in ((0, 30, slice(0, 20)), (20, 60, slice(10, 40)), (60, 100, slice(0, 40))):
        want, wl, a, err = ref.prompt_attend(q[:, lo:hi], k[:, lo:hi], v[:, lo:hi], [hi - lo], [hi - lo], 0.125)
        ref.check_attention(out[:, lo:hi][:, own], lse[:, lo:hi][:, own], want[:, own], wl[:, own], a[:, own], err[:, own], 64, BF, f"{lo}")


def test_infinite_and_nan_keys_stay_in_their_sequence():
    """A sequence with broken values leaves its neighbours' results as they are, and so do rows of no sequence."""
    g = torch.Generator().manual_seed(12)
    lens = [40, 50, 64, 33]
    n = sum(lens) + 20
    for dtype in (BF, F):
        q, k, v = (ref.randn(g, 4, n, 64, dtype=dtype).to(DEV) for _ in range(3))
        cu = i32(starts(lens))
        clean = binding.reform_prompt_attend(q, k, v, cu, 0.125)
        k[:, 60], v[:, 61], q[:, 62] = math.nan, math.inf, math.nan
        k[:, sum(lens):], v[:, sum(lens):] = math.nan, math.nan
        dirty = binding.reform_prompt_attend(q, k, v, cu, 0.125)
        for x, y in zip(clean, dirty):
            assert torch.equal(x[:, :40], y[:, :40]) and torch.equal(x[:, 90:sum(lens)], y[:, 90:sum(lens)])
        assert bool(torch.isnan(dirty[0][:, 62]).all())


def test_same_results_as_the_single_sequence_call():
    """One sequence without a cache is what reform_chunk_attend_score computes; both round within the same bounds."""
    g = torch.Generator().manual_seed(2)
    q, k, v = ref.randn(g, 8, 700, 128, dtype=BF).to(DEV), ref.randn(g, 2, 700, 128, dtype=BF).to(DEV), ref.randn(g, 2, 700, 128, dtype=BF).to(DEV)
    out, lse = binding.reform_prompt_attend(q, k, v, i32([0, 700]), 128 ** -0.5)
    other, other_lse, _ = binding.reform_chunk_attend_score(q, k, v, 0, 128 ** -0.5, want_score=False)
    want, wl, a, err = ref.prompt_attend(q.cpu(), k.cpu(), v.cpu(), [700], [700], 128 ** -0.5)
    for o, e in ((out, lse), (other, other_lse)):
        ref.check_attention(o, e, want, wl, a, err, 700, BF)


def test_runs_are_bitwise_alike_and_lse_may_be_missing():
    import ctypes
    g = torch.Generator().manual_seed(21)
    q, k, v = ref.randn(g, 8, 3000, 64, dtype=BF).to(DEV), ref.randn(g, 2, 3000, 64, dtype=BF).to(DEV), ref.randn(g, 2, 3000, 64, dtype=BF).to(DEV)
    cu = i32([0, 1000, 1001, 2900])
    first = binding.reform_prompt_attend(q, k, v, cu, 0.125)
    again = binding.reform_prompt_attend(q, k, v, cu, 0.125)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    out = torch.zeros_like(q)
    desc = binding.prompt_desc(q, k, v, out, cu, 0.125)
    rc = binding.load_library().reform_prompt_attend(ctypes.byref(desc), q.data_ptr(), k.data_ptr(), v.data_ptr(), cu.data_ptr(), None,
                                                     out.data_ptr(), None, None, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(out, first[0])


@pytest.mark.parametrize("n,d,dtype", [(1025, 64, BF), (1500, 128, BF), (4500, 64, BF), (1100, 32, F)])
def test_sequences_that_are_searched(n, d, dtype):
    """More sequences than are counted one by one, and than one step of the search has lanes for; many of them empty, the first
    boundary behind rows of no sequence."""
    rnd = random.Random(n)
    lens = [rnd.choice([0, 0, 1, 2, rnd.randint(0, 9)]) for _ in range(n)]
    lens[n // 3], lens[-1] = 150, 70
    run_case(4, 2, d, lens, lens, dtype, seed=n, spare=5)
    q_lens = [9] + lens          # the first sequence is left out of the call: its rows keep what they held
    g = torch.Generator().manual_seed(n)
    q, k, v = (ref.randn(g, h, sum(q_lens), d, dtype=dtype) for h in (4, 2, 2))
    cu = i32(starts(q_lens)[1:])
    out = torch.full(q.shape, KEPT, dtype=dtype, device=DEV)
    got, lse = binding.reform_prompt_attend(q.to(DEV), k.to(DEV), v.to(DEV), cu, d ** -0.5, out=out)
    whole, whole_lse = binding.reform_prompt_attend(q.to(DEV)[:, 9:], k.to(DEV)[:, 9:], v.to(DEV)[:, 9:], i32(starts(lens)), d ** -0.5)
    assert torch.equal(got[:, 9:], whole) and torch.equal(lse[:, 9:], whole_lse) and bool((got[:, :9] == KEPT).all())


def test_descending_boundaries_of_many_sequences_touch_nothing_outside():
    """Where boundaries descend, it is open what rows are computed; the tensors' surroundings stay as they were, and so does the
    next call's result."""
    rnd = random.Random(9)
    g = torch.Generator().manual_seed(9)
    n, rows = 1400, 600
    cu = [rnd.choice([-5, 0, rows, 1 << 30, rnd.randint(0, rows)]) for _ in range(n + 1)]
    held = torch.full((4, rows + 200, 64), KEPT, dtype=BF, device=DEV)
    q, k, v = (ref.randn(g, h, rows, 64, dtype=BF).to(DEV) for h in (4, 2, 2))
    out = held[:, 100:100 + rows]
    binding.reform_prompt_attend(q, k, v, i32(cu), 0.125, out=out)
    assert bool((held[:, :100] == KEPT).all()) and bool((held[:, 100 + rows:] == KEPT).all())
    out, lse = binding.reform_prompt_attend(q, k, v, i32([0, rows]), 0.125)
    want, wl, a, err = ref.prompt_attend(q.cpu(), k.cpu(), v.cpu(), [rows], [rows], 0.125)
    ref.check_attention(out, lse, want, wl, a, err, rows, BF)


@pytest.mark.parametrize("hq,hkv,d,q_lens,k_lens,dtype", [
    (8, 2, 128, [3], [9000], BF), (4, 4, 128, [1, 0, 5, 2], [4000, 0, 3, 6001], BF), (16, 2, 128, [7, 1], [5000, 64], BF),
    (4, 4, 64, [1] * 3, [9000, 33, 8000], BF), (6, 2, 64, [9, 1, 30], [9000, 9000, 0], BF), (4, 1, 64, [40, 3], [9000, 2], BF),
    (8, 2, 128, [20, 6], [4, 7000], BF), (2, 1, 128, [1] * 30, [4000] * 29 + [5], BF),
    (4, 2, 64, [3, 0, 20], [3000, 5, 7], F), (2, 2, 128, [1, 2], [2500, 1], F), (8, 1, 36, [5], [6000], F), (4, 2, 200, [2, 9], [1200, 4], F),
])
def test_keys_shared_out(hq, hkv, d, q_lens, k_lens, dtype):
    """Few rows behind many keys: blocks that several workgroups go through, beside sequences without rows or keys and rows that see nothing."""
    q, kv = torch.empty((hq, sum(q_lens), d), dtype=dtype, device="meta"), torch.empty((hkv, sum(k_lens), d), dtype=dtype, device="meta")
    assert binding.prompt_workspace_bytes(binding.prompt_desc(q, kv, kv, q, torch.empty(len(q_lens) + 1), 0.1)) > 0
    got = run_case(hq, hkv, d, q_lens, k_lens, dtype, seed=sum(q_lens) + d, spare=3)
    again = run_case(hq, hkv, d, q_lens, k_lens, dtype, seed=sum(q_lens) + d, spare=3)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    run_case(hq, hkv, d, q_lens, k_lens, dtype, seed=d, layout="tokens", sharp=9.0)


def test_shared_out_boundaries_and_workspace():
    """Boundaries outside are moved in here as well; a workspace of NaN leaves no trace; one that is too small is refused."""
    g = torch.Generator().manual_seed(31)
    q, k, v = ref.randn(g, 4, 12, 128, dtype=BF).to(DEV), ref.randn(g, 2, 9000, 128, dtype=BF).to(DEV), ref.randn(g, 2, 9000, 128, dtype=BF).to(DEV)
    cu_q, cu_k = i32([-3, 4, 4, 2, 6, 1 << 30]), i32([-9, 5000, 70, 100, 8000, 1 << 30])
    need = binding.prompt_workspace_bytes(binding.prompt_desc(q, k, v, q, cu_q, 0.1))
    assert need > 0
    ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device=DEV)
    out, lse = binding.reform_prompt_attend(q, k, v, cu_q, 0.1, cu_k=cu_k, workspace=ws)
    # [0, 4) over keys [0, 5000), [2, 6) over [100, 8000), [6, 12) over [8000, 9000); rows 2 and 3 belong to two
    for lo, hi, k0, k1, own in ((0, 4, 0, 5000, slice(0, 2)), (2, 6, 100, 8000, slice(2, 4)), (6, 12, 8000, 9000, slice(0, 6))):
        want, wl, a, err = ref.prompt_attend(q[:, lo:hi].cpu(), k[:, k0:k1].cpu(), v[:, k0:k1].cpu(), [hi - lo], [k1 - k0], 0.1)
        ref.check_attention(out[:, lo:hi][:, own], lse[:, lo:hi][:, own], want[:, own], wl[:, own], a[:, own], err[:, own], k1 - k0, BF, f"{lo}")
    with pytest.raises(binding.ReformError, match="WORKSPACE"):
        binding.reform_prompt_attend(q, k, v, cu_q, 0.1, cu_k=cu_k, workspace=ws[:need // 2])
    # a broken sequence leaves its neighbours as they are
    k[:, 20], v[:, 30] = math.nan, math.inf
    dirty = binding.reform_prompt_attend(q, k, v, cu_q, 0.1, cu_k=cu_k, workspace=ws)
    assert torch.equal(dirty[0][:, 4:], out[:, 4:]) and torch.equal(dirty[1][:, 4:], lse[:, 4:]) and bool(torch.isnan(dirty[0][:, :2]).all())


def test_many_heads_of_one_group():
    run_case(64, 1, 64, [70, 3, 0, 1], [70, 3, 0, 1], BF, seed=64)
    run_case(64, 1, 128, [2, 1], [5000, 9000], BF, seed=65)
    run_case(48, 1, 32, [9, 20], [9, 1700], F, seed=66)


def test_shared_out_calls_replay_from_a_graph():
    """Captured with its workspace, replayed on new lengths with eager calls of the same workspace in between."""
    g = torch.Generator().manual_seed(77)
    q, k, v = (ref.randn(g, h, n, 128, dtype=BF).to(DEV) for h, n in ((8, 20), (2, 12000), (2, 12000)))
    cu_q, cu_k = i32([0, 4, 20]), i32([0, 5000, 12000])
    out, lse = torch.zeros_like(q), torch.zeros((8, 20), device=DEV)
    need = binding.prompt_workspace_bytes(binding.prompt_desc(q, k, v, out, cu_q, 0.1))
    assert need > 0
    ws = torch.empty(need + 256, dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.reform_prompt_attend(q, k, v, cu_q, 0.1, cu_k=cu_k, out=out, lse=lse, workspace=ws)
    for cuts, ends in (([0, 4, 20], [0, 5000, 12000]), ([0, 19, 20], [0, 30, 12000]), ([0, 0, 20], [0, 11000, 11900]), ([0, 4, 20], [0, 5000, 12000])):
        cu_q.copy_(torch.tensor(cuts))
        cu_k.copy_(torch.tensor(ends))
        graph.replay()
        got = out.clone(), lse.clone()
        eager = binding.reform_prompt_attend(q, k, v, cu_q, 0.1, cu_k=cu_k, workspace=ws)
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])


@pytest.mark.parametrize("hq,hkv,d,q_lens,k_lens,block", [
    (8, 2, 128, [3, 40], [9000, 70], 16), (32, 8, 128, [6, 5, 7, 6], [5000, 4000, 6000, 5200], 32), (32, 8, 128, [16], [11000], 64),
    (32, 8, 128, [30, 3, 0, 31], [8000, 5, 9000, 15000], 128), (32, 8, 64, [6, 5, 7, 6], [6500, 64, 13000, 6500], 32),
    (32, 8, 64, [12, 10, 14, 12], [7000, 7000, 7000, 7031], 64), (16, 4, 64, [30, 20], [32001, 33000], 128),
])
def test_every_shared_form(hq, hkv, d, q_lens, k_lens, block):
    """Blocks of each size, by the workspace's; lengths that differ, tiles that end inside a share, rows that see nothing."""
    q, kv = torch.empty((hq, sum(q_lens), d), dtype=BF, device="meta"), torch.empty((hkv, sum(k_lens), d), dtype=BF, device="meta")
    units = torch.cuda.get_device_properties(0).multi_processor_count if torch.cuda.is_available() else 256
    shares = min((2 if block == 128 or (d == 64 and block <= 32) else 1) * units, 512)
    need = binding.prompt_workspace_bytes(binding.prompt_desc(q, kv, kv, q, torch.empty(len(q_lens) + 1), 0.1))
    assert need == 2 * shares * min(block, sum(q_lens) * hq // hkv) * (4 * d + 8)
    run_case(hq, hkv, d, q_lens, k_lens, BF, seed=block + d, spare=2)
    run_case(hq, hkv, d, q_lens, k_lens, BF, seed=block + d + 1, layout="tokens", sharp=9.0)
