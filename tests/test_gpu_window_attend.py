"""GPU: reform_window_attend against the 64-bit definition: windows of one key to more than there are, first keys inside, outside
and beyond the window, prompts behind keys, boundaries on the device, strides, graphs."""
import math
import random

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


def starts(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def run_case(hq, hkv, d, q_lens, k_lens, window, sinks, dtype, seed, spare=3, sharp=1.0):
    g = torch.Generator().manual_seed(seed)
    nq, nk = sum(q_lens) + spare, sum(k_lens) + spare
    q = (sref.randn(g, hq, nq, d) * sharp).to(dtype)
    k, v = (sref.randn(g, hkv, nk, d, dtype=dtype) for _ in range(2))
    k[:, nk - spare:], v[:, nk - spare:] = math.nan, math.nan            # rows of no sequence are never looked at
    print(f"[window] {hq}/{hkv} d={d} {dtype} q={q_lens[:6]} k={k_lens[:6]} window={window} sinks={sinks}", flush=True)
    out, lse = torch.full((hq, nq, d), KEPT, dtype=dtype, device=DEV), torch.full((hq, nq), KEPT, device=DEV)
    got, got_lse = binding.reform_window_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(starts(q_lens)), d ** -0.5, window, n_sink=sinks,
                                                cu_k=i32(starts(k_lens)), out=out, lse=lse)
    want, want_lse, a, err = ref.window_attend(q, k, v, q_lens, k_lens, d ** -0.5, window, sinks)
    m = sum(q_lens)
    check_attention(got[:, :m], got_lse[:, :m], want[:, :m], want_lse[:, :m], a[:, :m], err[:, :m], min(max(k_lens), window + sinks), dtype)
    assert bool((got[:, m:] == KEPT).all()) and bool((got_lse[:, m:] == KEPT).all())
    return got, got_lse


@pytest.mark.parametrize("hq,hkv,d,lens,dtype", [
    (4, 4, 64, [1], BF), (8, 2, 128, [1, 31, 33, 200], BF), (24, 8, 64, [17, 129, 300, 1], BF), (4, 1, 128, [700], BF),
    (14, 2, 64, [257, 64], BF), (16, 1, 128, [90], BF), (2, 2, 128, [1100, 30], BF), (3, 1, 64, [500], BF),
    (4, 4, 64, [128, 70, 1], F), (6, 2, 36, [90], F), (2, 1, 256, [70, 33], F), (8, 1, 100, [40], F), (3, 3, 128, [65], F),
])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (64, 0), (64, 64), (100, 7), (129, 130), (4000, 4)])
def test_windows(hq, hkv, d, lens, dtype, window, sinks):
    run_case(hq, hkv, d, lens, lens, window, sinks, dtype, seed=window + sinks + d)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 4), (256, 70), (1000, 300)])
def test_prompts_behind_keys(dtype, d, window, sinks):
    """Keys in front of the first row, none at all, fewer keys than rows: then the first rows see none."""
    run_case(8, 2, d, [5, 200, 1, 40, 3, 20], [905, 700, 1, 0, 300, 11], window, sinks, dtype, seed=window)


@pytest.mark.parametrize("hq,hkv,d,n,window,sinks", [(8, 2, 128, 2100, 300, 100), (4, 4, 64, 3000, 1024, 0), (32, 8, 128, 700, 200, 256),
                                                     (8, 8, 128, 1500, 64, 4), (16, 2, 64, 900, 511, 65)])
def test_one_long_prompt(hq, hkv, d, n, window, sinks):
    run_case(hq, hkv, d, [n], [n], window, sinks, BF, seed=n)


@pytest.mark.parametrize("hq,hkv,d,lens,window,sinks", [
    # a size of every form: 128, 32 and 16 rows at head_dim 64; 128, 128 by two groups, 32 and 16 at 128 (test_window_plan.py)
    (32, 8, 64, [1200], 300, 0), (16, 2, 64, [900], 511, 65), (8, 2, 64, [100], 7, 2), (8, 2, 128, [2100], 300, 100), (32, 8, 128, [700], 200, 256),
    (2, 1, 128, [6164], 12, 64), (16, 2, 128, [700, 600, 500], 833, 5), (16, 2, 128, [70, 66, 65, 65], 8, 64),
    (8, 2, 128, [60], 33, 5)])
def test_every_form(hq, hkv, d, lens, window, sinks):
    run_case(hq, hkv, d, lens, lens, window, sinks, BF, seed=sum(lens))


@pytest.mark.parametrize("d,rows,keys,window,sinks", [(128, 3, 9000, 8000, 4), (64, 1, 12000, 11000, 300), (128, 20, 5000, 4000, 64)])
def test_few_rows_behind_many_keys(d, rows, keys, window, sinks):
    run_case(8, 2, d, [rows, 1], [keys, keys - 77], window, sinks, BF, seed=rows)


def test_many_sequences():
    rnd = random.Random(3)
    lens = [rnd.choice([0, 1, 7, 33]) for _ in range(90)]
    run_case(4, 2, 64, lens, lens, 9, 2, BF, seed=1)
    run_case(2, 1, 32, lens, lens, 9, 2, F, seed=2)
    lens = [rnd.choice([0, 1, 2]) for _ in range(1100)]
    run_case(2, 1, 64, lens, lens, 2, 1, BF, seed=3)


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_wide_window_is_causal_attention(dtype):
    g = torch.Generator().manual_seed(4)
    q, k, v = (sref.randn(g, h, 333, 64, dtype=dtype).to(DEV) for h in (8, 2, 2))
    cu = i32([0, 200, 333])
    want, want_lse = binding.reform_prompt_attend(q, k, v, cu, 0.125)
    for window, sinks in ((200, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 200), (100, 100)):
        out, lse = binding.reform_window_attend(q, k, v, cu, 0.125, window, n_sink=sinks)
        # the same terms in another order: rounding of the result and of the probabilities
        tol = 4 * sref.half_step(dtype) if dtype == BF else 1e-5
        torch.testing.assert_close(out.float(), want.float(), rtol=tol, atol=tol)
        torch.testing.assert_close(lse, want_lse, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("dtype", [BF, F])
def test_first_keys_weigh_as_they_should(dtype):
    """All logits alike: the output is the mean of the seen values, which a key seen twice or not at all would shift."""
    n, d, window, sinks = 150, 64, 32, 10
    q = torch.zeros(1, n, d, dtype=dtype, device=DEV)
    k = torch.randn(1, n, d, device=DEV).to(dtype)
    v = torch.zeros(1, n, d, dtype=dtype, device=DEV)
    v[0, :, 0] = torch.arange(n, device=DEV).to(dtype)
    v[0, :, 1] = 1.0
    out, lse = binding.reform_window_attend(q, k, v, i32([0, n]), 0.125, window, n_sink=sinks)
    seen = ref.seen_by(n, n, window, sinks).double()
    want = (seen * v[0, :, 0].cpu().double()).sum(1) / seen.sum(1)
    u = sref.half_step(dtype)
    assert bool(((out[0, :, 0].cpu().double() - want).abs() <= u * want + 200 * sref.U24 * 150 + 1e-6).all())
    assert bool(((out[0, :, 1].cpu().double() - 1).abs() <= u + 200 * sref.U24).all())
    assert bool(((lse[0].cpu().double() - seen.sum(1).log()).abs() <= 200 * sref.U24 + 1e-6).all())


def test_sharp_logits():
    run_case(8, 2, 128, [400, 33], [500, 33], 50, 10, BF, seed=5, sharp=15.0)
    run_case(4, 2, 64, [300], [300], 50, 10, F, seed=5, sharp=15.0)


@pytest.mark.parametrize("dtype", [BF, F])
def test_strides(dtype):
    """Token-major tensors, keys and values side by side in one."""
    hq, hkv, d, lens = 6, 2, 64, [40, 61]
    n = sum(lens)
    g = torch.Generator().manual_seed(6)
    qkv = sref.randn(g, n, hq + 2 * hkv, d, dtype=dtype)
    x = qkv.to(DEV).transpose(0, 1)
    out = torch.zeros(n, hq, d, dtype=dtype, device=DEV).transpose(0, 1)
    got, lse = binding.reform_window_attend(x[:hq], x[hq:hq + hkv], x[hq + hkv:], i32(starts(lens)), 0.125, 17, n_sink=3, out=out)
    y = qkv.transpose(0, 1)
    want, wl, a, err = ref.window_attend(y[:hq], y[hq:hq + hkv], y[hq + hkv:], lens, lens, 0.125, 17, 3)
    check_attention(got, lse, want, wl, a, err, 20, dtype)


@pytest.mark.parametrize("dtype", [BF, F])
def test_broken_boundaries_touch_nothing(dtype):
    """Boundaries outside, descending: nothing outside the tensors is read or written, and all ends."""
    g = torch.Generator().manual_seed(7)
    q, k, v = (sref.randn(g, h, 100, 64, dtype=dtype).to(DEV) for h in (4, 2, 2))
    for cu_q, cu_k in (([0, 40, 20, 100], [0, 40, 60, 100]), ([-5, 50, 1 << 30, 60], [90, 10, 200, -7]), ([100, 0, 100, 0], [0, 100, 0, 100])):
        binding.reform_window_attend(q, k, v, i32(cu_q), 0.125, 7, n_sink=2, cu_k=i32(cu_k))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F])
def test_values_that_are_not_finite_stay_in_their_sequence(dtype):
    lens = [70, 90, 40]
    g = torch.Generator().manual_seed(8)
    q, k, v = (sref.randn(g, h, 200, 64, dtype=dtype) for h in (4, 2, 2))
    clean = binding.reform_window_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(starts(lens)), 0.125, 20, n_sink=4)
    k[:, 75], v[:, 80] = math.nan, math.inf
    got = binding.reform_window_attend(q.to(DEV), k.to(DEV), v.to(DEV), i32(starts(lens)), 0.125, 20, n_sink=4)
    for x, y in zip(got, clean):
        assert torch.equal(x[:, :70], y[:, :70]) and torch.equal(x[:, 160:], y[:, 160:])
    assert bool(torch.isnan(got[0][:, 75]).all())


def test_graph_follows_the_lengths():
    g = torch.Generator().manual_seed(9)
    q, k, v = (sref.randn(g, h, 500, 128, dtype=BF).to(DEV) for h in (8, 2, 2))
    cu = i32([0, 100, 500])
    out, lse = torch.zeros_like(q), torch.zeros(8, 500, device=DEV)
    ws = torch.empty(binding.window_workspace_bytes(binding.window_desc(q, k, v, out, cu, 0.1, 33, 5)) + 256, dtype=torch.uint8, device=DEV)
    call = lambda: binding.reform_window_attend(q, k, v, cu, 0.1, 33, n_sink=5, out=out, lse=lse, workspace=ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens in ([100, 400], [499, 1], [0, 500], [250, 250]):
        cu.copy_(i32(starts(lens)))
        q.copy_(torch.randn(q.shape, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        want = binding.reform_window_attend(q, k, v, cu, 0.1, 33, n_sink=5)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_another_stream():
    g = torch.Generator().manual_seed(10)
    q, k, v = (sref.randn(g, h, 300, 64, dtype=BF).to(DEV) for h in (4, 2, 2))
    cu = i32([0, 300])
    want = binding.reform_window_attend(q, k, v, cu, 0.125, 64)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = binding.reform_window_attend(q, k, v, cu, 0.125, 64, stream=st)
    st.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("hq,hkv,d,lens,dtype", [(8, 2, 64, [700, 650], BF), (8, 2, 64, [230], BF), (8, 1, 64, [60, 100], BF), (8, 2, 128, [720, 500], BF),
                                                 (2, 1, 128, [2300], BF), (4, 4, 128, [190], BF), (4, 2, 64, [170], F), (2, 1, 200, [150], F)])
@pytest.mark.parametrize("window", [1, 30, 64, 70])
def test_tiles_of_first_keys_and_window(hq, hkv, d, lens, dtype, window):
    """The first keys end anywhere inside a tile, whose other keys are the window's: next to them, a tile away, or further."""
    for sinks in (1, 15, 16, 17, 31, 33, 63, 65, 100):
        run_case(hq, hkv, d, lens, [n + (0 if sinks % 2 else 37) for n in lens], window, sinks, dtype, seed=sinks)


def test_two_groups_of_waves_and_first_keys_inside_a_tile():
    for sinks in (1, 33, 63, 70, 130):
        run_case(2, 1, 128, [6164], [6164], 12, sinks, BF, seed=sinks)
        run_case(16, 2, 128, [700, 600, 500], [700, 600, 500], 833, sinks, BF, seed=sinks)
