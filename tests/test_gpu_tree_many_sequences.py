"""GPU: reform_tree_attend with hundreds to thousands of sequences whose caches are shared out: the search in the list of all sequences'
key tiles takes 64 of them, then 256 at a time, so the third step begins at sequence 320 and the fourth at 576.  Long caches and
sequences without nodes stand where these steps meet."""
import random

import pytest
import torch

import serving_checks
import serving_reference as ref
from paper_2506_01215_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KEPT = 5.0
BF, F = torch.bfloat16, torch.float32
CAP, APART = 20000, 37


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("hq,hkv,d,T,n,dtype,by_item", [
    (2, 1, 64, 2, 1500, BF, False), (4, 2, 128, 3, 700, BF, False), (4, 1, 64, 12, 650, BF, False), (8, 2, 64, 17, 700, BF, False),
    (16, 2, 128, 40, 600, BF, False), (2, 1, 32, 2, 1300, F, False),
    (2, 1, 64, 1, 500, BF, True), (4, 1, 32, 3, 450, F, True),               # no more items than shares: put together item by item
])
def test_lists_of_many_sequences(hq, hkv, d, T, n, dtype, by_item):
    rnd = random.Random(n + T)
    lens = [rnd.choice([0, 1, 33, rnd.randint(0, 60), rnd.randint(0, 120)]) for _ in range(n)]
    counts = [rnd.choice([T, T, rnd.randint(0, T)]) for _ in range(n)]
    for edge in (64, 320, 576, 832, 1088, n):                                # where steps of the search end
        for b, length, count in ((edge - 3, 700, T), (edge - 2, 5, 0), (edge - 1, 64, T), (edge, 3000, 0), (edge + 1, 900, T), (edge + 2, 31, 1)):
            if b < n:
                lens[b], counts[b] = length, count
    for b in (330, 400, n - 90, n - 1):
        lens[b], counts[b] = rnd.randint(2000, 3000), T
    # the caches are windows into one store, APART rows from one another: many, each of the capacity that the host chooses by
    rows = APART * (n - 1) + CAP
    g = torch.Generator().manual_seed(n)
    q = ref.randn(g, n, hq, T, d, dtype=dtype)
    store = [ref.randn(g, hkv, rows, d, dtype=dtype) for _ in range(2)]
    window = lambda x: x.as_strided((n, hkv, CAP, d), (APART * d, rows * d, d, 1))  # noqa: E731
    parents = [ref.random_parents(rnd, T) for _ in range(n)]
    dq, dk, dv = q.to(DEV), *(window(x.to(DEV)) for x in store)
    out = torch.full(q.shape, KEPT, dtype=dtype, device=DEV)
    lse = torch.full(q.shape[:3], KEPT, device=DEV)
    need = binding.tree_workspace_bytes(binding.tree_desc(dq, dk, dv, out, d ** -0.5))
    units = torch.cuda.get_device_properties(0).multi_processor_count
    assert need > 0 and by_item == (n * hkv <= 2 * units)
    print(f"[many] {hq}/{hkv} d={d} T={T} n={n} {dtype}", flush=True)
    ws = torch.full((need + 256,), 0xff, dtype=torch.uint8, device=DEV)       # NaN: nothing is read that was not written
    binding.reform_tree_attend(dq, dk, dv, i32(lens), d ** -0.5, parent=i32(parents), node_count=i32(counts), out=out, lse=lse, workspace=ws)
    want, want_lse, a, err = ref.tree_attend(q, window(store[0]), window(store[1]), lens, parents, counts, d ** -0.5)
    out, lse = out.cpu(), lse.cpu()
    for b in range(n):
        m = counts[b]
        if m:
            serving_checks.check_attention(out[b, :, :m], lse[b, :, :m], want[b, :, :m], want_lse[b, :, :m], a[b, :, :m], err[b, :, :m],
                                           lens[b] + m, dtype, f"sequence {b}")
        assert bool((out[b, :, m:] == KEPT).all()) and bool((lse[b, :, m:] == KEPT).all()), b
