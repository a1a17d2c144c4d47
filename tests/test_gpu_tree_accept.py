"""GPU: reform_tree_accept against the walk written out, exact: paths, tokens, lengths, and the caches with every
row where it belongs."""
import random

import pytest
import torch

import serving_reference as ref
from paper_2506_01215_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def run_case(S, T, hkv, cap, d, dtype, layers, chain, vocab, seed, counts=None, lens=None):
    rnd = random.Random(seed)
    shape = (layers, S, hkv, cap, d) if layers else (S, hkv, cap, d)
    g = torch.Generator().manual_seed(seed)
    k, v = ref.randn(g, *shape, dtype=dtype), ref.randn(g, *shape, dtype=dtype)
    parent = None if chain else [ref.random_parents(rnd, T) for _ in range(S)]
    drafted, target = ([[rnd.randrange(vocab) for _ in range(T)] for _ in range(S)] for _ in range(2))
    lens = [rnd.randint(0, cap - T) for _ in range(S)] if lens is None else lens
    kd, vd = k.to(DEV), v.to(DEV)
    print(f"[accept] S={S} T={T} hkv={hkv} cap={cap} d={d} {dtype} layers={layers} chain={chain}", flush=True)
    path, accepted, nxt, new_len = binding.reform_tree_accept(
        None if chain else i32(parent), i32(drafted), i32(target), i32(lens), kd, vd,
        node_count=None if counts is None else i32(counts))
    wk, wv = k.clone(), v.clone()
    for b in range(S):
        m = T if counts is None else min(max(counts[b], 0), T)
        if not 0 <= lens[b] <= cap - m:
            m = 0
        want, token = ref.accept(None if chain else parent[b], drafted[b], target[b], m)
        assert path[b].tolist() == want + [-1] * (T - len(want)), b
        assert (int(accepted[b]), int(nxt[b]), int(new_len[b])) == (len(want), token, lens[b] + len(want)), b
        for x in (wk, wv):
            rows = x[..., b, :, :, :] if layers else x[b]
            rows[..., lens[b]:lens[b] + len(want), :] = rows[..., [lens[b] + i for i in want], :].clone()
    assert torch.equal(kd.cpu(), wk) and torch.equal(vd.cpu(), wv)
    return accepted.tolist()


@pytest.mark.parametrize("S,T,hkv,cap,d,dtype,layers,chain,vocab", [
    (1, 1, 1, 1, 64, torch.bfloat16, 0, True, 2),          # one token: nothing to move
    (5, 7, 2, 40, 64, torch.bfloat16, 0, False, 2),
    (3, 64, 8, 200, 128, torch.bfloat16, 0, False, 2),
    (3, 64, 2, 64, 256, torch.float32, 2, False, 1),       # every token fits: the longest paths, two layers
    (2, 64, 1, 100, 1024, torch.float32, 0, False, 1),     # 4 KB rows: several passes of the workgroup
    (2, 33, 3, 90, 24, torch.bfloat16, 3, True, 3),        # 48-byte rows
    (70, 16, 4, 50, 128, torch.bfloat16, 0, False, 3),
    (4, 50, 1, 60, 8, torch.bfloat16, 0, True, 1),         # a chain that is accepted whole
])
def test_matches_the_walk(S, T, hkv, cap, d, dtype, layers, chain, vocab):
    got = run_case(S, T, hkv, cap, d, dtype, layers, chain, vocab, seed=S + T)
    if vocab == 1 and chain:
        assert got == [T] * S


def test_padded_batches_and_lengths_outside():
    """Sequences without nodes, with fewer, with counts and lengths that are out of range."""
    run_case(7, 12, 2, 40, 64, torch.bfloat16, 0, False, 2, seed=4, counts=[0, 3, 12, 99, -5, 1, 12], lens=[5, 37, 28, 0, 3, 39, 29])
    run_case(3, 4, 2, 10, 64, torch.float32, 0, True, 1, seed=5, lens=[-1, 1 << 30, 6])


def test_broken_parents_end_the_path():
    """Parents that do not lie before their node are children of nothing; the first of two equal children wins."""
    parent = i32([[-1, 1, 0, 0, 7, -9, 3, 2]])
    drafted = i32([[0, 5, 5, 5, 5, 5, 5, 5]])
    target = i32([[5] * 8])
    path, accepted, nxt, new_len = binding.reform_tree_accept(parent, drafted, target, i32([3]))
    assert path.tolist() == [[0, 2, 7] + [-1] * 5]
    assert accepted.tolist() == [3] and nxt.tolist() == [5] and new_len.tolist() == [6]


def test_strided_caches_keep_their_neighbours():
    """Caches that are part of a larger tensor: rows of other heads, sequences and layers stay."""
    S, hkv, cap, d, T = 3, 2, 20, 64, 6
    g = torch.Generator().manual_seed(1)
    big = ref.randn(g, 2, S + 1, hkv + 1, cap, d, dtype=torch.bfloat16)
    dev = big.to(DEV)
    k, v = dev[0, :S, :hkv], dev[1, :S, :hkv]
    parent = i32([[-1, 0, 0, 2, 2, 4]] * S)
    drafted, target = i32([[9, 1, 2, 3, 4, 5]] * S), i32([[2, 0, 4, 0, 5, 8]] * S)
    lens = [0, 7, 14]
    path, *_ = binding.reform_tree_accept(parent, drafted, target, i32(lens), k, v)
    assert path.tolist() == [[0, 2, 4, 5, -1, -1]] * S
    for b in range(S):
        rows = big[:, b, :hkv, [lens[b] + i for i in (0, 2, 4, 5)]].clone()
        big[:, b, :hkv, lens[b]:lens[b] + 4] = rows
    assert torch.equal(dev.cpu(), big)
