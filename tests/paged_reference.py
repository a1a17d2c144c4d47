"""Plain 64-bit implementations of the calls on sliding windows and on caches in pages, on the CPU, with the bounds of
serving_reference.py.  One more is needed, for the score: a probability is off by a factor of at most 1 + 2 E + (n + 8) 2^-24
(exponent, sum), and adding those of G heads, and what was there before, rounds G + 1 times:
   |d score| <= sum_h p_h (2 E_h + (n + 8) 2^-24) + (G + 1) 2^-24 |score|
Single tokens over pages take the probabilities of P.V in two bf16 parts, the second the rounded rest of the first: off by
u(bf16)^2 = 2^-16 of each at most, not by u(bf16).
"""
import math

import torch

from serving_reference import U24, half_step
from serving_checks import finite


def check_single(out, lse, want_out, want_lse, a, err, keys, dtype, what=""):
    """As serving_reference.check_attention, with the bound of probabilities in two parts, and every number required to be one."""
    out, lse, u = out.double().cpu(), lse.double().cpu(), half_step(dtype)
    for t, name in ((out, "outputs"), (want_out, "reference"), (a, "bound"), (err, "bound")):
        finite(t, f"{what} {name}")
    rel = 2 * err + (keys + 8) * U24 + (u * u if dtype == torch.bfloat16 else 0.0)
    bound = rel[..., None] * a * 1.01 + u * want_out.abs() * 1.01 + 1e-30
    bad = (out - want_out).abs() > bound
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} outputs off, worst {float(((out - want_out).abs() / bound).max()):.2f} of the bound"
    empty = want_lse == -math.inf
    finite(lse[~empty], f"{what} lse")
    assert bool((lse[empty] == -math.inf).all()), f"{what}: lse of rows that see nothing"
    bad = ((lse - want_lse).abs() > err + (keys + 8) * U24 + 4 * U24 * (want_lse.abs() + 1)) & ~empty
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} lse off"


def rows(q, k, v, scale, seen):
    """One head: q [m, d], k, v [n, d], seen [m, n].  out, lse, the bounds' A and E, and the probabilities."""
    q, k, v = q.double(), torch.where(seen.any(0)[:, None], k.double(), 0.0), torch.where(seen.any(0)[:, None], v.double(), 0.0)
    s = torch.where(seen, (q @ k.t()) * scale, -math.inf)
    lse = torch.logsumexp(s, -1) if s.shape[1] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    size = torch.where(seen, (q.abs() @ k.abs().t()) * scale, 0.0)
    top = size.amax(-1) if s.shape[1] else torch.zeros_like(lse)
    return p @ v, lse, p @ v.abs(), ((q.shape[1] + 4) * U24 + 2 * 3 * U24 * 1.4427) * top, p


def seen_by(nq, nk, window, n_sink):
    """[nq, nk] truth values of reform_window_attend."""
    t = torch.arange(nq)[:, None] + (nk - nq)
    j = torch.arange(nk)[None]
    return (j <= t) & ((j > t - window) | (j < n_sink))


def window_attend(q, k, v, q_lens, k_lens, scale, window, n_sink):
    """q [Hq, nq, d], k, v [Hkv, nk, d] packed.  out, lse, A, E for the rows of the sequences; NaN elsewhere."""
    hq, hkv = q.shape[0], k.shape[0]
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse = torch.full(q.shape[:2], math.nan, dtype=torch.float64)
    a, err = torch.full_like(out, math.nan), torch.full_like(lse, math.nan)
    i = j = 0
    for m, n in zip(q_lens, k_lens):
        seen = seen_by(m, n, window, n_sink)
        for h in range(hq):
            g = h * hkv // hq
            out[h, i:i + m], lse[h, i:i + m], a[h, i:i + m], err[h, i:i + m], _ = rows(q[h, i:i + m], k[g, j:j + n], v[g, j:j + n], scale, seen)
        i, j = i + m, j + n
    return out, lse, a, err


def gather(pool, table, n):
    """Rows of a sequence's first n keys [Hkv, n, d] from a pool [pages, Hkv, page_len, d], NaN where there is no such page; and
    which are there."""
    pages, hkv, page_len, d = pool.shape
    x = torch.full((hkv, n, d), math.nan, dtype=torch.float64)
    there = torch.zeros(n, dtype=torch.bool)
    for i in range(0, n, page_len):
        at, m = int(table[i // page_len]), min(page_len, n - i)
        if 0 <= at < pages:
            x[:, i:i + m] = pool[at, :, :m].double()
            there[i:i + m] = True
    return x, there


def paged_attend(q, k, v, table, lens, scale, window=0, n_sink=0):
    """q [S, Hq, d].  out, lse, A, E [S, Hq]; per sequence the score [Hkv, n], its bound without the final rounding, and which keys
    are seen."""
    S, hq, d = q.shape
    hkv = k.shape[1]
    G = hq // hkv
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.zeros((S, hq), dtype=torch.float64)
    a, err, scores = torch.zeros_like(out), torch.zeros_like(lse), []
    for b in range(S):
        n = lens[b]
        kk, there = gather(k, table[b], n)
        vv, _ = gather(v, table[b], n)
        j = torch.arange(n)
        seen = there & ((j >= n - window) | (j < n_sink)) if window else there
        score, off = torch.zeros((hkv, n), dtype=torch.float64), torch.zeros((hkv, n), dtype=torch.float64)
        for g in range(hkv):
            h = slice(g * G, (g + 1) * G)
            out[b, h], lse[b, h], a[b, h], err[b, h], p = rows(q[b, h], kk[g], vv[g], scale, seen[None].expand(G, n))
            score[g] = p.sum(0)
            off[g] = (p * (2 * err[b, h] + (n + 8) * U24)[:, None]).sum(0)
        scores.append((score, off, seen))
    return out, lse, a, err, scores


def evict(score, n, budget, n_sink, n_recent):
    """Kept keys of one head, ascending: exhaustive sort."""
    if n <= budget:
        return list(range(n))
    middle = sorted(range(n_sink, n - n_recent), key=lambda j: (-float(score[j]), j))[:budget - n_sink - n_recent]
    return list(range(n_sink)) + sorted(middle) + list(range(n - n_recent, n))


def make_table(rnd, lens, page_len, spare=2, columns=None):
    """Pages in no order, -1 behind a sequence's last one.  table [S][columns], pages of the pool."""
    need = [-(-n // page_len) for n in lens]
    order = list(range(sum(need) + spare))
    rnd.shuffle(order)
    columns = max(need + [1]) if columns is None else columns
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [-1] * (columns - n))
        at += n
    return table, len(order)
