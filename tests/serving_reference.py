"""Plain 64-bit implementations of the serving calls, on the CPU, and the error bounds their tests use.

Bounds.  u(t) = torch.finfo(t).eps / 2 is the largest relative error of one rounding to t.
  attention: logits are sums of d products formed in 32 bits, |ds| <= E = (d + 4) 2^-24 scale sum |q||k| (the
    largest over a row's keys), so a probability is off by a factor of at most about exp(2 E), and a sum over n
    keys in any order by (n + 8) 2^-24 more.  bf16 rounds the probabilities of P.V (u(bf16) of each) and the
    result (u(bf16) of it).  With A = sum_j p_j |v_j|:
       |d out| <= (2 E + (n + 8) 2^-24 [+ u(bf16)]) A + u |out|,   |d lse| <= E + (n + 8) 2^-24 + 4 * 2^-24 (|lse| + 1)
    Exponentials are formed as exp2(s c - m c) with c = scale log2 e rounded and v_exp_f32 within 2^-23: the exponent's
    error, 3 * 2^-24 (|s| + |m|) log2 e, joins E.
  rotary: sine and cosine are within 2^-23 of exact ones and products and sums of two terms are rounded in 32 bits:
       |dy| <= 4 * 2^-23 magnitude (|x| + |x'|) + u |y|
"""
import math

import torch

U24 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def randn(gen, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen).to(dtype)


def softmax_rows(q, k, v, scale, seen):
    """One head: q [m, d], k, v [n, d], seen [m, n] truth values.  Returns out, lse and the bounds' A and E (per row)."""
    q, k, v = q.double(), k.double(), v.double()
    s = (q @ k.t()) * scale
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, -1) if s.shape[1] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    p = torch.exp(s - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[:, None])
    size = (q.abs() @ k.abs().t()) * scale
    big = torch.where(seen, size, torch.zeros_like(size))
    top = big.amax(-1) if s.shape[1] else torch.zeros_like(lse)
    err = ((q.shape[1] + 4) * U24 + 2 * 3 * U24 * 1.4427) * top
    return p @ v, lse, p @ v.abs(), err


def check_attention(out, lse, want_out, want_lse, a, err, keys, dtype, what=""):
    """out [.., d], lse [..] against the reference with the bounds above; keys: keys of a row (an upper bound)."""
    out, lse = out.double().cpu(), lse.double().cpu()
    u = half_step(dtype)
    rel = 2 * err + (keys + 8) * U24 + (u if dtype == torch.bfloat16 else 0.0)
    bound = rel[..., None] * a * 1.01 + u * want_out.abs() * 1.01 + 1e-30
    bad = (out - want_out).abs() > bound
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} outputs off, worst " \
        f"{float(((out - want_out).abs() / bound).max()):.2f} of the bound"
    assert bool(torch.isfinite(out).all())
    empty = want_lse == -math.inf
    assert bool((lse[empty] == -math.inf).all()), f"{what}: lse of rows that see nothing"
    lb = err + (keys + 8) * U24 + 4 * U24 * (want_lse.abs() + 1)
    bad = ((lse - want_lse).abs() > lb) & ~empty
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} lse off"


def prompt_attend(q, k, v, q_lens, k_lens, scale):
    """q [Hq, nq, d], k, v [Hkv, nk, d] packed.  out, lse, A, E for the rows of the sequences; NaN elsewhere."""
    hq, hkv = q.shape[0], k.shape[0]
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse = torch.full(q.shape[:2], math.nan, dtype=torch.float64)
    a, err = torch.full_like(out, math.nan), torch.full_like(lse, math.nan)
    i = j = 0
    for m, n in zip(q_lens, k_lens):
        seen = torch.arange(n)[None] <= torch.arange(m)[:, None] + (n - m)
        for h in range(hq):
            g = h * hkv // hq
            r = softmax_rows(q[h, i:i + m], k[g, j:j + n], v[g, j:j + n], scale, seen)
            out[h, i:i + m], lse[h, i:i + m], a[h, i:i + m], err[h, i:i + m] = r
        i, j = i + m, j + n
    return out, lse, a, err


def line_of(parent, i):
    """Node i and its ancestors; a parent that does not lie before its node is none."""
    got = [i]
    while True:
        up = i - 1 if parent is None else int(parent[i])
        if not 0 <= up < i:
            return got
        got.append(up)
        i = up


def tree_attend(q, k, v, lens, parents, counts, scale):
    """q [S, Hq, T, d], k, v [S, Hkv, cap, d]; parents [S][T] or None.  NaN for rows that are not computed."""
    s_, hq, t, _ = q.shape
    hkv = k.shape[1]
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse = torch.full(q.shape[:3], math.nan, dtype=torch.float64)
    a, err = torch.full_like(out, math.nan), torch.full_like(lse, math.nan)
    for b in range(s_):
        n, m = lens[b], counts[b]
        seen = torch.zeros((m, n + m), dtype=torch.bool)
        seen[:, :n] = True
        for i in range(m):
            for j in line_of(None if parents is None else parents[b], i):
                seen[i, n + j] = True
        for h in range(hq):
            g = h * hkv // hq
            r = softmax_rows(q[b, h, :m], k[b, g, :n + m], v[b, g, :n + m], scale, seen)
            out[b, h, :m], lse[b, h, :m], a[b, h, :m], err[b, h, :m] = r
    return out, lse, a, err


def frequencies(rot, theta, scaling=None, factor=1.0, original_len=0, turns_high=32.0, turns_low=1.0):
    """Radians per position of every pair, from the definitions one pair at a time."""
    f = []
    for c in range(rot // 2):
        w = theta ** (-2.0 * c / rot)
        if scaling == "linear":
            w /= factor
        elif scaling == "base":
            w = (theta * factor ** (rot / (rot - 2.0))) ** (-2.0 * c / rot)
        elif scaling == "parts":
            at = [rot * math.log(original_len / (2 * math.pi * t)) / (2 * math.log(theta)) for t in (turns_high, turns_low)]
            lo, hi = (min(max(x, 0), rot - 1) for x in (math.floor(at[0]), math.ceil(at[1])))
            r = min(max((c - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            w = w * (1 - r) + w / factor * r
        elif scaling == "bands":
            turns = original_len * w / (2 * math.pi)
            r = 1.0 - min(max((turns - turns_low) / (turns_high - turns_low), 0.0), 1.0)
            w = w * (1 - r) + w / factor * r
        f.append(w)
    return torch.tensor(f, dtype=torch.float64)


def rotary(x, pos, rot, freq, adjacent=False, inverse=False, magnitude=1.0):
    """x [H, n, d].  Returns y and |x| + |x'| (0 behind the rotated part), 64 bits."""
    x = x.double()
    a = pos.double()[:, None] * freq[None] * (-1.0 if inverse else 1.0)
    cs, sn = torch.cos(a) * magnitude, torch.sin(a) * magnitude
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if adjacent else (slice(0, rot // 2), slice(rot // 2, rot))
    y, size = x.clone(), torch.zeros_like(x)
    y[..., one] = x[..., one] * cs - x[..., two] * sn
    y[..., two] = x[..., two] * cs + x[..., one] * sn
    size[..., one] = size[..., two] = x[..., one].abs() + x[..., two].abs()
    return y, size


def check_rotary(got, want, size, dtype, magnitude=1.0, what=""):
    got = got.double().cpu()
    bound = 4 * 2.0 ** -23 * magnitude * size + half_step(dtype) * want.abs() * (size > 0) * 1.0001
    bad = (got - want).abs() > bound
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((got - want).abs().max()):.3e}"


def accept(parent, drafted, target, count):
    """Greedy walk of one sequence: path, next token."""
    if count == 0:
        return [], -1
    path = [0]
    while True:
        fit = [c for c in range(path[-1] + 1, count)
               if (c - 1 if parent is None else int(parent[c])) == path[-1] and int(drafted[c]) == int(target[path[-1]])]
        if not fit:
            return path, int(target[path[-1]])
        path.append(fit[0])


def random_parents(rnd, t):
    """-1 for node 0, an earlier node for the others, nearer ones more often."""
    return [-1] + [rnd.randint(max(0, i - rnd.choice([1, 3, 9])), i - 1) for i in range(1, t)]
