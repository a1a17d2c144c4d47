"""The operators of paged caches and sliding windows as measurable cases: what a program does with prompts whose
rows see a window, and with a batch of sequences whose keys and values lie in pages.

  window   reform_window_attend: packed prompts; a row sees the keys of a window behind it and a few first ones
  paged    reform_paged_attend: one new token for each sequence of a batch over its pages, with or without a window, with or
           without the attention weight that every key receives (added to what it received before)
  evict    reform_paged_evict: caches that outgrew their budget keep the keys that received the most attention weight, moved
           together in their pages

Where `own` is false, `run` computes the same in elementary torch operations.  Sizes are those of the repository's
workloads, of its tests, or generic.  `draw` gives more cases of the same ranges.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
LEFT = 2.0 ** -6      # what output rows hold that no call may write


def _binding():
    from paper_2506_01215_amd import binding
    return binding


# ------------------------------------------------------------------------------------- the cases

def _window(name, dtype, hq, hkv, d, lens, window, sinks, prefix=0, spare=0):
    """lens: query rows of each sequence; prefix: keys that every sequence has before its first query row; spare: rows
    behind the last sequence, which stay as they are."""
    return {"name": name, "kind": "window", "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "lens": lens, "window": window,
            "sinks": sinks, "prefix": prefix, "spare": spare}


def _paged(name, dtype, hq, hkv, d, lens, page, window=0, sinks=0, score=False):
    """lens: keys of each sequence, the new token's among them; page: rows of a page; window 0: every key is seen."""
    return {"name": name, "kind": "paged", "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "lens": lens, "page": page,
            "window": window, "sinks": sinks, "score": score}


def _evict(name, dtype, hkv, d, lens, page, budget, sinks, recent):
    """lens: keys of each sequence; those with more than `budget` keep that many, `sinks` first and `recent` last ones among them."""
    return {"name": name, "kind": "evict", "dtype": dtype, "hkv": hkv, "d": d, "lens": lens, "page": page, "budget": budget,
            "sinks": sinks, "recent": recent}


def _text(lens):
    return ",".join(str(int(x)) for x in lens)


def _numbers(text):
    return [int(x) for x in text.split(",")]


def listed():
    return [
        # seven questions of different lengths in one batch, one of a single token, a short window
        _window("window_ragged_7", "bf16", 24, 8, 64, "1,17,300,64,129,517,411", 128, 4, spare=33),
        # the same in fp32, with sizes of workload 1
        _window("window_f32_3", "f32", 4, 4, 64, "128,301,256", 64, 4),
        # chunks of a batch of longer inputs: 500 keys of each are there already
        _window("window_prefix_12", "bf16", 16, 4, 128, "700,64,1500,333,90,1024,41,800,256,612,77,1203", 256, 16, prefix=500),
        # one long input (the paper's larger budget) whose rows see a quarter of it and 256 first tokens
        _window("window_one_16k", "bf16", 32, 8, 128, "16384", 4096, 256),
        # a few short sequences, one with its first token: latency
        _paged("paged_few", "bf16", 24, 8, 64, "1,17,300,64", 16),
        # one sequence of workload 2's length
        _paged("paged_one_128k", "bf16", 32, 8, 128, "131072", 64),
        # a batch whose caches are to be compressed later: the weight of every key is added up token by token
        _paged("paged_score_32", "bf16", 32, 8, 128, _text([8192] * 8 + [(i * 1237) % 7900 + 100 for i in range(24)]), 16, score=True),
        # long sequences that see 4096 keys and 64 first ones
        _paged("paged_window_16", "bf16", 24, 8, 64, _text([16640] * 8 + [16640 - 997 * i for i in range(8)]), 32, window=4096, sinks=64),
        # workload 1's heads and length
        _paged("paged_f32_4", "f32", 4, 4, 64, "2048,1,777,256", 16, score=True),
        # every 256 tokens a batch goes back to its budget of 4096
        _evict("evict_16", "bf16", 8, 128, _text([4352] * 12 + [4097, 100, 4200, 4000]), 16, 4096, 256, 256),
        # one sequence with workload 3's budget
        _evict("evict_one_32k", "bf16", 8, 128, "33024", 64, 32768, 256, 256),
        # workload 1's heads and budget: latency
        _evict("evict_f32_4", "f32", 4, 64, "384,300,257,120", 16, 256, 4, 128),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


HEADS = [(32, 8), (8, 8), (24, 8), (14, 2), (16, 4), (4, 4), (16, 2), (8, 1)]
PAGES = [16, 16, 16, 32, 64, 64, 128, 256, 1, 8, 20]


def draw(rng):
    kind = rng.choice(["window", "window", "paged", "paged", "paged", "evict"])
    hq, hkv = rng.choice(HEADS)
    d = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "window":
        seqs, total = _spread(rng, 1, 32), _spread(rng, 30, 1500 if dtype == "f32" else 12000)
        share = [rng.expovariate(1.0) + 0.02 for _ in range(seqs)]
        lens = [max(1, int(total * x / sum(share))) for x in share]
        c = _window("", dtype, hq, hkv, d, _text(lens), _spread(rng, 1, 4096), rng.choice([0, 1, 4, _spread(rng, 1, 256)]),
                    prefix=rng.choice([0, 0, _spread(rng, 1, 300 if dtype == "f32" else 2000)]), spare=rng.choice([0, 0, 19]))
    elif kind == "paged":
        seqs = _spread(rng, 1, 48)
        most = _spread(rng, 30, min(4000 if dtype == "f32" else 100000, 130000000 // (seqs * hkv * d)))
        lens = [rng.randint(1, most) if rng.random() < 0.6 else most for _ in range(seqs)]
        window = rng.choice([0, 0, 0, _spread(rng, 1, 8192)])
        c = _paged("", dtype, hq, hkv, d, _text(lens), rng.choice(PAGES), window=window,
                   sinks=rng.choice([0, 1, 4, 64]) if window else 0, score=rng.random() < 0.5)
    else:
        seqs = _spread(rng, 1, 24)
        budget = _spread(rng, 60, min(30000, 33000000 // (seqs * hkv * d)))
        more = _spread(rng, 1, max(1, budget // 4))
        lens = [budget + more if rng.random() < 0.6 else rng.randint(1, budget + more) for _ in range(seqs)]
        c = _evict("", dtype, hkv, d, _text(lens), rng.choice(PAGES), budget, rng.randint(0, budget // 8), more + rng.randint(0, budget // 8))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------ the inputs

def _states(gen, heads, rows, d, shared):
    """States of `heads` heads: half of their energy lies in 16 directions that the heads share and is common to one
    token, so attention concentrates."""
    return torch.randn((heads, rows, d), generator=gen, device=DEV).mul_(math.sqrt(0.5)).add_(shared)


def _shared(gen, rows, d):
    basis = torch.linalg.qr(torch.randn((d, 16), generator=gen, device=DEV))[0].t()
    return (torch.randn((rows, 16), generator=gen, device=DEV) @ basis) * math.sqrt(d / 32.0)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _starts(lens):
    return [0] + list(np.cumsum(lens))


def _prepare_window(c, gen, rnd):
    dt, hq, hkv, d = DTYPE[c["dtype"]], c["hq"], c["hkv"], c["d"]
    lens = _numbers(c["lens"])
    klens = [x + c["prefix"] for x in lens]
    nq, nk = sum(lens) + c["spare"], sum(klens) + c["spare"]
    shared = _shared(gen, nk, d)
    s = {"k": _states(gen, hkv, nk, d, shared).to(dt), "v": torch.randn((hkv, nk, d), generator=gen, device=DEV).to(dt)}
    rows = torch.cat([torch.arange(b - n, b) for n, b in zip(lens, _starts(klens)[1:])] + [torch.arange(nk - c["spare"], nk)])
    s["q"] = _states(gen, hq, nq, d, shared[rows.to(DEV)]).to(dt)
    s["cu_q"], s["cu_k"] = _i32(_starts(lens)), _i32(_starts(klens)) if c["prefix"] else None
    s["out"] = torch.full((hq, nq, d), LEFT, dtype=dt, device=DEV)
    s["lse"] = torch.full((hq, nq), LEFT, dtype=torch.float32, device=DEV)
    s["scale"] = d ** -0.5
    return s


def _pages(c, rnd):
    """A table of pages that were handed out in no order: [sequences, most pages of one], -1 behind a sequence's last page.
    Returns it and the pages of the pool, some of which nobody has."""
    need = [-(-n // c["page"]) for n in _numbers(c["lens"])]
    order = rnd.permutation(sum(need) + 3)
    table = np.full((len(need), max(need)), -1, np.int64)
    for i, (n, a) in enumerate(zip(need, _starts(need))):
        table[i, :n] = order[a:a + n]
    return _i32(table), sum(need) + 3


def _prepare_paged(c, gen, rnd):
    dt, hq, hkv, d, page = DTYPE[c["dtype"]], c["hq"], c["hkv"], c["d"], c["page"]
    lens = _numbers(c["lens"])
    s = {"lens": _i32(lens), "scale": d ** -0.5}
    s["table"], n = _pages(c, rnd)
    shared = _shared(gen, n * page, d).view(n, 1, page, d)
    for x in "kv":
        s[x] = torch.randn((n, hkv, page, d), generator=gen, device=DEV)
    s["k"].mul_(math.sqrt(0.5)).add_(shared)
    s["k"], s["v"] = s["k"].to(dt), s["v"].to(dt)
    about = shared.reshape(n * page, d)[torch.from_numpy(rnd.randint(0, n * page, len(lens))).to(DEV)]
    s["q"] = _states(gen, hq, len(lens), d, about).transpose(0, 1).contiguous().to(dt)
    s["out"] = torch.full((len(lens), hq, d), LEFT, dtype=dt, device=DEV)
    s["lse"] = torch.full((len(lens), hq), LEFT, dtype=torch.float32, device=DEV)
    s["score"] = None
    if c["score"]:
        s["score"] = torch.randn((len(lens), hkv, s["table"].shape[1] * page), generator=gen, device=DEV).exp_()
    return s


def _prepare_evict(c, gen, rnd):
    dt, hkv, d, page = DTYPE[c["dtype"]], c["hkv"], c["d"], c["page"]
    lens = _numbers(c["lens"])
    s = {"lens": _i32(lens)}
    s["table"], n = _pages(c, rnd)
    for x in "kv":
        s[x] = torch.randn((n, hkv, page, d), generator=gen, device=DEV).to(dt)
    shape = (len(lens), hkv, s["table"].shape[1] * page)
    s["score"] = torch.randn(shape, generator=gen, device=DEV).mul_(2.0).exp_()
    s["score"].mul_(torch.rand(shape, generator=gen, device=DEV) > 0.05)       # some keys never received any
    s["pos"] = torch.arange(shape[2], dtype=torch.int32, device=DEV).repeat(shape[0], shape[1], 1)
    s["kept"] = torch.full((len(lens), hkv, c["budget"]), -1, dtype=torch.int32, device=DEV)
    s["new_len"] = torch.zeros(len(lens), dtype=torch.int32, device=DEV)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    make = {"window": _prepare_window, "paged": _prepare_paged, "evict": _prepare_evict}
    return dict(make[case["kind"]](case, gen, np.random.RandomState(int(seed) % (1 << 31))), case=dict(case))


# ------------------------------------------------------------------ the calls, and their plain form

def run(state):
    s, c = state, state["case"]
    return (_own if own else _plain)[c["kind"]](s, c)


def _workspace(s, query, desc):
    """The program's workspace, which it keeps from its first call on."""
    if "ws" not in s:
        s["ws"] = torch.empty(query(desc()) + 256, dtype=torch.uint8, device=DEV)
    return s["ws"]


def _own_window(s, c):
    b = _binding()
    ws = _workspace(s, b.window_workspace_bytes, lambda: b.window_desc(s["q"], s["k"], s["v"], s["out"], s["cu_q"], s["scale"], c["window"], c["sinks"]))
    out, lse = b.reform_window_attend(s["q"], s["k"], s["v"], s["cu_q"], s["scale"], c["window"], n_sink=c["sinks"], cu_k=s["cu_k"],
                                      out=s["out"], lse=s["lse"], workspace=ws)
    return {"out": out, "lse": lse}


def _own_paged(s, c):
    b = _binding()
    ws = _workspace(s, b.paged_workspace_bytes, lambda: b.paged_desc(s["q"], s["k"], s["v"], s["out"], s["table"], s["scale"], window=c["window"],
                                                                     n_sink=c["sinks"], score=s["score"], accumulate=True))
    out, lse = b.reform_paged_attend(s["q"], s["k"], s["v"], s["table"], s["lens"], s["scale"], window=c["window"], n_sink=c["sinks"],
                                     score=s["score"], accumulate=True, out=s["out"], lse=s["lse"], workspace=ws)
    return {"out": out, "lse": lse, "score": s["score"]}


def _own_evict(s, c):
    b = _binding()
    ws = _workspace(s, b.paged_evict_workspace_bytes, lambda: b.paged_evict_desc(s["k"], s["v"], s["score"], s["table"], c["budget"],
                                                                                n_sink=c["sinks"], n_recent=c["recent"]))
    new_len = b.reform_paged_evict(s["k"], s["v"], s["score"], s["table"], s["lens"], c["budget"], n_sink=c["sinks"], n_recent=c["recent"],
                                   pos=s["pos"], kept_idx=s["kept"], new_len=s["new_len"], workspace=ws)
    return {"k": s["k"], "v": s["v"], "score": s["score"], "pos": s["pos"], "kept": s["kept"], "new_len": new_len}


def _softmax(x, dim):
    """Exponentials against the largest, and their sum and log, over keys of which some rows see none."""
    top = x.amax(dim, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    x = (x - top).exp_()
    total = x.sum(dim, keepdim=True)
    return x / torch.where(total == 0, torch.ones_like(total), total), (top + total.log()).squeeze(dim)


def _plain_window(s, c):
    lens = _numbers(c["lens"])
    hq, hkv, d, group = c["hq"], c["hkv"], c["d"], c["hq"] // c["hkv"]
    step = 1024
    for n, q0, k0 in zip(lens, _starts(lens), _starts([n + c["prefix"] for n in lens])):
        for r in range(0, n, step):              # only the keys that a row of the block sees
            m = min(step, n - r)
            last = torch.arange(r, r + m, device=DEV) + c["prefix"]
            lo, hi = max(0, r + c["prefix"] - c["window"] + 1), r + m + c["prefix"]
            keys = torch.cat([torch.arange(min(c["sinks"], lo), device=DEV), torch.arange(lo, hi, device=DEV)])
            q = s["q"][:, q0 + r:q0 + r + m].float().reshape(hkv, group * m, d)
            x = torch.matmul(q, s["k"][:, k0 + keys].float().transpose(1, 2).contiguous()).mul_(s["scale"]).view(hkv, group, m, -1)
            seen = (keys <= last[:, None]) & ((keys > last[:, None] - c["window"]) | (keys < c["sinks"]))
            p, e = _softmax(x.masked_fill_(~seen, float("-inf")), -1)
            o = torch.matmul(p.view(hkv, group * m, -1), s["v"][:, k0 + keys].float())
            s["out"][:, q0 + r:q0 + r + m] = o.view(hq, m, d).to(s["out"].dtype)
            s["lse"][:, q0 + r:q0 + r + m] = e.view(hq, m)
    return {"out": s["out"], "lse": s["lse"]}


def _plain_paged(s, c):
    hkv, group, page = c["hkv"], c["hq"] // c["hkv"], c["page"]
    n = s["lens"].long()[:, None]
    seqs, most = n.shape[0], s["table"].shape[1] * page
    if c["window"]:                              # the first keys, then the window's, [sequences, rows]
        first = torch.arange(min(c["sinks"], most), device=DEV).expand(seqs, -1)
        last = torch.arange(-min(c["window"], most), 0, device=DEV) + n
        rows = torch.cat([first, last], 1)
        seen = torch.cat([first < (n - c["window"]).clamp(min=0), last >= 0], 1)
    else:
        rows = torch.arange(most, device=DEV).expand(seqs, -1)
        seen = rows < n
    rows = torch.where(seen, rows, torch.zeros_like(rows))
    at = s["table"].long().gather(1, rows // page)
    k, v = (s[x][at, :, rows % page].transpose(1, 2).float() for x in "kv")              # [sequences, heads, rows, elements]
    q = s["q"].view(seqs, hkv, group, -1).float().transpose(2, 3).contiguous()
    x = torch.matmul(k, q).mul_(s["scale"]).masked_fill_(~seen[:, None, :, None], float("-inf"))
    p, e = _softmax(x, 2)
    out = torch.matmul(p.transpose(2, 3).contiguous(), v.contiguous())
    s["out"].copy_(out.view(s["out"].shape))
    s["lse"].copy_(e.view(s["lse"].shape))
    if s["score"] is not None:
        seq, row = seen.nonzero(as_tuple=True)
        place = rows[seq, row]
        before = torch.where((place == n[seq, 0] - 1)[:, None], torch.zeros((), device=DEV), s["score"][seq, :, place])   # the new key has none
        s["score"][seq, :, place] = before + p.sum(3)[seq, :, row]
    return {"out": s["out"], "lse": s["lse"], "score": s["score"]}


def _plain_evict(s, c):
    page, budget = c["page"], c["budget"]
    n = s["lens"].long()[:, None, None]
    seqs, hkv, most = s["score"].shape
    rows = torch.arange(most, device=DEV)
    always = (rows < c["sinks"]) | (rows >= n - c["recent"])
    x = s["score"].masked_fill(always, float("inf")).masked_fill(rows >= n, float("-inf"))
    kept = x.sort(dim=-1, descending=True, stable=True)[1][..., :budget].sort(dim=-1)[0]         # those behind the last key come last
    seq, head, r = (torch.arange(kept.shape[-1], device=DEV) < n).expand(kept.shape).nonzero(as_tuple=True)
    old = kept[seq, head, r]
    src, dst = s["table"].long()[seq, old // page], s["table"].long()[seq, r // page]
    for x in ("k", "v"):
        s[x][dst, head, r % page] = s[x][src, head, old % page]
    for x in ("score", "pos"):
        s[x][seq, head, r] = s[x][seq, head, old]
    s["kept"][seq, head, r] = old.int()
    s["new_len"].copy_(s["lens"].clamp(max=budget))
    return {"k": s["k"], "v": s["v"], "score": s["score"], "pos": s["pos"], "kept": s["kept"], "new_len": s["new_len"]}


_own = {"window": _own_window, "paged": _own_paged, "evict": _own_evict}
_plain = {"window": _plain_window, "paged": _plain_paged, "evict": _plain_evict}


# ---------------------------------------------------------------------------- the definition, 64 bits

def _attend64(q, k, v, scale, hide):
    """Out, log of the sums and probabilities of rows q [m, d] over keys [n, d], those of `hide` [m, n] left out."""
    x = (q.double() * scale) @ k.double().t().contiguous()
    x[hide] = float("-inf")
    e = torch.logsumexp(x, -1)
    p = torch.exp(x - torch.where(e == float("-inf"), torch.zeros_like(e), e)[:, None])
    return p @ v.double(), e, p


def _exact_window(s, c):
    out = torch.full(s["q"].shape, LEFT, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, LEFT, dtype=torch.float64, device=DEV)
    lens, w = _numbers(c["lens"]), c["window"]
    qs, ks = _starts(lens), _starts([n + c["prefix"] for n in lens])
    for i, n in enumerate(lens):
        for r in range(0, n, 2048):
            m = min(2048, n - r)
            place = torch.arange(r, r + m, device=DEV)[:, None] + c["prefix"]
            j = torch.arange(r + m + c["prefix"], device=DEV)[None]
            hide = (j > place) | ((place - j >= w) & (j >= c["sinks"]))
            for h in range(c["hq"]):
                g, b = h * c["hkv"] // c["hq"], slice(ks[i], ks[i] + j.shape[1])
                a = slice(qs[i] + r, qs[i] + r + m)
                out[h, a], lse[h, a], _ = _attend64(s["q"][h, a], s["k"][g, b], s["v"][g, b], s["scale"], hide)
    return {"out": out, "lse": lse}


def _row_list(s, i, n, page):
    """Pool rows of sequence i's first n keys."""
    table = s["table"][i].tolist()
    return torch.tensor([table[j // page] * page + j % page for j in range(n)], dtype=torch.long, device=DEV)


def _flat(x):
    """[pages, heads, rows, d] as [heads, all rows, d]."""
    return x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])


def _exact_paged(s, c):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    score = None if s["score"] is None else s["score"].double()
    k, v = _flat(s["k"]), _flat(s["v"])
    group = c["hq"] // c["hkv"]
    for i, n in enumerate(_numbers(c["lens"])):
        rows, j = _row_list(s, i, n, c["page"]), torch.arange(n, device=DEV)[None].expand(group, n)
        hide = (j < n - c["window"]) & (j >= c["sinks"]) if c["window"] else j < 0
        for g in range(c["hkv"]):
            h = slice(g * group, (g + 1) * group)
            out[i, h], lse[i, h], p = _attend64(s["q"][i, h], k[g, rows], v[g, rows], s["scale"], hide)
            if score is not None:
                score[i, g, n - 1] = 0.0
                score[i, g, :n] += p.sum(0)
    return {"out": out, "lse": lse, "score": score}


def _exact_evict(s, c):
    k, v, score = (s[x].double().cpu().numpy() for x in ("k", "v", "score"))
    pos, kept, table = (s[x].cpu().numpy() for x in ("pos", "kept", "table"))
    page, lens = c["page"], _numbers(c["lens"])
    for i, n in enumerate(lens):
        for g in range(c["hkv"]):
            keep = np.arange(n)
            if n > c["budget"]:
                middle = np.arange(c["sinks"], n - c["recent"])
                best = middle[np.lexsort((middle, -score[i, g, middle]))][:c["budget"] - c["sinks"] - c["recent"]]
                keep = np.concatenate([np.arange(c["sinks"]), np.sort(best), np.arange(n - c["recent"], n)])
            to = np.arange(len(keep))
            a, b = table[i, to // page], table[i, keep // page]
            for x in (k, v):
                x[a, g, to % page] = x[b, g, keep % page].copy()
            for x in (score, pos):
                x[i, g, to] = x[i, g, keep].copy()
            kept[i, g, to] = keep
    return {"k": k, "v": v, "score": score, "pos": pos, "kept": kept, "new_len": _i32([min(n, c["budget"]) for n in lens])}


def exact(case, seed):
    return {"window": _exact_window, "paged": _exact_paged, "evict": _exact_evict}[case["kind"]](prepare(case, seed), case)


# ------------------------------------------------------------------------------------ what it takes

def work(case):
    """Inputs read once, outputs written once; products of the visible pairs."""
    c, e = case, SIZE[case["dtype"]]
    lens = _numbers(c["lens"])
    if c["kind"] == "window":
        pairs = 0
        for n in lens:
            last = np.arange(n, dtype=np.int64) + c["prefix"]
            lo = np.maximum(last - c["window"] + 1, 0)
            pairs += int((last - lo + 1 + np.minimum(c["sinks"], lo)).sum())
        nq, nk = sum(lens), sum(n + c["prefix"] for n in lens)
        return {"bytes": 2.0 * e * c["d"] * (c["hq"] * nq + c["hkv"] * nk) + 4.0 * c["hq"] * nq,
                "flops": 4.0 * c["d"] * c["hq"] * pairs}
    if c["kind"] == "paged":
        seen = sum(min(n, c["window"]) + min(c["sinks"], max(0, n - c["window"])) if c["window"] else n for n in lens)
        return {"bytes": 2.0 * e * c["d"] * (c["hkv"] * seen + c["hq"] * len(lens)) + 4.0 * c["hq"] * len(lens)
                + (8.0 * c["hkv"] * seen if c["score"] else 0.0) + 4.0 * seen / c["page"],
                "flops": 4.0 * c["d"] * c["hq"] * seen}
    over = [n for n in lens if n > c["budget"]]
    # nearly all rows behind the first keys move: among these the first one that goes comes early
    moved = float(len(over) * (c["budget"] - c["sinks"]) * c["hkv"])
    return {"bytes": 4.0 * c["hkv"] * sum(over) + moved * (4.0 * e * c["d"] + 16.0) + 4.0 * c["hkv"] * sum(min(n, c["budget"]) for n in lens),
            "flops": 0.0}
