"""The serving operators as measurable cases: what a program does with a prompt, a batch of prompts
or a batch of drafted tokens around the library's caches.

  rotary   reform_rotary_embed: queries rotated to their positions, keys rotated and stored with the
           values in the caches (or everything rotated where it stands, or rotated back)
  prompt   reform_prompt_attend: causal attention over whole prompts of different lengths, packed
  tree     reform_tree_attend: drafted tokens (a tree of them, a chain, or one token) over the caches
  accept   reform_rotary_embed of a step's drafted keys and values into the caches, then
           reform_tree_accept: the path of drafted tokens that the model agrees with, its rows moved
           together behind the cached ones

Where `own` is false, `run` computes the same in elementary torch operations.  Sizes are those of the
repository's workloads, of its tests, or generic.  `draw` gives more cases of the same ranges.
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

def _rotary(name, dtype, n, hq, hkv, d, rot, far, scaling="none", interleaved=False, inverse=False, blocks=0):
    """n tokens at positions up to `far`; blocks > 0: the keys and values go to rows of as many caches,
    else keys are rotated into a tensor of their own and there are no values."""
    return {"name": name, "kind": "rotary", "dtype": dtype, "n": n, "hq": hq, "hkv": hkv, "d": d, "rot": rot,
            "far": far, "scaling": scaling, "interleaved": interleaved, "inverse": inverse, "blocks": blocks}


def _prompt(name, dtype, hq, hkv, d, lens, prefix=0, spare=0):
    """lens: query rows of each sequence; prefix: keys that every sequence has before its first query
    row; spare: rows behind the last sequence, which stay as they are."""
    return {"name": name, "kind": "prompt", "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "lens": lens,
            "prefix": prefix, "spare": spare}


def _tree(name, dtype, hq, hkv, d, nodes, lens, cap, chain=False, ragged=False):
    """nodes: drafted tokens per sequence; lens: cached rows of each sequence; ragged: every other
    sequence has fewer nodes than the batch has room for."""
    return {"name": name, "kind": "tree", "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "nodes": nodes,
            "lens": lens, "cap": cap, "chain": chain, "ragged": ragged}


def _accept(name, dtype, hkv, d, nodes, seqs, cap, agree):
    """agree: drafted tokens on the path that the model agrees with, the first one included."""
    return {"name": name, "kind": "accept", "dtype": dtype, "hkv": hkv, "d": d, "nodes": nodes,
            "seqs": seqs, "cap": cap, "agree": agree}


def _text(lens):
    return ",".join(str(int(x)) for x in lens)


def _numbers(text):
    return [int(x) for x in text.split(",")]


def listed():
    return [
        # one generated token for each of 16 sequences, into their caches, far positions: latency
        _rotary("rotary_token_16", "bf16", 16, 32, 8, 128, 128, 1000000, blocks=16),
        # a chunk of 8192 tokens of a stream longer than the model was trained for (workload 2's heads)
        _rotary("rotary_chunk_8k", "bf16", 8192, 32, 8, 128, 128, 131072, scaling="parts", blocks=1),
        # the gradient with respect to the states before rotation: fp32, pairs side by side, half of each head
        _rotary("rotary_back_f32", "f32", 2001, 14, 2, 64, 32, 30000, interleaved=True, inverse=True),
        # seven questions of different lengths in one batch, one of a single token (64-wide heads)
        _prompt("prompt_ragged_7", "bf16", 24, 8, 64, "1,17,300,64,129,517,411", spare=33),
        # the same in fp32, with sizes of workload 1
        _prompt("prompt_f32_3", "f32", 4, 4, 64, "128,301,256"),
        # a batch of prompts behind a shared kind of preamble of 500 tokens that is cached already
        _prompt("prompt_prefix_12", "bf16", 16, 4, 128, "700,64,1500,333,90,1024,41,800,256,612,77,1203", prefix=500),
        # 16384 recomputed tokens (the paper's larger budget) of one input
        _prompt("prompt_one_16k", "bf16", 32, 8, 128, "16384"),
        # the same number of tokens from ten inputs of different lengths
        _prompt("prompt_ten_16k", "bf16", 32, 8, 128, "5000,17,2048,1111,640,3333,90,2500,133,1512"),
        # one token for each of eight sequences over their recomputed caches
        _tree("tree_token_8", "bf16", 32, 8, 128, 1, "16640,300,8192,4097,12000,1,16000,9001", 16704),
        # 48 drafted tokens of one sequence over a 16k cache
        _tree("tree_48_one", "bf16", 32, 8, 128, 48, "16640", 16704),
        # up to 17 drafted tokens for each of 16 sequences over a full compressed cache, 64-wide heads
        _tree("tree_17_ragged", "bf16", 24, 8, 64, 17, _text([4096] * 10 + [100, 2047, 3000, 4000, 555, 31]), 4160, ragged=True),
        # 8 heads of 12 sequences, 32 drafted tokens each, seven accepted
        _accept("accept_12", "bf16", 8, 128, 32, 12, 600, 7),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


HEADS = [(32, 8), (8, 8), (24, 8), (14, 2), (16, 4), (4, 4), (16, 2), (8, 1)]


def draw(rng):
    kind = rng.choice(["rotary", "prompt", "prompt", "tree", "tree", "accept"])
    hq, hkv = rng.choice(HEADS)
    d = rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "rotary":
        n = _spread(rng, 1, 16000)
        blocks = rng.choice([0, 1, min(n, rng.randint(2, 24))])
        c = _rotary("", dtype, n, hq, hkv, d, rng.choice([d, d, d // 2, d // 4]), _spread(rng, 1000, 2000000),
                    scaling=rng.choice(["none", "linear", "base", "parts", "bands"]),
                    interleaved=rng.random() < 0.5, inverse=rng.random() < 0.3, blocks=blocks)
    elif kind == "prompt":
        seqs, total = _spread(rng, 1, 32), _spread(rng, 30, 1500 if dtype == "f32" else 12000)
        share = [rng.expovariate(1.0) + 0.02 for _ in range(seqs)]
        lens = [max(1, int(total * x / sum(share))) for x in share]
        prefix = rng.choice([0, 0, _spread(rng, 1, 300 if dtype == "f32" else 2000)])
        c = _prompt("", dtype, hq, hkv, d, _text(lens), prefix=prefix, spare=rng.choice([0, 0, 19]))
    elif kind == "tree":
        nodes, seqs = rng.choice([1, 1, _spread(rng, 2, 64), _spread(rng, 2, 64)]), _spread(rng, 1, 32)
        most = _spread(rng, 100, (2000 if dtype == "f32" else 40000) // (1 if seqs < 8 else 4))
        lens = [rng.randint(0, most) if rng.random() < 0.6 else most for _ in range(seqs)]
        c = _tree("", dtype, hq, hkv, d, nodes, _text(lens), max(lens) + nodes + rng.randint(0, 40),
                  chain=rng.random() < 0.3, ragged=rng.random() < 0.4)
    else:
        nodes, seqs = _spread(rng, 2, 64), _spread(rng, 1, 24)
        c = _accept("", dtype, hkv, d, nodes, seqs, nodes + _spread(rng, 30, 1200), rng.randint(1, min(nodes, 12)))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------ the inputs

SCALING = {   # what a program passes with each kind of scaled positions
    "none": {},
    "linear": {"scaling": "linear", "factor": 4.0},
    "base": {"scaling": "base", "factor": 8.0},
    "parts": {"scaling": "parts", "factor": 16.0, "original_len": 8192, "turns_high": 32.0, "turns_low": 1.0,
              "magnitude": 0.1 * math.log(16.0) + 1.0},
    "bands": {"scaling": "bands", "factor": 8.0, "original_len": 8192, "turns_high": 4.0, "turns_low": 1.0},
}
THETA = 1e6


def _states(gen, heads, rows, d, shared):
    """States of `heads` heads: half of their energy lies in 16 directions that the heads share and
    is common to one token, so attention concentrates."""
    x = torch.randn((heads, rows, d), generator=gen, device=DEV).mul_(math.sqrt(0.5))
    return x.add_(shared)


def _shared(gen, rows, d):
    basis = torch.linalg.qr(torch.randn((d, 16), generator=gen, device=DEV))[0].t()
    return (torch.randn((rows, 16), generator=gen, device=DEV) @ basis) * math.sqrt(d / 32.0)


def _workspace(nbytes):
    return torch.empty(nbytes + 256, dtype=torch.uint8, device=DEV)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _prepare_rotary(c, gen, rnd):
    dt, n, hq, hkv, d = DTYPE[c["dtype"]], c["n"], c["hq"], c["hkv"], c["d"]
    # states come token by token from the projection, queries, keys and values side by side
    qkv = torch.randn((n, hq + 2 * hkv, d), generator=gen, device=DEV).to(dt).transpose(0, 1)
    s = {"q": qkv[:hq], "k": qkv[hq:hq + hkv], "v": qkv[hq + hkv:]}
    s["q_out"] = torch.full((hq, n, d), LEFT, dtype=dt, device=DEV)
    if c["blocks"]:
        b = c["blocks"]
        per = -(-n // b)
        cap = per + 5
        pos, slot = np.zeros(n, np.int64), np.zeros(n, np.int64)
        for j in range(b):                       # each cache gets a run of tokens, at consecutive positions
            at = np.arange(j * per, min(n, (j + 1) * per))
            pos[at] = rnd.randint(0, max(1, c["far"] - per)) + at - j * per
            slot[at] = j * cap + rnd.randint(0, 6) + at - j * per
        if n > 8:
            slot[rnd.randint(0, n)] = -1         # a padding token: its key and value are not stored
        s["slot"] = _i32(slot)
        s["k_out"] = torch.full((b, hkv, cap, d), LEFT, dtype=dt, device=DEV)
        s["v_out"] = torch.full_like(s["k_out"], LEFT)
    else:
        pos = np.sort(rnd.randint(0, c["far"], n))         # selected tokens keep their own positions
        s["slot"], s["v"], s["v_out"] = None, None, None
        s["k_out"] = torch.full((hkv, n, d), LEFT, dtype=dt, device=DEV)
    s["pos"] = _i32(pos)
    return s


def _starts(lens):
    return [0] + list(np.cumsum(lens))


def _prepare_prompt(c, gen, rnd):
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
    if own:
        b = _binding()
        s["ws"] = _workspace(b.prompt_workspace_bytes(b.prompt_desc(s["q"], s["k"], s["v"], s["out"], s["cu_q"], s["scale"])))
    return s


def _parents(rnd, nodes):
    """A drafted tree in order of depth: every node's parent is one of the few likeliest before it."""
    p = np.full(nodes, -1, np.int64)
    for i in range(1, nodes):
        p[i] = rnd.randint(max(0, (i - 1) // 3 - 2), (i + 1) // 2)
    return p


def _counts(c):
    t = c["nodes"]
    return [max(0, t - (i * 5) % (t + 1)) if c["ragged"] and i % 2 else t for i in range(len(_numbers(c["lens"])))]


def _prepare_tree(c, gen, rnd):
    dt, hq, hkv, d, t = DTYPE[c["dtype"]], c["hq"], c["hkv"], c["d"], c["nodes"]
    lens = _numbers(c["lens"])
    b, cap = len(lens), c["cap"]
    s = {x: torch.empty((b, hkv, cap, d), dtype=dt, device=DEV) for x in "kv"}
    s["q"] = torch.empty((b, hq, t, d), dtype=dt, device=DEV)
    for i, n in enumerate(lens):
        shared = _shared(gen, cap, d)
        s["k"][i] = _states(gen, hkv, cap, d, shared).to(dt)
        s["v"][i] = torch.randn((hkv, cap, d), generator=gen, device=DEV).to(dt)
        s["q"][i] = _states(gen, hq, t, d, shared[n:n + t]).to(dt)
    s["lens"] = _i32(lens)
    s["parent"] = None if c["chain"] else _i32(np.stack([_parents(rnd, t) for _ in lens]))
    s["count_list"] = _counts(c)
    s["counts"] = _i32(s["count_list"]) if c["ragged"] else None
    s["out"] = torch.full((b, hq, t, d), LEFT, dtype=dt, device=DEV)
    s["lse"] = torch.full((b, hq, t), LEFT, dtype=torch.float32, device=DEV)
    s["scale"] = d ** -0.5
    if own:
        bd = _binding()
        s["ws"] = _workspace(bd.tree_workspace_bytes(bd.tree_desc(s["q"], s["k"], s["v"], s["out"], s["scale"])))
    return s


def _prepare_accept(c, gen, rnd):
    dt, hkv, d, t, b, cap = DTYPE[c["dtype"]], c["hkv"], c["d"], c["nodes"], c["seqs"], c["cap"]
    s = {x: torch.randn((b, hkv, cap, d), generator=gen, device=DEV).to(dt) for x in ("k", "v")}
    for x in ("new_k", "new_v"):                 # the drafted tokens' states, token by token
        s[x] = torch.randn((b * t, hkv, d), generator=gen, device=DEV).to(dt).transpose(0, 1)
    lens = rnd.randint(0, cap - t + 1, b)
    parent, drafted, target = np.zeros((b, t), np.int64), np.zeros((b, t), np.int64), np.zeros((b, t), np.int64)
    depth, pos = np.zeros((b, t), np.int64), np.zeros((b, t), np.int64)
    for i in range(b):
        p = parent[i] = _parents(rnd, t)
        drafted[i], target[i] = rnd.randint(0, 32000, t), rnd.randint(32000, 64000, t)
        cur = 0
        for _ in range(c["agree"] - 1):          # the model agrees with one child after another
            kids = np.nonzero(p == cur)[0]
            if not kids.size:
                break
            nxt = int(rnd.choice(kids))
            target[i, cur] = drafted[i, nxt]
            cur = nxt
        for j in range(1, t):
            depth[i, j] = depth[i, p[j]] + 1
        pos[i] = lens[i] + depth[i]
    s["lens"], s["parent"], s["drafted"], s["target"] = _i32(lens), _i32(parent), _i32(drafted), _i32(target)
    s["pos"] = _i32(pos.reshape(-1))
    s["slot"] = _i32((np.arange(b)[:, None] * cap + lens[:, None] + np.arange(t)[None]).reshape(-1))
    for x, shape in (("path", (b, t)), ("accepted", (b,)), ("next", (b,)), ("new_len", (b,))):
        s[x] = torch.zeros(shape, dtype=torch.int32, device=DEV)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    make = {"rotary": _prepare_rotary, "prompt": _prepare_prompt, "tree": _prepare_tree, "accept": _prepare_accept}
    return dict(make[case["kind"]](case, gen, np.random.RandomState(int(seed) % (1 << 31))), case=dict(case))


# ------------------------------------------------------------------ the calls, and their plain form

def run(state):
    s, c = state, state["case"]
    return (_own if own else _plain)[c["kind"]](s, c)


def _own_rotary(s, c):
    q, k, v = _binding().reform_rotary_embed(
        s["q"], s["k"], s["v"], s["pos"], theta=THETA, rotary_dim=c["rot"], interleaved=c["interleaved"],
        inverse=c["inverse"], slot=s["slot"], q_out=s["q_out"], k_out=s["k_out"], v_out=s["v_out"], **SCALING[c["scaling"]])
    return {"q": q, "k": k, "v": v}


def _own_prompt(s, c):
    out, lse = _binding().reform_prompt_attend(s["q"], s["k"], s["v"], s["cu_q"], s["scale"], cu_k=s["cu_k"],
                                               out=s["out"], lse=s["lse"], workspace=s["ws"])
    return {"out": out, "lse": lse}


def _own_tree(s, c):
    out, lse = _binding().reform_tree_attend(s["q"], s["k"], s["v"], s["lens"], s["scale"], parent=s["parent"],
                                             node_count=s["counts"], out=s["out"], lse=s["lse"], workspace=s["ws"])
    return {"out": out, "lse": lse}


def _own_accept(s, c):
    b = _binding()
    b.reform_rotary_embed(None, s["new_k"], s["new_v"], s["pos"], theta=THETA, slot=s["slot"], k_out=s["k"], v_out=s["v"])
    path, accepted, following, new_len = b.reform_tree_accept(
        s["parent"], s["drafted"], s["target"], s["lens"], s["k"], s["v"], path=s["path"], accepted=s["accepted"],
        next_token=s["next"], new_len=s["new_len"])
    return {"path": path, "accepted": accepted, "next": following, "new_len": new_len, "k": s["k"], "v": s["v"]}


def _angles(pos, rot, scaling):
    """cos and sin of every position and pair in 64 bits, rounded to 32: the angle of a far position
    has more digits than 32 bits hold."""
    c = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    a = SCALING[scaling]
    theta = THETA
    if scaling == "base":
        theta = THETA * a["factor"] ** (rot / (rot - 2.0))
    f = theta ** (-2.0 * c / rot)
    if scaling == "linear":
        f = f / a["factor"]
    elif scaling == "parts":     # pairs that turn often in the trained length stay, those that hardly turn are stretched
        pair = [rot * math.log(a["original_len"] / (2.0 * math.pi * t)) / (2.0 * math.log(THETA))
                for t in (a["turns_high"], a["turns_low"])]
        low, high = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), rot - 1)
        ramp = ((c - low) / max(high - low, 0.001)).clamp(0.0, 1.0)
        f = f * (1.0 - ramp) + f / a["factor"] * ramp
    elif scaling == "bands":
        turns = a["original_len"] * f / (2.0 * math.pi)
        keep = ((turns - a["turns_low"]) / (a["turns_high"] - a["turns_low"])).clamp(0.0, 1.0)
        f = f * keep + f / a["factor"] * (1.0 - keep)
    angle = pos.double()[:, None] * f[None]
    m = a.get("magnitude", 1.0)
    return (angle.cos() * m).float(), (angle.sin() * m).float()


def _turn(x, cos, sin, rot, interleaved, inverse):
    """x [heads, rows, d] in 32 bits, its first `rot` elements rotated."""
    if inverse:
        sin = -sin
    y = x.float().clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., first].float(), x[..., second].float()
    y[..., first] = a * cos - b * sin
    y[..., second] = b * cos + a * sin
    return y


def _store(dst, rows, slot, cap):
    """rows [heads, n, d] to the cache rows that slot names."""
    at = (slot >= 0) & (slot < dst.shape[0] * cap)
    w = slot.long()[at]
    dst[w // cap, :, w % cap] = rows[:, at].transpose(0, 1).to(dst.dtype)


def _plain_rotary(s, c):
    cos, sin = _angles(s["pos"], c["rot"], c["scaling"])
    s["q_out"].copy_(_turn(s["q"], cos, sin, c["rot"], c["interleaved"], c["inverse"]))
    k = _turn(s["k"], cos, sin, c["rot"], c["interleaved"], c["inverse"])
    if s["slot"] is None:
        s["k_out"].copy_(k)
    else:
        cap = s["k_out"].shape[2]
        _store(s["k_out"], k, s["slot"], cap)
        _store(s["v_out"], s["v"], s["slot"], cap)
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _softmax_rows(q, k, v, scale, seen):
    """q [G, rows, d], k and v [n, d], seen [rows, n] or None: attention and log of the sums, 32 bits."""
    x = torch.matmul(q.float(), k.float().t().contiguous()).mul_(scale)
    x.masked_fill_(~seen, float("-inf"))
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x, v.float()) / torch.where(total == 0, torch.ones_like(total), total)
    return out, (top + total.log()).squeeze(-1)


def _plain_prompt(s, c):
    lens = _numbers(c["lens"])
    group, at_q, at_k = c["hq"] // c["hkv"], 0, 0
    for n in lens:
        nk = n + c["prefix"]
        keys = torch.arange(nk, device=DEV)
        for r in range(0, n, 4096):
            m = min(4096, n - r)
            seen = keys[None] <= torch.arange(r, r + m, device=DEV)[:, None] + c["prefix"]
            for h in range(c["hkv"]):
                heads, rows = slice(h * group, (h + 1) * group), slice(at_q + r, at_q + r + m)
                o, e = _softmax_rows(s["q"][heads, rows], s["k"][h, at_k:at_k + nk], s["v"][h, at_k:at_k + nk], s["scale"], seen)
                s["out"][heads, rows], s["lse"][heads, rows] = o.to(s["out"].dtype), e
        at_q, at_k = at_q + n, at_k + nk
    return {"out": s["out"], "lse": s["lse"]}


def _ancestors(parent, t):
    """[t, t] truth values: node i sees node j."""
    if parent is None:
        return torch.ones((t, t), dtype=torch.bool, device=DEV).tril()
    step = torch.eye(t, dtype=torch.float32, device=DEV)
    up = parent.long()
    step[torch.arange(t, device=DEV), torch.where(up >= 0, up, torch.arange(t, device=DEV))] = 1.0
    for _ in range(max(1, (t - 1).bit_length())):          # 1, 2, 4, ... steps up
        step = (step @ step > 0).float()
    return step > 0


def _plain_tree(s, c):
    t, group = c["nodes"], c["hq"] // c["hkv"]
    for i, n in enumerate(_numbers(c["lens"])):
        m = s["count_list"][i]
        if m == 0:
            continue
        tree = _ancestors(None if s["parent"] is None else s["parent"][i, :m], m)
        seen = torch.cat([torch.ones((m, n), dtype=torch.bool, device=DEV), tree], 1)
        for h in range(c["hkv"]):
            heads = slice(h * group, (h + 1) * group)
            o, e = _softmax_rows(s["q"][i, heads, :m], s["k"][i, h, :n + m], s["v"][i, h, :n + m], s["scale"], seen)
            s["out"][i, heads, :m], s["lse"][i, heads, :m] = o.to(s["out"].dtype), e
    return {"out": s["out"], "lse": s["lse"]}


def _plain_accept(s, c):
    b, t, cap = c["seqs"], c["nodes"], c["cap"]
    cos, sin = _angles(s["pos"], c["d"], "none")
    _store(s["k"], _turn(s["new_k"], cos, sin, c["d"], False, False), s["slot"], cap)
    _store(s["v"], s["new_v"], s["slot"], cap)
    one, nodes = torch.arange(b, device=DEV), torch.arange(t, device=DEV)
    parent, drafted, target = s["parent"].long(), s["drafted"], s["target"]
    path = torch.full((b, t), -1, dtype=torch.long, device=DEV)
    path[:, 0] = 0
    cur, live, n = torch.zeros(b, dtype=torch.long, device=DEV), torch.ones(b, dtype=torch.bool, device=DEV), torch.ones(b, dtype=torch.long, device=DEV)
    for i in range(1, t):                        # every sequence goes down one node at a time
        fits = (parent == cur[:, None]) & (drafted == target[one, cur][:, None]) & (nodes[None] > cur[:, None])
        live = live & fits.any(1)
        nxt = torch.where(fits, nodes[None], t).amin(1)
        cur = torch.where(live, nxt, cur)
        path[:, i] = torch.where(live, cur, path[:, i])
        n = n + live
    s["path"].copy_(path)
    s["accepted"].copy_(n)
    s["next"].copy_(target[one, cur])
    s["new_len"].copy_(s["lens"] + n)
    at = path >= 0
    seq, place = one[:, None].expand(b, t)[at], (s["lens"].long()[:, None] + nodes[None])[at]
    for x in (s["k"], s["v"]):
        x[seq, :, place] = x[seq, :, (s["lens"].long()[:, None] + path)[at]]
    return {"path": s["path"], "accepted": s["accepted"], "next": s["next"], "new_len": s["new_len"], "k": s["k"], "v": s["v"]}


_own = {"rotary": _own_rotary, "prompt": _own_prompt, "tree": _own_tree, "accept": _own_accept}
_plain = {"rotary": _plain_rotary, "prompt": _plain_prompt, "tree": _plain_tree, "accept": _plain_accept}


# ---------------------------------------------------------------------------- the definition, 64 bits

def _frequency64(rot, scaling):
    """Radians per position of every pair, one at a time."""
    a, f = SCALING[scaling], []
    for c in range(rot // 2):
        base = THETA if scaling != "base" else THETA * a["factor"] ** (rot / (rot - 2.0))
        w = math.exp(-2.0 * c / rot * math.log(base))
        if scaling == "linear":
            w /= a["factor"]
        elif scaling == "parts":
            lo = rot / 2.0 * math.log(a["original_len"] / (2 * math.pi * a["turns_high"]), THETA)
            hi = rot / 2.0 * math.log(a["original_len"] / (2 * math.pi * a["turns_low"]), THETA)
            lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rot - 1)
            far = min(1.0, max(0.0, (c - lo) / max(hi - lo, 1e-3)))
            w *= 1.0 - far + far / a["factor"]
        elif scaling == "bands":
            wave = 2 * math.pi / w
            near = min(1.0, max(0.0, (a["original_len"] / wave - a["turns_low"]) / (a["turns_high"] - a["turns_low"])))
            w *= near + (1.0 - near) / a["factor"]
        f.append(w)
    return torch.tensor(f, dtype=torch.float64, device=DEV)


def _rotate64(x, pos, rot, scaling, interleaved, inverse):
    """Pairs as complex numbers, multiplied by the position's."""
    x = x.double()
    head, rest = x[..., :rot], x[..., rot:]
    z = head.unflatten(-1, (rot // 2, 2)) if interleaved else head.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    z = torch.view_as_complex(z.contiguous())
    a = pos.double()[:, None] * _frequency64(rot, scaling)
    m = SCALING[scaling].get("magnitude", 1.0)
    z = torch.view_as_real(z * torch.polar(torch.full_like(a, m), -a if inverse else a))
    z = z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, rest], -1)


def _attend64(out, lse, q, k, v, scale, limit, extra=None):
    """Row by row blocks of one query head: keys below limit[row], and those behind `n` that `extra` names."""
    k, v = k.double(), v.double()
    for r in range(0, q.shape[0], 2048):
        x = (q[r:r + 2048].double() * scale) @ k.t().contiguous()
        hide = torch.arange(k.shape[0], device=DEV)[None] >= limit[r:r + 2048, None]
        if extra is not None:
            hide[:, -extra.shape[1]:] &= ~extra[r:r + 2048]
        x[hide] = float("-inf")
        e = torch.logsumexp(x, -1)
        p = torch.exp(x - torch.where(e == float("-inf"), torch.zeros_like(e), e)[:, None])
        out[r:r + 2048], lse[r:r + 2048] = p @ v, e


def _exact_prompt(s, c):
    out, lse = torch.full(s["q"].shape, LEFT, dtype=torch.float64, device=DEV), torch.full(s["lse"].shape, LEFT, dtype=torch.float64, device=DEV)
    lens = _numbers(c["lens"])
    qs, ks = _starts(lens), _starts([n + c["prefix"] for n in lens])
    for i, n in enumerate(lens):
        limit = torch.arange(n, device=DEV) + 1 + c["prefix"]
        for h in range(c["hq"]):
            g = h * c["hkv"] // c["hq"]
            a, b = slice(qs[i], qs[i] + n), slice(ks[i], ks[i + 1])
            _attend64(out[h, a], lse[h, a], s["q"][h, a], s["k"][g, b], s["v"][g, b], s["scale"], limit)
    return {"out": out, "lse": lse}


def _exact_tree(s, c):
    out, lse = torch.full(s["q"].shape, LEFT, dtype=torch.float64, device=DEV), torch.full(s["lse"].shape, LEFT, dtype=torch.float64, device=DEV)
    for i, n in enumerate(_numbers(c["lens"])):
        m = s["count_list"][i]
        if not m:
            continue
        sees = np.zeros((m, m), bool)
        for j in range(m):
            up = j
            while up >= 0:
                sees[j, up] = True
                up = up - 1 if s["parent"] is None else int(s["parent"][i, up])
        sees, limit = torch.from_numpy(sees).to(DEV), torch.full((m,), n, device=DEV)
        for h in range(c["hq"]):
            g = h * c["hkv"] // c["hq"]
            _attend64(out[i, h, :m], lse[i, h, :m], s["q"][i, h, :m], s["k"][i, g, :n + m], s["v"][i, g, :n + m], s["scale"], limit, sees)
    return {"out": out, "lse": lse}


def _exact_rotary(s, c):
    turn = lambda x: _rotate64(x, s["pos"], c["rot"], c["scaling"], c["interleaved"], c["inverse"])  # noqa: E731
    q, k = turn(s["q"]), turn(s["k"])
    if s["slot"] is None:
        return {"q": q, "k": k, "v": None}
    cap = s["k_out"].shape[2]
    caches = [torch.full(s["k_out"].shape, LEFT, dtype=torch.float64, device=DEV) for _ in range(2)]
    for i, w in enumerate(s["slot"].tolist()):
        if 0 <= w < caches[0].shape[0] * cap:
            caches[0][w // cap, :, w % cap] = k[:, i]
            caches[1][w // cap, :, w % cap] = s["v"][:, i].double()
    return {"q": q, "k": caches[0], "v": caches[1]}


def _exact_accept(s, c):
    k, v = s["k"].double(), s["v"].double()
    turned = _rotate64(s["new_k"], s["pos"], c["d"], "none", False, False)
    parent, drafted, target, lens = (s[x].tolist() for x in ("parent", "drafted", "target", "lens"))
    t = c["nodes"]
    path = [[-1] * t for _ in lens]
    accepted, following = [], []
    for i, n in enumerate(lens):
        rows = slice(i * t, (i + 1) * t)
        k[i, :, n:n + t], v[i, :, n:n + t] = turned[:, rows], s["new_v"][:, rows].double()
        way = [0]
        while True:
            fits = [j for j in range(way[-1] + 1, t) if parent[i][j] == way[-1] and drafted[i][j] == target[i][way[-1]]]
            if not fits:
                break
            way.append(fits[0])
        path[i][:len(way)] = way
        accepted.append(len(way))
        following.append(target[i][way[-1]])
        at = torch.tensor(way, device=DEV) + n
        k[i, :, n:n + len(way)], v[i, :, n:n + len(way)] = k[i][:, at], v[i][:, at]
    return {"path": _i32(path), "accepted": _i32(accepted), "next": _i32(following),
            "new_len": _i32([a + b for a, b in zip(lens, accepted)]), "k": k, "v": v}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "prompt": _exact_prompt, "tree": _exact_tree, "accept": _exact_accept}[case["kind"]](s, case)


# ------------------------------------------------------------------------------------ what it takes

def work(case):
    """Inputs read once, outputs written once; products of the visible pairs."""
    c, e = case, SIZE[case["dtype"]]
    if c["kind"] == "rotary":
        rows = 2.0 * (c["hq"] + c["hkv"] * (2 if c["blocks"] else 1))
        return {"bytes": e * c["d"] * c["n"] * rows + c["n"] * (8.0 if c["blocks"] else 4.0),
                "flops": 3.0 * c["rot"] * c["n"] * (c["hq"] + c["hkv"])}
    if c["kind"] == "prompt":
        lens = _numbers(c["lens"])
        pairs = sum(n * c["prefix"] + n * (n + 1) / 2.0 for n in lens)
        nq, nk = sum(lens), sum(n + c["prefix"] for n in lens)
        return {"bytes": 2.0 * e * c["d"] * (c["hq"] * nq + c["hkv"] * nk) + 4.0 * c["hq"] * nq,
                "flops": 4.0 * c["d"] * c["hq"] * pairs}
    if c["kind"] == "tree":
        lens, counts = _numbers(c["lens"]), _counts(c)
        keys = sum(n + m for n, m in zip(lens, counts) if m)
        pairs = sum(m * n + m for n, m in zip(lens, counts))
        return {"bytes": 2.0 * e * c["d"] * (c["hkv"] * keys + c["hq"] * sum(counts)) + 4.0 * c["hq"] * sum(counts),
                "flops": 4.0 * c["d"] * c["hq"] * pairs}
    rows, h = float(c["seqs"] * c["nodes"]), c["hkv"]
    moved = float(c["seqs"] * (c["agree"] - 1))
    return {"bytes": e * c["d"] * h * 4.0 * (rows + moved) + rows * 20.0 + 4.0 * rows, "flops": 3.0 * c["d"] * rows * h}
