"""GPU: reform_rotary_embed against the 64-bit definition: both pairings, parts of the head, scaled positions,
in place, into caches by slots, inverse, odd sizes and strides."""
import math
import random

import pytest
import torch

import serving_reference as ref
from paper_2506_01215_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SCALED = {
    None: {},
    "linear": dict(scaling="linear", factor=4.0),
    "base": dict(scaling="base", factor=3.0),
    "parts": dict(scaling="parts", factor=16.0, original_len=4096, turns_high=32.0, turns_low=1.0),
    "bands": dict(scaling="bands", factor=8.0, original_len=8192, turns_high=4.0, turns_low=1.0),
}


def case(n, hq, hkv, d, dtype, far, seed):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (ref.randn(g, h, n, d, dtype=dtype) for h in (hq, hkv, hkv))
    pos = torch.randint(-far // 7, far, (n,), generator=g).int()
    return q, k, v, pos


@pytest.mark.parametrize("n,hq,hkv,d,rot,dtype,adjacent,inverse,scaling,far", [
    (1, 32, 8, 128, 128, torch.bfloat16, False, False, None, 2000000),
    (1, 1, 1, 64, 64, torch.float32, True, False, "bands", 1000),
    (77, 14, 2, 64, 32, torch.bfloat16, False, True, "parts", 300000),
    (77, 14, 2, 64, 32, torch.bfloat16, True, False, "parts", 300000),
    (300, 3, 3, 96, 48, torch.float32, False, False, "linear", 5000),
    (129, 5, 1, 72, 8, torch.float32, True, True, "base", 5000),
    (513, 8, 4, 256, 64, torch.bfloat16, True, False, "base", 100000),
    (65, 2, 1, 512, 512, torch.float32, False, False, "bands", 100000),
    (40, 4, 2, 80, 24, torch.bfloat16, True, False, None, 4000),       # three pieces turn, seven do not
    (33, 2, 2, 128, 0, torch.bfloat16, False, False, None, 4000),      # nothing turns: a copy
    (1025, 9, 3, 128, 128, torch.bfloat16, False, False, "linear", 1 << 30),
])
def test_matches_definition(n, hq, hkv, d, rot, dtype, adjacent, inverse, scaling, far):
    q, k, v, pos = case(n, hq, hkv, d, dtype, far, n + d)
    mag = 1.25 if scaling == "parts" else 1.0
    kw = dict(SCALED[scaling], theta=500000.0)
    freq = ref.frequencies(rot, **kw)
    print(f"[rotary] n={n} heads={hq}/{hkv} d={d} rot={rot} {dtype} adjacent={adjacent} {scaling}", flush=True)
    qo, ko, vo = binding.reform_rotary_embed(q.to(DEV), k.to(DEV), v.to(DEV), pos.to(DEV), rotary_dim=rot, interleaved=adjacent,
                                             inverse=inverse, magnitude=mag, **kw)
    for got, x in ((qo, q), (ko, k)):
        want, size = ref.rotary(x, pos, rot, freq, adjacent, inverse, mag)
        ref.check_rotary(got, want, size, dtype, mag)
    assert torch.equal(vo.cpu(), v)


@pytest.mark.parametrize("dtype,adjacent,rot", [(torch.bfloat16, False, 64), (torch.float32, True, 128)])
def test_in_place_leaves_the_rest(dtype, adjacent, rot):
    """The same tensors in and out, as views of one token-major projection."""
    n, hq, hkv, d = 61, 6, 2, 128
    g = torch.Generator().manual_seed(5)
    qkv = ref.randn(g, n, hq + 2 * hkv, d, dtype=dtype)
    pos = torch.randint(0, 9000, (n,), generator=g).int()
    dev = qkv.to(DEV)
    q, k, v = (dev[:, a:b].transpose(0, 1) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    binding.reform_rotary_embed(q, k, v, pos.to(DEV), rotary_dim=rot, interleaved=adjacent, q_out=q, k_out=k, v_out=v)
    want, size = ref.rotary(qkv[:, :hq + hkv].transpose(0, 1), pos, rot, ref.frequencies(rot, 10000.0), adjacent)
    ref.check_rotary(dev[:, :hq + hkv].transpose(0, 1), want, size, dtype)
    assert torch.equal(dev[:, hq + hkv:].cpu(), qkv[:, hq + hkv:])
    assert torch.equal(dev[:, :hq + hkv, rot:].cpu(), qkv[:, :hq + hkv, rot:])


def test_slots_into_caches():
    """Keys and values to rows of four caches, padding tokens to none, everything else untouched; queries are
    rotated all the same."""
    n, hq, hkv, d, blocks, cap = 90, 4, 2, 64, 4, 37
    q, k, v, pos = case(n, hq, hkv, d, torch.bfloat16, 70000, 11)
    rnd = random.Random(3)
    slot = rnd.sample(range(blocks * cap), n)
    for i, bad in ((5, -1), (17, blocks * cap), (40, -(1 << 31)), (89, (1 << 31) - 1)):
        slot[i] = bad
    kc = torch.full((blocks, hkv, cap, d), 3.0, dtype=torch.bfloat16, device=DEV)
    vc = torch.full_like(kc, -3.0)
    want_k, want_v = kc.cpu().clone(), vc.cpu().clone()
    qo, _, _ = binding.reform_rotary_embed(q.to(DEV), k.to(DEV), v.to(DEV), pos.to(DEV), theta=1e6,
                                           slot=torch.tensor(slot, dtype=torch.int32, device=DEV), k_out=kc, v_out=vc)
    freq = ref.frequencies(d, 1e6)
    wq, sq = ref.rotary(q, pos, d, freq)
    ref.check_rotary(qo, wq, sq, torch.bfloat16)
    turned, size = ref.rotary(k, pos, d, freq)
    got = kc.cpu()
    for i, w in enumerate(slot):
        if 0 <= w < blocks * cap:
            ref.check_rotary(got[w // cap, :, w % cap], turned[:, i], size[:, i], torch.bfloat16, what=f"token {i}")
            want_k[w // cap, :, w % cap] = got[w // cap, :, w % cap]
            want_v[w // cap, :, w % cap] = v[:, i]
    assert torch.equal(got, want_k) and torch.equal(vc.cpu(), want_v)
    one = torch.zeros((hkv, 2 * n, d), dtype=torch.bfloat16, device=DEV)       # a single cache, keys alone
    binding.reform_rotary_embed(None, k.to(DEV), None, pos.to(DEV), theta=1e6, k_out=one,
                                slot=torch.arange(n, dtype=torch.int32, device=DEV) + 50)
    ref.check_rotary(one[:, 50:50 + n], turned, size, torch.bfloat16)
    assert not bool(one[:, :50].any()) and not bool(one[:, 50 + n:].any())


def test_broadcast_inputs_and_large_row_stride():
    """One head's states for all heads (stride 0), rows far apart."""
    n, d = 19, 64
    g = torch.Generator().manual_seed(8)
    wide = ref.randn(g, n, 40 * d)
    pos = torch.arange(n).int()
    x = wide.to(DEV)[:, 3 * d:4 * d].unsqueeze(0).expand(5, n, d)
    qo, _, _ = binding.reform_rotary_embed(x, None, None, pos.to(DEV))
    want, size = ref.rotary(wide[None, :, 3 * d:4 * d].expand(5, n, d), pos, d, ref.frequencies(d, 10000.0))
    ref.check_rotary(qo, want, size, torch.float32)
    empty = torch.zeros((4, 0, d), device=DEV)
    assert binding.reform_rotary_embed(empty, None, None, pos[:0].to(DEV))[0].shape == (4, 0, d)


@pytest.mark.parametrize("adjacent,scaling", [(False, None), (True, "parts")])
def test_inverse_is_the_gradient(adjacent, scaling):
    """inverse = 1 takes the gradient of sum(w * y) with respect to y to that with respect to x: against the
    64-bit formula's (autograd of the definition) and against differences of the call itself."""
    n, h, d, rot = 23, 3, 64, 32
    kw = dict(SCALED[scaling], theta=10000.0)
    mag = 1.25 if scaling else 1.0
    q, _, _, pos = case(n, h, 1, d, torch.float32, 9000, 2)
    g = torch.Generator().manual_seed(9)
    w = ref.randn(g, h, n, d)
    x = q.double().requires_grad_()
    freq = ref.frequencies(rot, **kw)
    (ref.rotary(x, pos, rot, freq, adjacent, False, mag)[0] * w.double()).sum().backward()
    call = lambda t, inv: binding.reform_rotary_embed(t.to(DEV), None, None, pos.to(DEV), rotary_dim=rot, interleaved=adjacent,  # noqa: E731
                                                      inverse=inv, magnitude=mag, **kw)[0]
    grad = call(w, True)
    _, size = ref.rotary(w, pos, rot, freq, adjacent, True, mag)
    ref.check_rotary(grad, x.grad, size, torch.float32, mag)
    step = ref.randn(g, h, n, d)
    # the map is linear: a difference over a whole step is the derivative but for rounding, 4 * 2^-23 of each of the
    # h n d terms' size on both sides
    diff = ((call(q + step, False).double() - call(q, False).double()).cpu() * w.double()).sum()
    along = (grad.double().cpu() * step.double()).sum()
    scale = float((w.double().abs() * (q.double().abs() + step.double().abs() + 1)).sum()) * 8
    assert abs(float(diff - along)) <= 8 * 2.0 ** -23 * mag * scale
    # and with 1 / magnitude it takes the rotation back
    back = binding.reform_rotary_embed(call(q, False), None, None, pos.to(DEV), rotary_dim=rot, interleaved=adjacent, inverse=True,
                                       magnitude=1 / mag, **kw)[0]
    assert float((back.cpu() - q).abs().max()) <= 16 * 2.0 ** -23 * mag * float(q.abs().max()) * 2 / min(mag, 1.0)
    assert math.isfinite(float(diff))
