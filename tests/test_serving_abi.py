"""The serving calls reject bad arguments on the host, before anything could be launched (no GPU is needed: no call
here gets past its checks), and sizes of nothing do nothing."""
import ctypes

import pytest
import torch

from paper_2506_01215_amd import binding

FAKE = 0x1000
size = ctypes.sizeof


def rotary(**kw):
    base = dict(struct_size=size(binding.RotaryDesc), dtype=1, n_tokens=10, n_q_heads=4, n_kv_heads=2, head_dim=128, rotary_dim=128,
                pairs=0, inverse=0, scaling=0, theta=1e4, factor=1.0, turns_high=32.0, turns_low=1.0, original_len=0, magnitude=1.0,
                block_len=0, n_blocks=0, block_stride=0, q_head_stride=1280, q_row_stride=128, k_head_stride=1280, k_row_stride=128,
                v_head_stride=1280, v_row_stride=128, q_out_head_stride=1280, q_out_row_stride=128, kv_out_head_stride=1280,
                kv_out_row_stride=128)
    return binding.RotaryDesc(**{**base, **kw})


def call_rotary(d, q=FAKE, k=FAKE, v=FAKE, pos=FAKE, slot=None, qo=2 * FAKE, ko=2 * FAKE, vo=2 * FAKE):
    return binding.load_library().reform_rotary_embed(ctypes.byref(d), q, k, v, pos, slot, qo, ko, vo, None)


@pytest.mark.parametrize("field,value,status", [
    ("struct_size", 8, 1), ("dtype", 2, 1), ("n_tokens", -1, 1), ("n_q_heads", -1, 1), ("head_dim", 0, 1), ("rotary_dim", 130, 1),
    ("rotary_dim", 7, 1), ("rotary_dim", -2, 1), ("pairs", 2, 1), ("inverse", 2, 1), ("scaling", 5, 1), ("scaling", -1, 1),
    ("theta", 1.0, 1), ("theta", float("inf"), 1), ("theta", float("nan"), 1), ("magnitude", 0.0, 1), ("magnitude", float("nan"), 1),
    ("q_head_stride", -128, 1), ("q_out_row_stride", 64, 1), ("q_out_head_stride", 64, 1), ("kv_out_head_stride", 0, 1),
    ("rotary_dim", 8, 2), ("rotary_dim", 24, 2), ("head_dim", 1024, 2), ("k_row_stride", 132, 2), ("n_kv_heads", 40000, 2),
])
def test_rotary_rejects(field, value, status):
    d = rotary()
    setattr(d, field, value)
    if field == "head_dim" and value == 1024:
        d.q_out_row_stride = d.kv_out_row_stride = 1024
        d.q_out_head_stride = d.kv_out_head_stride = 10240
    assert call_rotary(d) == status


def test_rotary_rejects_scalings_pointers_and_slots():
    for kw in (dict(scaling=1, factor=0.5), dict(scaling=2, factor=float("nan")), dict(scaling=3, factor=2.0, original_len=0),
               dict(scaling=3, factor=2.0, original_len=9, turns_low=0.0), dict(scaling=4, factor=2.0, original_len=9, turns_high=1.0),
               dict(scaling=4, factor=2.0, original_len=9, turns_high=float("inf"))):
        assert call_rotary(rotary(**kw)) == 1
    assert call_rotary(rotary(dtype=0, rotary_dim=2, scaling=2, factor=2.0, pairs=1)) == 1      # theta' has no value
    assert call_rotary(rotary(pairs=1, rotary_dim=4)) == 2
    for kw in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(vo=None), dict(v=None), dict(pos=None)):
        assert call_rotary(rotary(), **kw) == 1
    assert call_rotary(rotary(n_kv_heads=0)) == 1                       # keys where there are none
    assert call_rotary(rotary(), q=FAKE + 8) == 2
    assert call_rotary(rotary(), qo=2 * FAKE + 4) == 2
    assert call_rotary(rotary(q_row_stride=256), qo=FAKE) == 1          # in place in another layout
    assert call_rotary(rotary(k_row_stride=256), ko=FAKE) == 1
    ok = dict(block_len=64, n_blocks=2, block_stride=2 * 64 * 128, kv_out_head_stride=64 * 128)
    assert call_rotary(rotary(**ok), slot=FAKE, ko=FAKE) == 1           # in place with slots
    for kw, rc in ((dict(block_len=0), 1), (dict(n_blocks=0), 1), (dict(block_stride=-8), 1), (dict(block_stride=64), 1),
                   (dict(block_stride=2 * 64 * 128 + 4), 2), (dict(kv_out_head_stride=128), 1),
                   (dict(block_len=1 << 20, n_blocks=1 << 12, kv_out_head_stride=1 << 27), 2)):
        assert call_rotary(rotary(**{**ok, **kw}), slot=FAKE) == rc, kw
    assert call_rotary(rotary(n_tokens=1 << 28, q_out_head_stride=1 << 40, kv_out_head_stride=1 << 40)) == 2
    none = rotary(n_tokens=0)
    assert call_rotary(none, None, None, None, None, None, None, None, None) == 0


def prompt(**kw):
    base = dict(struct_size=size(binding.PromptDesc), dtype=1, n_q_heads=8, n_kv_heads=2, head_dim=128, n_seq=2, n_q_rows=100, n_k_rows=100,
                scale=0.1, reserved=0, q_head_stride=12800, q_row_stride=128, k_head_stride=12800, k_row_stride=128,
                v_head_stride=12800, v_row_stride=128, o_head_stride=12800, o_row_stride=128)
    return binding.PromptDesc(**{**base, **kw})


def call_prompt(d, q=FAKE, k=FAKE, v=FAKE, cu=FAKE, out=FAKE):
    return binding.load_library().reform_prompt_attend(ctypes.byref(d), q, k, v, cu, None, out, None, None, 0, None)


@pytest.mark.parametrize("field,value,status", [
    ("struct_size", 4, 1), ("dtype", 3, 1), ("n_kv_heads", 3, 1), ("n_kv_heads", 0, 1), ("n_seq", -1, 1), ("n_q_rows", -1, 1),
    ("n_k_rows", -1, 1), ("scale", 0.0, 1), ("scale", float("nan"), 1), ("reserved", 1, 1), ("q_head_stride", -8, 1),
    ("k_row_stride", 132, 1), ("o_row_stride", 64, 1), ("o_head_stride", 128, 1), ("head_dim", 96, 2), ("head_dim", 256, 2),
    ("n_seq", 65537, 2), ("n_k_rows", 1 << 29, 2), ("n_q_rows", 1 << 24, 2), ("k_row_stride", 1 << 24, 2), ("v_row_stride", 1 << 25, 2),
])
def test_prompt_rejects(field, value, status):
    d = prompt()
    setattr(d, field, value)
    if field == "head_dim":
        d.o_row_stride, d.o_head_stride = 256, 25600
    if field == "n_q_rows" and value > 0:
        d.o_head_stride = value * 128
    assert call_prompt(d) == status


def test_prompt_rejects_pointers_and_types():
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(cu=None), dict(out=None), dict(q=FAKE + 8), dict(out=FAKE + 2)):
        assert call_prompt(prompt(), **kw) == 1
    assert call_prompt(prompt(dtype=0, head_dim=130, o_row_stride=132, o_head_stride=13200)) == 2
    assert call_prompt(prompt(dtype=0, head_dim=260, o_row_stride=260, o_head_stride=26000)) == 2
    assert call_prompt(prompt(n_q_rows=0), None, None, None, None, None) == 0
    assert call_prompt(prompt(n_seq=0), None, None, None, None, None) == 0


def tree(**kw):
    base = dict(struct_size=size(binding.TreeDesc), dtype=1, n_seq=3, n_q_heads=8, n_kv_heads=2, head_dim=128, n_nodes=5, max_cache_len=5000,
                capacity=5005, scale=0.1, q_seq_stride=5120, q_head_stride=640, q_row_stride=128, o_seq_stride=5120, o_head_stride=640,
                o_row_stride=128, kv_seq_stride=2 * 5005 * 128, kv_head_stride=5005 * 128)
    return binding.TreeDesc(**{**base, **kw})


def call_tree(d, q=FAKE, k=FAKE, v=FAKE, lens=FAKE, out=FAKE, ws=None, nbytes=0):
    return binding.load_library().reform_tree_attend(ctypes.byref(d), q, k, v, lens, None, None, out, None, ws, nbytes, None)


@pytest.mark.parametrize("field,value,status", [
    ("struct_size", 4, 1), ("dtype", -1, 1), ("n_kv_heads", 3, 1), ("n_seq", -1, 1), ("n_nodes", 0, 1), ("max_cache_len", -1, 1),
    ("max_cache_len", 5001, 1), ("capacity", 5004, 1), ("scale", -1.0, 1), ("q_row_stride", 4, 1), ("kv_seq_stride", -128, 1),
    ("o_row_stride", 64, 1), ("o_head_stride", 128, 1), ("o_seq_stride", 64, 1), ("head_dim", 96, 2), ("n_seq", 1 << 28, 2),
])
def test_tree_rejects(field, value, status):
    d = tree()
    setattr(d, field, value)
    lib = binding.load_library()
    assert lib.reform_tree_attend_workspace(ctypes.byref(d)) == 0
    assert call_tree(d) == status


def test_tree_rejects_pointers_nodes_and_workspaces():
    lib = binding.load_library()
    assert call_tree(tree(n_nodes=65, capacity=6000, o_head_stride=65 * 128)) == 2
    assert call_tree(tree(n_seq=1 << 17, o_seq_stride=1 << 20)) == 2
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(lens=None), dict(out=None), dict(k=FAKE + 8)):
        assert call_tree(tree(), **kw) == 1
    need = lib.reform_tree_attend_workspace(ctypes.byref(tree()))
    assert need > 0
    assert call_tree(tree()) == 3
    assert call_tree(tree(), ws=FAKE, nbytes=need - 1) == 3
    assert call_tree(tree(), ws=FAKE + 16, nbytes=need) == 3
    assert lib.reform_tree_attend_workspace(ctypes.byref(tree(max_cache_len=100))) == 0       # short caches are not shared out
    assert call_tree(tree(n_seq=0), None, None, None, None, None) == 0
    # the workspace's size follows the longest cache, not the capacity
    assert lib.reform_tree_attend_workspace(ctypes.byref(tree(capacity=1 << 20))) == need


def accept(**kw):
    base = dict(struct_size=size(binding.AcceptDesc), dtype=1, n_seq=3, n_kv_heads=2, head_dim=128, n_nodes=5, capacity=100, n_layers=1,
                kv_seq_stride=2 * 12800, kv_head_stride=12800, kv_layer_stride=0)
    return binding.AcceptDesc(**{**base, **kw})


def call_accept(d, drafted=FAKE, target=FAKE, lens=FAKE, k=FAKE, v=2 * FAKE, new_len=None):
    return binding.load_library().reform_tree_accept(ctypes.byref(d), None, drafted, target, lens, None, k, v, None, None, None, new_len, None)


@pytest.mark.parametrize("field,value,status", [
    ("struct_size", 4, 1), ("dtype", 9, 1), ("n_seq", -1, 1), ("n_kv_heads", 0, 1), ("head_dim", 0, 1), ("n_layers", 0, 1), ("n_nodes", 0, 1),
    ("capacity", 4, 1), ("kv_head_stride", 128, 1), ("kv_seq_stride", -16, 1), ("kv_seq_stride", 128, 1), ("n_layers", 2, 1),
    ("head_dim", 4, 2), ("n_nodes", 65, 2), ("kv_head_stride", 12804, 2),
])
def test_accept_rejects(field, value, status):
    d = accept()
    setattr(d, field, value)
    assert call_accept(d) == status


def test_accept_rejects_pointers():
    for kw in (dict(drafted=None), dict(target=None), dict(lens=None), dict(k=None), dict(v=None), dict(k=2 * FAKE), dict(new_len=FAKE)):
        assert call_accept(accept(), **kw) == 1
    assert call_accept(accept(), k=FAKE + 8) == 2
    assert call_accept(accept(head_dim=4096, capacity=8, kv_head_stride=1 << 20, kv_seq_stride=1 << 24)) == 2
    assert call_accept(accept(n_seq=1 << 20, kv_seq_stride=1 << 20, n_kv_heads=8)) == 2
    assert call_accept(accept(n_seq=0), None, None, None) == 0


def test_host_tensors_are_refused():
    """A tensor that is not on the current GPU raises before its address could be used."""
    z = torch.zeros
    i = lambda *s: z(s, dtype=torch.int32)  # noqa: E731
    q, kv = z(4, 3, 64), z(2, 3, 64)
    calls = [lambda: binding.reform_rotary_embed(q, kv, kv, i(3)),
             lambda: binding.reform_prompt_attend(q, kv, kv, i(2), 0.1),
             lambda: binding.reform_tree_attend(z(1, 4, 3, 64), z(1, 2, 9, 64), z(1, 2, 9, 64), i(1), 0.1),
             lambda: binding.reform_tree_accept(None, i(1, 3), i(1, 3), i(1))]
    for call in calls:
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            call()


def test_shapes_are_checked():
    z = torch.zeros
    i = lambda *s: z(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        binding.reform_rotary_embed(z(4, 3, 64), z(2, 4, 64), None, i(3))
    with pytest.raises(ValueError):
        binding.reform_rotary_embed(z(4, 3, 64), z(2, 3, 64), None, i(3), slot=i(3))          # no cache for the slots
    with pytest.raises(ValueError):
        binding.prompt_desc(z(4, 3, 64), z(2, 3, 32), z(2, 3, 32), z(4, 3, 64), i(2), 0.1)
    with pytest.raises(ValueError):
        binding.tree_desc(z(2, 4, 3, 64), z(1, 2, 9, 64), z(1, 2, 9, 64), z(2, 4, 3, 64), 0.1)
    with pytest.raises(TypeError, match="float16"):
        binding.reform_rotary_embed(z(4, 3, 64, dtype=torch.float16), None, None, i(3))
    with pytest.raises(TypeError, match="float16"):
        binding.prompt_desc(*(z(2, 3, 64, dtype=torch.float16) for _ in range(4)), i(2), 0.1)
    with pytest.raises(ValueError, match="cubic"):
        binding.reform_rotary_embed(z(4, 3, 64), None, None, i(3), q_out=z(4, 3, 64), scaling="cubic")


def test_outputs_that_overlap_are_refused():
    """Strides under which two rows of an output would share memory, and one tensor in two places."""
    # sequences inside one another's heads, heads inside one another's rows
    assert call_tree(tree(o_seq_stride=640)) == 1
    assert call_tree(tree(o_seq_stride=128, o_row_stride=384, o_head_stride=1920), ws=None) == 3       # [heads][nodes][sequences]: apart
    assert call_tree(tree(o_seq_stride=128, o_row_stride=256, o_head_stride=1920)) == 1
    # a paged cache whose blocks begin inside the heads of the one before; heads outside the blocks are apart
    paged = dict(block_len=64, n_blocks=3, kv_out_head_stride=64 * 128)
    assert call_rotary(rotary(**paged, block_stride=64 * 128), slot=FAKE, vo=3 * FAKE) == 1
    outside = rotary(n_tokens=1 << 28, block_len=64, n_blocks=3, kv_out_head_stride=3 * 64 * 128, block_stride=64 * 128,
                     q_out_head_stride=1 << 40)
    assert call_rotary(outside, slot=FAKE, ko=3 * FAKE, vo=4 * FAKE) == 2                              # refused for its tokens alone
    for kw in (dict(ko=2 * FAKE, vo=3 * FAKE), dict(ko=3 * FAKE, vo=2 * FAKE), dict(ko=3 * FAKE, vo=3 * FAKE)):
        assert call_rotary(rotary(), qo=2 * FAKE, **kw) == 1
    # two sequences' caches in each other's heads, layers inside a sequence
    assert call_accept(accept(kv_seq_stride=12800)) == 1
    assert call_accept(accept(n_layers=2, kv_layer_stride=2 * 12800)) == 1
    lib = binding.load_library()
    for at in range(4):
        outs = [None] * 4
        for taken in (FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE):                                   # an input
            outs[at] = taken
            assert lib.reform_tree_accept(ctypes.byref(accept()), FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE, None, None, *outs, None) == 1
        outs[at] = outs[at - 1] = 6 * FAKE                                                             # another output
        assert lib.reform_tree_accept(ctypes.byref(accept()), FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE, None, None, *outs, None) == 1


def test_prompts_that_need_a_workspace():
    lib = binding.load_library()
    many = prompt(n_q_rows=3, n_k_rows=20000, k_head_stride=20000 * 128, v_head_stride=20000 * 128)
    need = lib.reform_prompt_attend_workspace(ctypes.byref(many))
    assert need > 0 and call_prompt(many) == 3
    for ws, nbytes in ((FAKE, need - 1), (FAKE + 16, need)):
        assert lib.reform_prompt_attend(ctypes.byref(many), FAKE, FAKE, FAKE, FAKE, None, FAKE, None, ws, nbytes, None) == 3
    for kw in (dict(n_q_rows=0), dict(n_seq=0), dict(n_q_rows=100), dict(n_seq=65), dict(scale=0.0)):
        assert lib.reform_prompt_attend_workspace(ctypes.byref(prompt(**kw))) == 0
