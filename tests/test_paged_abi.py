"""The calls on sliding windows and on caches in pages reject bad arguments on the host, before anything could be launched (no GPU
is needed: no call here gets past its checks), and sizes of nothing do nothing."""
import ctypes

import pytest
import torch

from paper_2506_01215_amd import binding

FAKE = 0x1000
size = ctypes.sizeof


def lib():
    return binding.load_library()


def window(**kw):
    base = dict(struct_size=size(binding.WindowDesc), dtype=1, n_q_heads=8, n_kv_heads=2, head_dim=128, n_seq=2, n_q_rows=100, n_k_rows=100,
                scale=0.1, window=16, n_sink=4, reserved=0, q_head_stride=12800, q_row_stride=128, k_head_stride=12800, k_row_stride=128,
                v_head_stride=12800, v_row_stride=128, o_head_stride=12800, o_row_stride=128)
    return binding.WindowDesc(**{**base, **kw})


def call_window(d, q=FAKE, k=FAKE, v=FAKE, cu=FAKE, out=2 * FAKE):
    return lib().reform_window_attend(ctypes.byref(d), q, k, v, cu, None, out, None, None, 0, None)


@pytest.mark.parametrize("field,value,status", [
    ("struct_size", 4, 1), ("dtype", 3, 1), ("n_kv_heads", 3, 1), ("n_kv_heads", 0, 1), ("n_seq", -1, 1), ("n_q_rows", -1, 1),
    ("n_k_rows", -1, 1), ("scale", 0.0, 1), ("scale", float("nan"), 1), ("reserved", 1, 1), ("window", 0, 1), ("window", -1, 1),
    ("n_sink", -1, 1), ("q_head_stride", -8, 1), ("k_row_stride", 132, 1), ("o_row_stride", 64, 1), ("o_head_stride", 128, 1),
    ("head_dim", 96, 2), ("head_dim", 256, 2), ("n_seq", 65537, 2), ("n_k_rows", 1 << 29, 2), ("n_q_rows", 1 << 24, 2),
    ("k_row_stride", 1 << 24, 2), ("v_row_stride", 1 << 25, 2),
])
def test_window_rejects(field, value, status):
    d = window()
    setattr(d, field, value)
    if field == "head_dim":
        d.o_row_stride, d.o_head_stride = 256, 25600
    if field == "n_q_rows" and value > 0:
        d.o_head_stride = value * 128
    assert lib().reform_window_attend_workspace(ctypes.byref(d)) == 0
    assert call_window(d) == status


def test_window_rejects_pointers_and_types():
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(cu=None), dict(out=None), dict(q=FAKE + 8), dict(out=FAKE + 2), dict(out=FAKE)):
        assert call_window(window(), **kw) == 1
    assert call_window(window(dtype=0, head_dim=130, o_row_stride=132, o_head_stride=13200)) == 2
    assert call_window(window(dtype=0, head_dim=260, o_row_stride=260, o_head_stride=26000)) == 2
    assert call_window(window(n_q_rows=0), None, None, None, None, None) == 0
    assert call_window(window(n_seq=0), None, None, None, None, None) == 0
    assert lib().reform_window_attend(None, FAKE, FAKE, FAKE, FAKE, None, FAKE, None, None, 0, None) == 1


def paged(**kw):
    base = dict(struct_size=size(binding.PagedDesc), dtype=1, n_seq=3, n_q_heads=8, n_kv_heads=2, head_dim=128, page_len=16, n_pages=500,
                max_pages=400, max_len=6400, window=0, n_sink=0, want_score=0, accumulate=0, scale=0.1, reserved=0, q_seq_stride=1024,
                q_head_stride=128, o_seq_stride=1024, o_head_stride=128, kv_page_stride=2 * 16 * 128, kv_head_stride=16 * 128,
                kv_row_stride=128, table_stride=400, score_seq_stride=12800, score_head_stride=6400)
    return binding.PagedDesc(**{**base, **kw})


def call_paged(d, q=FAKE, k=FAKE, v=FAKE, table=FAKE, lens=FAKE, score=None, out=2 * FAKE, ws=None, nbytes=0):
    return lib().reform_paged_attend(ctypes.byref(d), q, k, v, table, lens, score, out, None, ws, nbytes, None)


@pytest.mark.parametrize("field,value,status", [
    ("struct_size", 4, 1), ("dtype", -1, 1), ("n_kv_heads", 3, 1), ("n_seq", -1, 1), ("page_len", 0, 1), ("n_pages", -1, 1),
    ("max_pages", -1, 1), ("max_pages", 399, 1), ("max_len", -1, 1), ("max_len", 6401, 1), ("window", -1, 1), ("n_sink", -1, 1),
    ("want_score", 2, 1), ("accumulate", 2, 1), ("scale", -1.0, 1), ("scale", float("inf"), 1), ("reserved", 1, 1), ("q_head_stride", 4, 1),
    ("kv_page_stride", -128, 1), ("kv_row_stride", 4, 1), ("o_head_stride", 64, 1), ("o_seq_stride", 128, 1), ("table_stride", -1, 1),
    ("score_seq_stride", -1, 1), ("head_dim", 96, 2), ("n_seq", 1 << 20, 2), ("n_pages", 1 << 27, 2), ("kv_row_stride", 1 << 24, 2),
])
def test_paged_rejects(field, value, status):
    d = paged()
    setattr(d, field, value)
    assert lib().reform_paged_attend_workspace(ctypes.byref(d)) == 0
    assert call_paged(d) == status


def test_paged_rejects_pointers_scores_and_sizes():
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(lens=None), dict(out=None), dict(table=None), dict(k=FAKE + 8), dict(out=FAKE + 4),
               dict(score=3 * FAKE), dict(out=FAKE)):
        assert call_paged(paged(), **kw) == 1, kw
    assert call_paged(paged(want_score=1)) == 1                         # a score is wanted and there is none
    assert call_paged(paged(want_score=1), score=2 * FAKE) == 1         # it is the output
    assert call_paged(paged(want_score=1, score_head_stride=6399), score=3 * FAKE) == 1       # heads overlap
    assert call_paged(paged(want_score=1, score_seq_stride=6400), score=3 * FAKE) == 1
    huge = dict(page_len=1 << 20, n_pages=2047, max_pages=2048, kv_head_stride=128 << 20, kv_page_stride=256 << 20)
    assert call_paged(paged(max_len=(1 << 31) - 65535, **huge)) == 2
    assert call_paged(paged(n_seq=0), None, None, None, None, None, None, None) == 0


def test_paged_workspace_follows_what_is_asked_for():
    need = lib().reform_paged_attend_workspace
    plain, score = (need(ctypes.byref(paged(want_score=x))) for x in (0, 1))
    assert score >= plain + 3 * 8 * 6400 * 4                            # the logits
    assert need(ctypes.byref(paged(want_score=1, window=64, n_sink=4))) < score / 20      # of what the window shows
    d = paged(want_score=1)
    assert call_paged(d, score=3 * FAKE) == 3
    assert call_paged(d, score=3 * FAKE, ws=FAKE, nbytes=score - 1) == 3
    assert call_paged(d, score=3 * FAKE, ws=FAKE + 16, nbytes=score) == 3


def evict(**kw):
    base = dict(struct_size=size(binding.PagedEvictDesc), dtype=1, n_seq=3, n_kv_heads=2, head_dim=128, page_len=16, n_pages=500,
                max_pages=400, max_len=6400, budget=4096, n_sink=4, n_recent=64, kv_page_stride=2 * 16 * 128, kv_head_stride=16 * 128,
                kv_row_stride=128, table_stride=400, score_seq_stride=12800, score_head_stride=6400)
    return binding.PagedEvictDesc(**{**base, **kw})


def call_evict(d, k=FAKE, v=2 * FAKE, score=3 * FAKE, table=4 * FAKE, lens=5 * FAKE, new_len=None, ws=None, nbytes=0):
    return lib().reform_paged_evict(ctypes.byref(d), k, v, score, None, table, lens, None, new_len, ws, nbytes, None)


@pytest.mark.parametrize("field,value,status", [
    ("struct_size", 4, 1), ("dtype", 2, 1), ("n_kv_heads", 0, 1), ("n_seq", -1, 1), ("page_len", 0, 1), ("n_pages", -1, 1), ("max_pages", 399, 1),
    ("max_len", 6401, 1), ("budget", 0, 1), ("n_sink", -1, 1), ("n_sink", 4033, 1), ("n_recent", -1, 1), ("n_recent", 4093, 1),
    ("head_dim", 0, 1), ("kv_page_stride", 2048, 1), ("kv_head_stride", 128, 1), ("kv_row_stride", 64, 1), ("score_head_stride", 6399, 1),
    ("score_seq_stride", 6400, 1), ("table_stride", -1, 1), ("n_pages", 1 << 27, 2), ("n_seq", 1 << 22, 2),
])
def test_evict_rejects(field, value, status):
    d = evict()
    setattr(d, field, value)
    if field == "n_seq" and value > 0:
        d.score_seq_stride = 12800
    assert lib().reform_paged_evict_workspace(ctypes.byref(d)) == 0
    assert call_evict(d) == status


def test_evict_rejects_pointers_rows_and_workspaces():
    assert call_evict(evict(max_pages=1 << 28, table_stride=1 << 28, max_len=(1 << 31) - 65535, score_head_stride=1 << 31, score_seq_stride=1 << 32)) == 2
    for kw in (dict(k=None), dict(v=None), dict(score=None), dict(table=None), dict(lens=None), dict(v=FAKE), dict(new_len=5 * FAKE), dict(new_len=3 * FAKE), dict(score=FAKE)):
        assert call_evict(evict(), **kw) == 1, kw
    assert call_evict(evict(), k=FAKE + 8) == 2
    assert call_evict(evict(head_dim=4)) == 2                            # rows of 8 bytes
    wide = dict(head_dim=4096, kv_row_stride=4096, kv_head_stride=4096 * 16, kv_page_stride=4096 * 32)
    assert call_evict(evict(**wide)) == 2
    assert call_evict(evict(kv_row_stride=132, kv_head_stride=132 * 16, kv_page_stride=132 * 32)) == 2
    need = lib().reform_paged_evict_workspace(ctypes.byref(evict()))
    assert need >= 3 * 2 * 4096 * 4
    assert call_evict(evict()) == 3
    assert call_evict(evict(), ws=FAKE, nbytes=need - 1) == 3
    assert call_evict(evict(), ws=FAKE + 16, nbytes=need) == 3
    assert lib().reform_paged_evict_workspace(ctypes.byref(evict(max_len=4096))) == 0      # nobody outgrows the budget
    assert call_evict(evict(n_seq=0), None, None, None, None, None) == 0


def test_binding_rejects_what_does_not_fit():
    q, out = torch.zeros(2, 4, 64), torch.zeros(2, 4, 64)
    k = torch.zeros(5, 2, 16, 64)
    table, lens = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    score = torch.zeros(2, 2, 48)
    paged_call, evict_call = binding.reform_paged_attend, binding.reform_paged_evict
    for bad in (lambda: paged_call(q, k, k, table, lens, 0.1),                                          # host tensors
                lambda: paged_call(q, k, k[:4], table, lens, 0.1), lambda: paged_call(q, k, k.transpose(2, 3), table, lens, 0.1),
                lambda: paged_call(q, k[..., :32], k[..., :32], table, lens, 0.1), lambda: paged_call(q, k.bfloat16(), k.bfloat16(), table, lens, 0.1),
                lambda: paged_call(q, k, k, table.long(), lens, 0.1), lambda: paged_call(q, k, k, table[:1], lens, 0.1),
                lambda: paged_call(q, k, k, table.t().contiguous().t(), lens, 0.1), lambda: paged_call(q, k, k, table, lens, 0.1, out=out[:, :2]),
                lambda: paged_call(q, k, k, table, lens, 0.1, score=score[:, :1]), lambda: paged_call(q, k, k, table, lens, 0.1, score=score.double()),
                lambda: paged_call(q, k, k, table, lens, 0.1, score=score[..., ::2]), lambda: paged_call(q, k, k, table, lens, 0.1, score=score, max_len=49),
                lambda: paged_call(q, k, k, table, lens, 0.1, lse=torch.zeros(2, 5)),
                lambda: evict_call(k, k.clone(), score, table, lens, 8, pos=torch.zeros(2, 2, 48)),
                lambda: evict_call(k, k.clone(), score, table, lens, 8, pos=torch.zeros(2, 2, 47, dtype=torch.int32)),
                lambda: evict_call(k, k.clone(), score, table, lens, 8)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        paged_call(q.half(), k.half(), k.half(), table, lens, 0.1, out=out.half())
    d = binding.paged_desc(q, k, k, out, table, 0.1, score=score[..., :40])
    assert d.max_len == 40 and d.want_score == 1 and d.max_pages == 3 and d.n_pages == 5 and d.score_seq_stride == 96
    w = torch.zeros(4, 10, 64)
    with pytest.raises(ValueError):
        binding.reform_window_attend(w, w[:2, :9], w[:2, :9], torch.zeros(2, dtype=torch.int32), 0.1, 4)
