"""Thin ctypes binding of libreform_hip.so (the C ABI declared in include/reform.h).

Argument marshalling only: torch tensors supply device memory and the current HIP stream;
every step of the path runs in the library's kernels.  There is no fallback: if the shared
library is missing or a call returns a non-OK status, a ReformError is raised.
"""
import ctypes
import functools
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libreform_hip.so")
_LIB = None
_RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None)

REFORM_F32, REFORM_BF16 = 0, 1
STATUS = {0: "REFORM_OK", 1: "REFORM_ERR_INVALID_ARG", 2: "REFORM_ERR_UNSUPPORTED",
          3: "REFORM_ERR_WORKSPACE", 4: "REFORM_ERR_RUNTIME"}

EXPORTED = [
    "reform_chunk_attend_score_workspace", "reform_chunk_attend_score",
    "reform_evict_topk_compact_workspace", "reform_evict_topk_compact",
    "reform_evict_topk_compact_static", "reform_debug_set_move_spin_limit",
    "reform_gather_topk_workspace", "reform_gather_topk", "reform_gather_similarity",
    "reform_gather_pooled_workspace", "reform_gather_pooled", "reform_embed_save_selected",
    "reform_rerotate_keys", "reform_gather_rows", "reform_rotary_embed",
    "reform_prompt_attend_workspace", "reform_prompt_attend",
    "reform_tree_attend_workspace", "reform_tree_attend", "reform_tree_accept",
    "reform_window_attend_workspace", "reform_window_attend",
    "reform_paged_attend_workspace", "reform_paged_attend",
    "reform_paged_evict_workspace", "reform_paged_evict",
    "reform_probe_mfma_bf16", "reform_probe_stream",
    "reform_status_string", "reform_version",
]


class ReformError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__(f"{where}: {STATUS.get(int(status), status)}")


class AttnDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32),
                ("cache_len", ctypes.c_int32), ("chunk_len", ctypes.c_int32),
                ("capacity", ctypes.c_int32),
                ("q_head_stride", ctypes.c_int64), ("q_row_stride", ctypes.c_int64),
                ("o_head_stride", ctypes.c_int64), ("o_row_stride", ctypes.c_int64),
                ("scale", ctypes.c_float), ("obs_window", ctypes.c_int32),
                ("accumulate", ctypes.c_int32), ("phases", ctypes.c_int32)]


class EvictDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("n_valid", ctypes.c_int32), ("budget", ctypes.c_int32),
                ("capacity", ctypes.c_int32),
                ("n_sink", ctypes.c_int32), ("n_recent", ctypes.c_int32)]


class GatherDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("n_ctx", ctypes.c_int64),
                ("dim", ctypes.c_int32), ("n_query", ctypes.c_int32), ("k", ctypes.c_int32),
                ("radius", ctypes.c_int32), ("n_head_keep", ctypes.c_int32),
                ("n_tail_keep", ctypes.c_int32), ("eps", ctypes.c_float)]


class PooledDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("n_ctx", ctypes.c_int64),
                ("dim", ctypes.c_int32), ("n_query", ctypes.c_int32), ("budget", ctypes.c_int32),
                ("pool_window", ctypes.c_int32), ("n_head_keep", ctypes.c_int32),
                ("n_tail_keep", ctypes.c_int32), ("eps", ctypes.c_float)]


class EmbedDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("n_rows", ctypes.c_int64),
                ("head_dim", ctypes.c_int32), ("emb_col", ctypes.c_int32),
                ("src_row_stride", ctypes.c_int64), ("emb_row_stride", ctypes.c_int64),
                ("eps", ctypes.c_float), ("n_heads", ctypes.c_int32), ("src_head_stride", ctypes.c_int64)]


class RowsDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("reserved", ctypes.c_int32),
                ("n_table", ctypes.c_int64), ("n_idx", ctypes.c_int64), ("row_bytes", ctypes.c_int64)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("budget", ctypes.c_int32),
                ("rotary_dim", ctypes.c_int32), ("theta", ctypes.c_float)]


class RotaryDesc(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                 ("n_tokens", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                 ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                 ("rotary_dim", ctypes.c_int32), ("pairs", ctypes.c_int32),
                 ("inverse", ctypes.c_int32), ("scaling", ctypes.c_int32),
                 ("theta", ctypes.c_double), ("factor", ctypes.c_double),
                 ("turns_high", ctypes.c_double), ("turns_low", ctypes.c_double),
                 ("original_len", ctypes.c_int32), ("magnitude", ctypes.c_float),
                 ("block_len", ctypes.c_int32), ("n_blocks", ctypes.c_int32),
                 ("block_stride", ctypes.c_int64)]
                + [(f"{t}_{u}_stride", ctypes.c_int64) for t in ("q", "k", "v", "q_out", "kv_out")
                   for u in ("head", "row")])


class PromptDesc(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                 ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                 ("n_seq", ctypes.c_int32), ("n_q_rows", ctypes.c_int32), ("n_k_rows", ctypes.c_int32),
                 ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]
                + [(f"{t}_{u}_stride", ctypes.c_int64) for t in "qkvo" for u in ("head", "row")])


class TreeDesc(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("n_seq", ctypes.c_int32),
                 ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                 ("n_nodes", ctypes.c_int32), ("max_cache_len", ctypes.c_int32), ("capacity", ctypes.c_int32),
                 ("scale", ctypes.c_float)]
                + [(f"{t}_{u}_stride", ctypes.c_int64) for t in "qo" for u in ("seq", "head", "row")]
                + [("kv_seq_stride", ctypes.c_int64), ("kv_head_stride", ctypes.c_int64)])


class AcceptDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("n_seq", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("n_nodes", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("kv_seq_stride", ctypes.c_int64), ("kv_head_stride", ctypes.c_int64),
                ("kv_layer_stride", ctypes.c_int64)]


class WindowDesc(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32),
                 ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                 ("n_seq", ctypes.c_int32), ("n_q_rows", ctypes.c_int32), ("n_k_rows", ctypes.c_int32),
                 ("scale", ctypes.c_float), ("window", ctypes.c_int32), ("n_sink", ctypes.c_int32), ("reserved", ctypes.c_int32)]
                + [(f"{t}_{u}_stride", ctypes.c_int64) for t in "qkvo" for u in ("head", "row")])


class PagedDesc(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("n_seq", ctypes.c_int32),
                 ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                 ("page_len", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("max_len", ctypes.c_int32),
                 ("window", ctypes.c_int32), ("n_sink", ctypes.c_int32), ("want_score", ctypes.c_int32),
                 ("accumulate", ctypes.c_int32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]
                + [(f"{t}_stride", ctypes.c_int64) for t in ("q_seq", "q_head", "o_seq", "o_head", "kv_page", "kv_head", "kv_row", "table",
                                                             "score_seq", "score_head")])


class PagedEvictDesc(ctypes.Structure):
    _fields_ = ([("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("n_seq", ctypes.c_int32),
                 ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                 ("page_len", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("max_len", ctypes.c_int32),
                 ("budget", ctypes.c_int32), ("n_sink", ctypes.c_int32), ("n_recent", ctypes.c_int32)]
                + [(f"{t}_stride", ctypes.c_int64) for t in ("kv_page", "kv_head", "kv_row", "table", "score_seq", "score_head")])


def library_path():
    return _LIB_PATH


def load_library():
    """Load libreform_hip.so (built by paper_2506_01215_amd.build); raises if it is absent."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} not found: build it with `python -m paper_2506_01215_amd.build`"
                           " (there is no CPU fallback)")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    lib.reform_chunk_attend_score_workspace.restype = sz
    lib.reform_chunk_attend_score_workspace.argtypes = [ctypes.POINTER(AttnDesc)]
    lib.reform_chunk_attend_score.restype = ctypes.c_int
    lib.reform_chunk_attend_score.argtypes = [ctypes.POINTER(AttnDesc), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.reform_evict_topk_compact_workspace.restype = sz
    lib.reform_evict_topk_compact_workspace.argtypes = [ctypes.POINTER(EvictDesc)]
    lib.reform_evict_topk_compact.restype = ctypes.c_int
    lib.reform_evict_topk_compact.argtypes = [ctypes.POINTER(EvictDesc), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.reform_evict_topk_compact_static.restype = ctypes.c_int
    lib.reform_evict_topk_compact_static.argtypes = [ctypes.POINTER(EvictDesc), vp, vp, vp, vp, vp, vp]
    lib.reform_debug_set_move_spin_limit.restype = None
    lib.reform_debug_set_move_spin_limit.argtypes = [ctypes.c_int32]
    lib.reform_gather_topk_workspace.restype = sz
    lib.reform_gather_topk_workspace.argtypes = [ctypes.POINTER(GatherDesc)]
    lib.reform_gather_topk.restype = ctypes.c_int
    lib.reform_gather_topk.argtypes = [ctypes.POINTER(GatherDesc), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.reform_gather_similarity.restype = ctypes.c_int
    lib.reform_gather_similarity.argtypes = [ctypes.POINTER(GatherDesc), vp, vp, vp, vp]
    lib.reform_gather_pooled_workspace.restype = sz
    lib.reform_gather_pooled_workspace.argtypes = [ctypes.POINTER(PooledDesc)]
    lib.reform_gather_pooled.restype = ctypes.c_int
    lib.reform_gather_pooled.argtypes = [ctypes.POINTER(PooledDesc), vp, vp, vp, vp, vp, sz, vp]
    lib.reform_embed_save_selected.restype = ctypes.c_int
    lib.reform_embed_save_selected.argtypes = [ctypes.POINTER(EmbedDesc), vp, vp, vp]
    lib.reform_rerotate_keys.restype = ctypes.c_int
    lib.reform_rerotate_keys.argtypes = [ctypes.POINTER(RopeDesc), vp, vp, vp]
    lib.reform_gather_rows.restype = ctypes.c_int
    lib.reform_gather_rows.argtypes = [ctypes.POINTER(RowsDesc), vp, vp, vp, vp, vp, vp]
    lib.reform_rotary_embed.restype = ctypes.c_int
    lib.reform_rotary_embed.argtypes = [vp] * 10        # descriptors packed or as structures
    lib.reform_prompt_attend_workspace.restype = sz
    lib.reform_prompt_attend_workspace.argtypes = [vp]
    lib.reform_prompt_attend.restype = ctypes.c_int
    lib.reform_prompt_attend.argtypes = [vp] * 9 + [sz, vp]
    lib.reform_tree_attend_workspace.restype = sz
    lib.reform_tree_attend_workspace.argtypes = [vp]
    lib.reform_tree_attend.restype = ctypes.c_int
    lib.reform_tree_attend.argtypes = [vp] * 10 + [sz, vp]
    lib.reform_tree_accept.restype = ctypes.c_int
    lib.reform_tree_accept.argtypes = [vp] * 13
    for name in ("window_attend", "paged_attend", "paged_evict"):
        getattr(lib, f"reform_{name}_workspace").restype = sz
        getattr(lib, f"reform_{name}_workspace").argtypes = [vp]
        getattr(lib, f"reform_{name}").restype = ctypes.c_int
    lib.reform_window_attend.argtypes = [vp] * 9 + [sz, vp]
    lib.reform_paged_attend.argtypes = [vp] * 10 + [sz, vp]
    lib.reform_paged_evict.argtypes = [vp] * 10 + [sz, vp]
    lib.reform_probe_mfma_bf16.restype = ctypes.c_int
    lib.reform_probe_mfma_bf16.argtypes = [vp, vp, ctypes.c_int32, ctypes.c_int32, vp]
    lib.reform_probe_stream.restype = ctypes.c_int
    lib.reform_probe_stream.argtypes = [vp, vp, sz, vp, vp]
    lib.reform_status_string.restype = ctypes.c_char_p
    lib.reform_status_string.argtypes = [ctypes.c_int]
    lib.reform_version.restype = ctypes.c_int32
    _LIB = lib
    return lib


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return REFORM_BF16
    if t.dtype == torch.float32:
        return REFORM_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


# A call on a short problem is bound by what happens on the host before its launches: pointers go to
# ctypes as plain integers (the argument types are declared), and a workspace that the caller keeps is
# neither sliced nor measured here, since the library checks its size.
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None:      # the handle alone where this torch gives it: building the Stream object takes 2 us
        if _RAW_STREAM is not None:
            return _RAW_STREAM(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _workspace(query, desc, device, workspace, stream=None):
    """(address, bytes) of the 256-byte aligned part of the workspace; query(desc) gives the bytes a
    temporary one needs when the caller has none."""
    if workspace is None:
        nbytes = query(desc)
        if nbytes == 0:
            return None, 0
        workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        if stream is not None:
            # a temporary that is dropped on return while the kernels are only enqueued: tell the
            # caching allocator which stream still uses the block
            workspace.record_stream(stream)
    base = workspace.data_ptr()
    off = -base % 256
    return base + off, max(workspace.numel() - off, 0)


def debug_set_move_spin_limit(polls):
    """Testing aid, see include/reform.h: polls of the bounded waits between workgroups (0 forces the
    give-up branches, a negative value restores the default)."""
    load_library().reform_debug_set_move_spin_limit(int(polls))


def evict_status_word(workspace):
    """The device-side status word of reform_evict_topk_compact (first int32 of the 256-byte
    aligned workspace the caller passed): 0 unless the in-place move's bounded wait expired.
    Reads it back, so it synchronises with the device."""
    off = (-workspace.data_ptr()) % 256
    return int(workspace[off:off + 4].view(torch.int32).item())


def _check(rc, where):
    if rc != 0:
        raise ReformError(rc, where)


# ------------------------------------------------------------------------------------------
def attn_desc(q, k, out, cache_len, scale, obs_window=0, accumulate=False, phases=0):
    Hq, Ct, d = q.shape
    Hkv, cap, d2 = k.shape
    assert d2 == d and q.stride(2) == 1 and out.stride(2) == 1
    return AttnDesc(ctypes.sizeof(AttnDesc), _dtype_code(q), Hq, Hkv, d, int(cache_len), Ct, cap,
                    q.stride(0), q.stride(1), out.stride(0), out.stride(1),
                    float(scale), int(obs_window), int(bool(accumulate)), int(phases))


def reform_chunk_attend_score(q, k, v, cache_len, scale, obs_window=0, accumulate=False,
                              out=None, lse=None, score=None, want_score=True,
                              workspace=None, stream=None, phases=0):
    """q [Hq,Ct,d]; k,v [Hkv,cap,d] (rows [0,M) cache, [M,M+Ct) chunk).  Returns (out, lse, score)."""
    lib = load_library()
    assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if lse is None:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    if score is None and want_score:
        if accumulate:
            raise ValueError("accumulate needs the previous score tensor")
        score = torch.zeros(k.shape[:2], dtype=torch.float32, device=q.device)
    desc = attn_desc(q, k, out, cache_len, scale, obs_window, accumulate, phases)
    ws, ws_bytes = _workspace(lib.reform_chunk_attend_score_workspace, ctypes.byref(desc), q.device, workspace, stream)
    rc = lib.reform_chunk_attend_score(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                       _ptr(lse), _ptr(score), ws,
                                       ws_bytes, _stream(stream))
    _check(rc, "reform_chunk_attend_score")
    return out, lse, score


def evict_desc(k, n_valid, budget, n_sink=0, n_recent=0):
    Hkv, cap, d = k.shape
    return EvictDesc(ctypes.sizeof(EvictDesc), _dtype_code(k), Hkv, d, int(n_valid), int(budget), cap,
                     int(n_sink), int(n_recent))


def reform_evict_topk_compact(k, v, score, n_valid, budget, n_sink=0, n_recent=0, pos=None,
                              kept_idx=None, workspace=None, stream=None):
    """In-place retention + compaction.  Returns new_len = min(n_valid, budget)."""
    lib = load_library()
    assert k.is_contiguous() and v.is_contiguous() and score.is_contiguous()
    assert score.dtype == torch.float32 and score.shape == k.shape[:2]
    if pos is not None:
        assert pos.dtype == torch.int32 and pos.is_contiguous() and pos.shape == k.shape[:2]
    if kept_idx is not None:
        assert kept_idx.dtype == torch.int32 and kept_idx.is_contiguous()
        assert kept_idx.shape == (k.shape[0], budget)
    desc = evict_desc(k, n_valid, budget, n_sink, n_recent)
    ws, ws_bytes = _workspace(lib.reform_evict_topk_compact_workspace, ctypes.byref(desc), k.device, workspace, stream)
    rc = lib.reform_evict_topk_compact(ctypes.byref(desc), _ptr(k), _ptr(v), _ptr(score), _ptr(pos),
                                       _ptr(kept_idx), ws, ws_bytes,
                                       _stream(stream))
    _check(rc, "reform_evict_topk_compact")
    return min(int(n_valid), int(budget))


STATIC_SCRATCH_BYTES = 8 << 20


def reform_evict_topk_compact_static(k, v, score, n_valid, budget, n_sink=0, n_recent=0, pos=None,
                                     kept_idx=None, stream=None):
    """reform_evict_topk_compact without a workspace (the library's static device scratch); the
    binding allocates nothing either.  k's device must be the current one."""
    lib = load_library()
    assert k.is_contiguous() and v.is_contiguous() and score.is_contiguous()
    assert score.dtype == torch.float32 and score.shape == k.shape[:2]
    desc = evict_desc(k, n_valid, budget, n_sink, n_recent)
    rc = lib.reform_evict_topk_compact_static(ctypes.byref(desc), _ptr(k), _ptr(v), _ptr(score),
                                              _ptr(pos), _ptr(kept_idx), _stream(stream))
    _check(rc, "reform_evict_topk_compact_static")
    return min(int(n_valid), int(budget))


def gather_desc(emb, qry, k, radius=0, n_head_keep=0, n_tail_keep=0, eps=1e-8):
    N, D = emb.shape
    nq, D2 = qry.shape
    assert D == D2 and emb.dtype == qry.dtype
    return GatherDesc(ctypes.sizeof(GatherDesc), _dtype_code(emb), N, D, nq, int(k), int(radius),
                      int(n_head_keep), int(n_tail_keep), float(eps))


def reform_gather_topk(emb, qry, k, radius=0, n_head_keep=0, n_tail_keep=0, eps=1e-8,
                       want_union=True, topk_idx=None, topk_score=None, union_idx=None,
                       union_count=None, workspace=None, stream=None):
    """Returns (topk_idx [nq,k] i32, topk_score [nq,k] f32, union_idx [N] i32 or None, union_count)."""
    lib = load_library()
    assert emb.is_contiguous() and qry.is_contiguous()
    N, nq = emb.shape[0], qry.shape[0]
    dev = emb.device
    if topk_idx is None:
        topk_idx = torch.empty((nq, k), dtype=torch.int32, device=dev)
    if topk_score is None:
        topk_score = torch.empty((nq, k), dtype=torch.float32, device=dev)
    if want_union:
        if union_idx is None:
            union_idx = torch.empty((N,), dtype=torch.int32, device=dev)
        if union_count is None:
            union_count = torch.zeros((1,), dtype=torch.int32, device=dev)
    desc = gather_desc(emb, qry, k, radius, n_head_keep, n_tail_keep, eps)
    ws, ws_bytes = _workspace(lib.reform_gather_topk_workspace, ctypes.byref(desc), dev, workspace, stream)
    rc = lib.reform_gather_topk(ctypes.byref(desc), _ptr(emb), _ptr(qry), _ptr(topk_idx),
                                _ptr(topk_score), _ptr(union_idx), _ptr(union_count), ws,
                                ws_bytes, _stream(stream))
    _check(rc, "reform_gather_topk")
    return topk_idx, topk_score, union_idx, union_count


def reform_gather_similarity(emb, qry, eps=1e-8, sim=None, stream=None):
    lib = load_library()
    assert emb.is_contiguous() and qry.is_contiguous()
    if sim is None:
        sim = torch.empty((qry.shape[0], emb.shape[0]), dtype=torch.float32, device=emb.device)
    desc = gather_desc(emb, qry, 1, eps=eps)
    rc = lib.reform_gather_similarity(ctypes.byref(desc), _ptr(emb), _ptr(qry), _ptr(sim), _stream(stream))
    _check(rc, "reform_gather_similarity")
    return sim


def reform_embed_save_selected(src, emb, row0, col, eps=1e-12, stream=None):
    """src [n_rows, d] (a view of one head's Q, K or V states; any row stride) or
    [n_heads, n_rows, d] (several heads of one tensor; any head and row strides); writes the
    normalised rows into emb[row0 : row0 + n_rows, col : col + n_heads * d]."""
    lib = load_library()
    if src.dim() == 2:
        src = src.unsqueeze(0)
    nh, n, d = src.shape
    assert nh >= 1 and src.stride(2) == 1 and emb.is_contiguous() and emb.dtype == src.dtype
    assert 0 <= row0 and row0 + n <= emb.shape[0]
    desc = EmbedDesc(ctypes.sizeof(EmbedDesc), _dtype_code(src), n, d, int(col), src.stride(1),
                     emb.shape[1], float(eps), nh, src.stride(0) if nh > 1 else 0)
    dst = emb[row0:] if n else emb
    rc = lib.reform_embed_save_selected(ctypes.byref(desc), _ptr(src), _ptr(dst), _stream(stream))
    _check(rc, "reform_embed_save_selected")
    return emb


def reform_rerotate_keys(k, kept_idx, n_rows, theta=10000.0, rotary_dim=None, stream=None):
    """Rotates the compacted key rows [0, n_rows) of every head in place by (r - kept_idx[r]) positions."""
    lib = load_library()
    assert k.is_contiguous() and kept_idx.is_contiguous() and kept_idx.dtype == torch.int32
    Hkv, cap, d = k.shape
    assert kept_idx.shape[0] == Hkv
    desc = RopeDesc(ctypes.sizeof(RopeDesc), _dtype_code(k), Hkv, d, cap, int(n_rows), kept_idx.shape[1],
                    d if rotary_dim is None else int(rotary_dim), float(theta))
    rc = lib.reform_rerotate_keys(ctypes.byref(desc), _ptr(k), _ptr(kept_idx), _stream(stream))
    _check(rc, "reform_rerotate_keys")
    return k


def reform_gather_rows(table, idx, count=None, out=None, err=None, stream=None):
    """out[i] = table[idx[i]]; `count` (device int32 scalar) limits the rows taken."""
    lib = load_library()
    assert table.is_contiguous() and idx.is_contiguous() and idx.dtype == torch.int32 and idx.dim() == 1
    row_bytes = table[0].numel() * table.element_size()
    if out is None:
        out = torch.empty((idx.shape[0],) + tuple(table.shape[1:]), dtype=table.dtype, device=table.device)
    assert out.is_contiguous() and out.shape[0] >= idx.shape[0]
    desc = RowsDesc(ctypes.sizeof(RowsDesc), 0, table.shape[0], idx.shape[0], row_bytes)
    rc = lib.reform_gather_rows(ctypes.byref(desc), _ptr(table), _ptr(idx), _ptr(count), _ptr(out),
                                _ptr(err), _stream(stream))
    _check(rc, "reform_gather_rows")
    return out


# The serving calls are made once per layer and generated token, so their descriptors are packed by `struct` (a ctypes
# structure takes 2 us to fill), in the layout that the classes above declare, and tensors are checked with as few calls as will do.
_CODES = {ctypes.c_uint32: "I", ctypes.c_int32: "i", ctypes.c_int64: "q", ctypes.c_float: "f", ctypes.c_double: "d"}


def _packer(cls):
    packer = struct.Struct("@" + "".join(_CODES[t] for _, t in cls._fields_))
    assert packer.size == ctypes.sizeof(cls)
    return functools.partial(packer.pack, ctypes.sizeof(cls))


_pack_rotary, _pack_prompt, _pack_tree, _pack_accept = map(_packer, (RotaryDesc, PromptDesc, TreeDesc, AcceptDesc))
_pack_window, _pack_paged, _pack_paged_evict = map(_packer, (WindowDesc, PagedDesc, PagedEvictDesc))


class _Codes(dict):
    def __missing__(self, dtype):
        raise TypeError(f"unsupported dtype {dtype}")


_DTYPES = _Codes({torch.float32: REFORM_F32, torch.bfloat16: REFORM_BF16})
_I32 = torch.int32


# The current device's index where torch has been initialised, as it has with a tensor on a GPU.
_CURRENT = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _gpu(t):
    """The current device's index if t is there: calls launch on it, and a host tensor's address would be read by the GPU."""
    dev = t.get_device()
    if dev < 0 or dev != _CURRENT():
        raise ValueError("all tensors have to be on the current GPU")
    return dev


def _at(t, dev):
    """Address of a tensor that has to be on the device `dev`, or None."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise ValueError("all tensors have to be on the current GPU")
    return t.data_ptr()


def _i32(t, n, dev, what):
    """Address of n contiguous int32 on the device, or None."""
    if t is None:
        return None
    if t.dtype is not _I32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what}: {n} contiguous int32 expected")
    if t.get_device() != dev:
        raise ValueError("all tensors have to be on the current GPU")
    return t.data_ptr()


def _stream_of(stream, dev):
    """As _stream, for the current device's index."""
    if stream is None and _RAW_STREAM is not None:
        return _RAW_STREAM(dev)
    return _stream(stream)


def _new(make, shape, dtype, device, stream):
    """A tensor that the call fills: made on the stream that the call runs on, so that nothing of another stream is still
    using its memory and its own clearing comes first."""
    if stream is None:
        return make(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype, device=device)


def _scratch(query, desc, dev, workspace, first, stream):
    """As _workspace, with the caller's one checked and a missing one made on the call's stream."""
    if workspace is None:
        nbytes = query(desc)
        if nbytes == 0:
            return None, 0
        workspace = _new(torch.empty, (nbytes + 256,), torch.uint8, first.device, stream)
        if stream is not None:
            workspace.record_stream(stream)
    elif workspace.get_device() != dev:
        raise ValueError("all tensors have to be on the current GPU")
    base = workspace.data_ptr()
    off = -base % 256
    return base + off, max(workspace.numel() - off, 0)


ROPE_SCALING = {None: 0, "none": 0, "linear": 1, "base": 2, "parts": 3, "bands": 4}


def reform_rotary_embed(q, k, v, pos, theta=10000.0, rotary_dim=None, interleaved=False, inverse=False,
                        scaling=None, factor=1.0, original_len=0, turns_high=32.0, turns_low=1.0,
                        magnitude=1.0, slot=None, q_out=None, k_out=None, v_out=None, stream=None):
    """q [Hq, n, d], k, v [Hkv, n, d] (any strides with contiguous elements; q, or k and v, or v may be None),
    pos [n] i32.  Queries and keys are rotated to their positions, values copied.  slot None: into q_out, k_out, v_out
    like the inputs (made where missing; the inputs themselves rotate in place).  slot [n] i32: keys and values go to
    caches k_out, v_out [Hkv, cap, d] or [blocks, Hkv, cap, d], row slot % cap of block slot // cap.
    Returns (q_out, k_out, v_out)."""
    lib = load_library()
    mode = ROPE_SCALING.get(scaling)
    if mode is None:
        raise ValueError(f"scaling {scaling!r}: one of {list(ROPE_SCALING)}")
    first = k if q is None else q
    if first is None or (k is None and v is not None):
        raise ValueError("queries, or keys with or without values")
    dtype = first.dtype
    shape = first.shape
    hkv = block_len = n_blocks = block_stride = 0
    qs = ks = vs = qos = kvos = (0, 0, 1)
    if q is not None:
        if q_out is None:
            q_out = _new(torch.empty, shape, dtype, q.device, stream)
        hq, n, d = shape
        qs, qos = q.stride(), q_out.stride()
        if q_out.shape != shape or q_out.dtype is not dtype or qs[2] != 1 or qos[2] != 1:
            raise ValueError("q_out: like q, elements of a row contiguous")
    else:
        hq, (_, n, d) = 0, shape
        if q_out is not None:
            raise ValueError("q_out without q")
    if k is not None:
        kshape = k.shape
        hkv = kshape[0]
        if kshape[1] != n or kshape[2] != d or k.dtype is not dtype:
            raise ValueError("k: as many rows and elements as q, same type")
        if slot is None:
            if k_out is None:
                k_out = _new(torch.empty, kshape, dtype, k.device, stream)
            if v_out is None and v is not None:
                v_out = _new(torch.empty, kshape, dtype, v.device, stream)
            oshape, kvos = k_out.shape, k_out.stride()
            if oshape != kshape:
                raise ValueError("k_out: like k")
        else:
            if k_out is None or k_out.dim() not in (3, 4):
                raise ValueError("slots need caches [heads, rows, d] or [blocks, heads, rows, d]")
            oshape, kvos = k_out.shape, k_out.stride()
            n_blocks = 1
            if len(oshape) == 4:
                n_blocks, block_stride = oshape[0], kvos[0]
            block_len = oshape[-2]
            if oshape[-3] != hkv or oshape[-1] != d:
                raise ValueError("caches with other heads or elements than k")
        ks = k.stride()
        if k_out.dtype is not dtype or ks[2] != 1 or kvos[-1] != 1:
            raise ValueError("k_out: k's type, elements of a row contiguous")
        if v is not None:
            vs = v.stride()
            if v_out is None or v.shape != kshape or v.dtype is not dtype or vs[2] != 1:
                raise ValueError("v: like k, and a v_out")
            if v_out.shape != oshape or v_out.stride() != kvos or v_out.dtype is not dtype:
                raise ValueError("v_out: like k_out")
        elif v_out is not None:
            raise ValueError("v_out without v")
    elif k_out is not None or v_out is not None:
        raise ValueError("k_out or v_out without k")
    desc = _pack_rotary(_DTYPES[dtype], n, hq, hkv, d, d if rotary_dim is None else rotary_dim, 1 if interleaved else 0,
                        1 if inverse else 0, mode, theta, factor, turns_high, turns_low, original_len, magnitude, block_len,
                        n_blocks, block_stride, qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], qos[0], qos[1], kvos[-3], kvos[-2])
    dev = _gpu(first)
    rc = lib.reform_rotary_embed(desc, _at(q, dev), _at(k, dev), _at(v, dev), _i32(pos, n, dev, "pos"), _i32(slot, n, dev, "slot"),
                                 _at(q_out, dev), _at(k_out, dev), _at(v_out, dev), _stream_of(stream, dev))
    _check(rc, "reform_rotary_embed")
    return q_out, k_out, v_out


def _prompt_fields(q, k, v, out, n_seq, scale):
    shape, kshape, dtype = q.shape, k.shape, q.dtype
    Hq, nq, d = shape
    Hkv, nk, dk = kshape
    qs, ks, vs, os = q.stride(), k.stride(), v.stride(), out.stride()
    if dk != d or v.shape != kshape or out.shape != shape:
        raise ValueError("shapes of q, k, v and out")
    if k.dtype is not dtype or v.dtype is not dtype or out.dtype is not dtype:
        raise ValueError("types of q, k, v and out")
    if qs[2] != 1 or ks[2] != 1 or vs[2] != 1 or os[2] != 1:
        raise ValueError("elements of a row have to be contiguous")
    return (_DTYPES[dtype], Hq, Hkv, d, n_seq, nq, nk, scale, 0, qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], os[0], os[1])


def prompt_desc(q, k, v, out, cu_q, scale):
    return PromptDesc(ctypes.sizeof(PromptDesc), *_prompt_fields(q, k, v, out, cu_q.shape[0] - 1, scale))


def reform_prompt_attend(q, k, v, cu_q, scale, cu_k=None, out=None, lse=None, workspace=None, stream=None):
    """q [Hq, nq, d], k, v [Hkv, nk, d] packed sequences (any strides with contiguous elements), cu_q [n_seq + 1] i32
    their boundaries, cu_k those of the keys (None: cu_q).  Causal attention inside every sequence, its last row seeing all of its
    keys.  Returns (out, lse [Hq, nq])."""
    lib = load_library()
    if out is None:
        out = _new(torch.zeros, q.shape, q.dtype, q.device, stream)
    if lse is None:
        lse = _new(torch.zeros, q.shape[:2], torch.float32, q.device, stream)
    n = cu_q.numel()
    fields = _prompt_fields(q, k, v, out, n - 1, scale)
    if n < 1 or (cu_k is None and fields[6] != fields[5]):
        raise ValueError("cu_k is needed where there are more or fewer key rows")
    if lse.dtype is not torch.float32 or lse.numel() != fields[1] * fields[5] or not lse.is_contiguous():
        raise ValueError("lse: [heads, rows] fp32")
    dev = _gpu(q)
    desc = _pack_prompt(*fields)
    ws, ws_bytes = _scratch(lib.reform_prompt_attend_workspace, desc, dev, workspace, q, stream)
    rc = lib.reform_prompt_attend(desc, q.data_ptr(), _at(k, dev), _at(v, dev), _i32(cu_q, n, dev, "cu_q"),
                                  _i32(cu_k, n, dev, "cu_k"), _at(out, dev), _at(lse, dev), ws, ws_bytes, _stream_of(stream, dev))
    _check(rc, "reform_prompt_attend")
    return out, lse


def _tree_fields(q, k, v, out, scale, max_cache_len):
    shape, kshape, dtype = q.shape, k.shape, q.dtype
    S, Hq, T, d = shape
    Sk, Hkv, cap, dk = kshape
    qs, ks, os = q.stride(), k.stride(), out.stride()
    if Sk != S or dk != d or v.shape != kshape or v.stride() != ks or out.shape != shape:
        raise ValueError("shapes of q, k, v and out")
    if k.dtype is not dtype or v.dtype is not dtype or out.dtype is not dtype:
        raise ValueError("types of q, k, v and out")
    if qs[3] != 1 or os[3] != 1 or ks[3] != 1 or (ks[2] != d and cap != 1):
        raise ValueError("elements of a row, and rows of the caches, have to be contiguous")
    return (_DTYPES[dtype], S, Hq, Hkv, d, T, cap - T if max_cache_len is None else max_cache_len, cap, scale,
            qs[0], qs[1], qs[2], os[0], os[1], os[2], ks[0], ks[1])


def tree_desc(q, k, v, out, scale, max_cache_len=None):
    return TreeDesc(ctypes.sizeof(TreeDesc), *_tree_fields(q, k, v, out, scale, max_cache_len))


def reform_tree_attend(q, k, v, cache_len, scale, parent=None, node_count=None, max_cache_len=None, out=None, lse=None,
                       workspace=None, stream=None):
    """q [S, Hq, T, d]: T drafted tokens of each of S sequences; k, v [S, Hkv, cap, d]: their caches, rows
    [0, cache_len[b]) cached, the drafted tokens' rows behind them.  parent [S, T] i32 (None: a chain), node_count [S] i32
    (None: T each).  max_cache_len bounds cache_len (None: cap - T).  Returns (out, lse [S, Hq, T])."""
    lib = load_library()
    if out is None:
        out = _new(torch.zeros, q.shape, q.dtype, q.device, stream)
    if lse is None:
        lse = _new(torch.zeros, q.shape[:3], torch.float32, q.device, stream)
    fields = _tree_fields(q, k, v, out, scale, max_cache_len)
    S, T = fields[1], fields[5]
    if lse.dtype is not torch.float32 or lse.numel() != S * fields[2] * T or not lse.is_contiguous():
        raise ValueError("lse: [sequences, heads, nodes] fp32")
    dev = _gpu(q)
    desc = _pack_tree(*fields)
    ws, ws_bytes = _scratch(lib.reform_tree_attend_workspace, desc, dev, workspace, q, stream)
    rc = lib.reform_tree_attend(desc, q.data_ptr(), _at(k, dev), _at(v, dev), _i32(cache_len, S, dev, "cache_len"),
                                _i32(parent, S * T, dev, "parent"), _i32(node_count, S, dev, "node_count"), _at(out, dev),
                                _at(lse, dev), ws, ws_bytes, _stream_of(stream, dev))
    _check(rc, "reform_tree_attend")
    return out, lse


def reform_tree_accept(parent, drafted, target, cache_len, k=None, v=None, node_count=None, path=None, accepted=None,
                       next_token=None, new_len=None, stream=None):
    """parent (None: a chain), drafted, target [S, T] i32; k, v [S, Hkv, cap, d] or [layers, S, Hkv, cap, d] caches whose accepted
    rows move together in place, or None.  Returns (path [S, T] i32, accepted [S], next_token [S], new_len [S])."""
    lib = load_library()
    S, T = drafted.shape
    if path is None or accepted is None or next_token is None or new_len is None:
        device = drafted.device
        path = _new(torch.empty, (S, T), _I32, device, stream) if path is None else path
        accepted, next_token, new_len = (_new(torch.empty, (S,), _I32, device, stream) if t is None else t
                                         for t in (accepted, next_token, new_len))
    dtype, Hkv, cap, d, layers, strides = REFORM_F32, 1, (1 << 31) - 1, 4, 1, (0, 0, 0)
    if k is not None:
        shape, ks = k.shape, k.stride()
        if len(shape) not in (4, 5) or v is None or v.shape != shape or v.stride() != ks or v.dtype is not k.dtype:
            raise ValueError("k and v: alike, 4 or 5 dimensions")
        Hkv, cap, d = shape[-3:]
        if shape[-4] != S or ks[-1] != 1 or (ks[-2] != d and cap != 1):
            raise ValueError("caches of other sequences, or rows not contiguous")
        dtype = _DTYPES[k.dtype]
        layers, strides = (shape[0], (ks[1], ks[2], ks[0])) if len(shape) == 5 else (1, (ks[0], ks[1], 0))
    elif v is not None:
        raise ValueError("v without k")
    dev = _gpu(drafted)
    n = S * T
    rc = lib.reform_tree_accept(_pack_accept(dtype, S, Hkv, d, T, cap, layers, *strides), _i32(parent, n, dev, "parent"),
                                _i32(drafted, n, dev, "drafted"), _i32(target, n, dev, "target"), _i32(cache_len, S, dev, "cache_len"),
                                _i32(node_count, S, dev, "node_count"), _at(k, dev), _at(v, dev), _i32(path, n, dev, "path"),
                                _i32(accepted, S, dev, "accepted"), _i32(next_token, S, dev, "next_token"),
                                _i32(new_len, S, dev, "new_len"), _stream_of(stream, dev))
    _check(rc, "reform_tree_accept")
    return path, accepted, next_token, new_len


def _window_fields(q, k, v, out, n_seq, scale, window, n_sink):
    f = _prompt_fields(q, k, v, out, n_seq, scale)       # its last scalar, `reserved`, gives way to window, n_sink and this one's
    return f[:8] + (window, n_sink, 0) + f[9:]


def window_desc(q, k, v, out, cu_q, scale, window, n_sink=0):
    return WindowDesc(ctypes.sizeof(WindowDesc), *_window_fields(q, k, v, out, cu_q.shape[0] - 1, scale, window, n_sink))


def reform_window_attend(q, k, v, cu_q, scale, window, n_sink=0, cu_k=None, out=None, lse=None, workspace=None, stream=None):
    """As reform_prompt_attend, each row seeing the last `window` keys up to its own and the first n_sink keys of its sequence.
    Returns (out, lse [Hq, nq])."""
    lib = load_library()
    if out is None:
        out = _new(torch.zeros, q.shape, q.dtype, q.device, stream)
    if lse is None:
        lse = _new(torch.zeros, q.shape[:2], torch.float32, q.device, stream)
    n = cu_q.numel()
    fields = _window_fields(q, k, v, out, n - 1, scale, window, n_sink)
    if n < 1 or (cu_k is None and fields[6] != fields[5]):
        raise ValueError("cu_k is needed where there are more or fewer key rows")
    if lse.dtype is not torch.float32 or lse.numel() != fields[1] * fields[5] or not lse.is_contiguous():
        raise ValueError("lse: [heads, rows] fp32")
    dev = _gpu(q)
    desc = _pack_window(*fields)
    ws, ws_bytes = _scratch(lib.reform_window_attend_workspace, desc, dev, workspace, q, stream)
    rc = lib.reform_window_attend(desc, q.data_ptr(), _at(k, dev), _at(v, dev), _i32(cu_q, n, dev, "cu_q"),
                                  _i32(cu_k, n, dev, "cu_k"), _at(out, dev), _at(lse, dev), ws, ws_bytes, _stream_of(stream, dev))
    _check(rc, "reform_window_attend")
    return out, lse


def _pool_fields(k, v, page_table, score, max_len, n_seq, Hkv):
    """What the calls on caches in pages have in common: (head_dim, page_len, n_pages, max_pages, max_len), and the strides of k and
    v, of the table and of the scores."""
    pages, heads, page_len, d = shape = k.shape
    ks = k.stride()
    if v.shape != shape or v.stride() != ks or v.dtype is not k.dtype or heads != Hkv or ks[3] != 1:
        raise ValueError("k and v: alike, [pages, heads, rows, elements], elements contiguous")
    seqs, columns = page_table.shape
    ts = page_table.stride()
    if page_table.dtype is not _I32 or seqs != n_seq or (ts[1] != 1 and columns != 1):
        raise ValueError("page_table: [sequences, pages] int32, a sequence's pages contiguous")
    if score is None:
        if max_len is None:
            max_len = min(columns * page_len, _MOST_KEYS)
        return (d, page_len, pages, columns, max_len), (ks[0], ks[1], ks[2], ts[0], 0, 0)
    seqs, heads, room = score.shape
    ss = score.stride()
    if seqs != n_seq or heads != Hkv or score.dtype is not torch.float32 or (ss[2] != 1 and room != 1):
        raise ValueError("score: [sequences, KV heads, keys] fp32, a head's keys contiguous")
    if max_len is None:
        max_len = min(columns * page_len, room, _MOST_KEYS)
    elif max_len > room:
        raise ValueError("score: max_len keys at least")
    return (d, page_len, pages, columns, max_len), (ks[0], ks[1], ks[2], ts[0], ss[0], ss[1])


_MOST_KEYS = (1 << 31) - 65536


def _paged_fields(q, k, v, out, page_table, scale, window, n_sink, score, accumulate, max_len):
    S, Hq, d = shape = q.shape
    qs, os, dtype, Hkv = q.stride(), out.stride(), q.dtype, k.shape[1]
    if out.shape != shape or k.dtype is not dtype or out.dtype is not dtype or qs[2] != 1 or os[2] != 1:
        raise ValueError("q and out: [sequences, heads, elements], of k's type, elements contiguous")
    pool, strides = _pool_fields(k, v, page_table, score, max_len, S, Hkv)
    if pool[0] != d:
        raise ValueError("k: as many elements as q")
    return (_DTYPES[dtype], S, Hq, Hkv, *pool, window, n_sink, score is not None, bool(accumulate), scale, 0,
            qs[0], qs[1], os[0], os[1], *strides)


def paged_desc(q, k, v, out, page_table, scale, window=0, n_sink=0, score=None, accumulate=False, max_len=None):
    return PagedDesc(ctypes.sizeof(PagedDesc), *_paged_fields(q, k, v, out, page_table, scale, window, n_sink, score, accumulate, max_len))


def reform_paged_attend(q, k, v, page_table, cache_len, scale, window=0, n_sink=0, score=None, accumulate=False, max_len=None,
                        out=None, lse=None, workspace=None, stream=None):
    """q [S, Hq, d]: one new token of each of S sequences; k, v [pages, Hkv, page_len, d]: a pool of pages (any strides with
    contiguous elements), page_table [S, max_pages] i32, cache_len [S] i32 (the new token's row counts).  window > 0: the last
    `window` keys and the first n_sink are seen.  score [S, Hkv, keys] f32: the attention that every key receives is written, or
    added.  max_len bounds cache_len (None: what table and score have room for).  Returns (out, lse [S, Hq])."""
    lib = load_library()
    if out is None:
        out = _new(torch.empty, q.shape, q.dtype, q.device, stream)
    if lse is None:
        lse = _new(torch.empty, q.shape[:2], torch.float32, q.device, stream)
    fields = _paged_fields(q, k, v, out, page_table, scale, window, n_sink, score, accumulate, max_len)
    S = fields[1]
    if lse.dtype is not torch.float32 or lse.numel() != S * fields[2] or not lse.is_contiguous():
        raise ValueError("lse: [sequences, heads] fp32")
    dev = _gpu(q)
    if k.get_device() != dev or v.get_device() != dev or page_table.get_device() != dev or out.get_device() != dev or lse.get_device() != dev:
        raise ValueError("all tensors have to be on the current GPU")
    desc = _pack_paged(*fields)
    ws, ws_bytes = _scratch(lib.reform_paged_attend_workspace, desc, dev, workspace, q, stream)
    rc = lib.reform_paged_attend(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), page_table.data_ptr(), _i32(cache_len, S, dev, "cache_len"),
                                 _at(score, dev), out.data_ptr(), lse.data_ptr(), ws, ws_bytes, _stream_of(stream, dev))
    _check(rc, "reform_paged_attend")
    return out, lse


def _paged_evict_fields(k, v, score, page_table, budget, n_sink, n_recent, max_len):
    S, Hkv, _ = score.shape
    pool, strides = _pool_fields(k, v, page_table, score, max_len, S, Hkv)
    return (_DTYPES[k.dtype], S, Hkv, *pool, budget, n_sink, n_recent, *strides)


def paged_evict_desc(k, v, score, page_table, budget, n_sink=0, n_recent=0, max_len=None):
    return PagedEvictDesc(ctypes.sizeof(PagedEvictDesc), *_paged_evict_fields(k, v, score, page_table, budget, n_sink, n_recent, max_len))


def reform_paged_evict(k, v, score, page_table, cache_len, budget, n_sink=0, n_recent=0, pos=None, kept_idx=None, new_len=None,
                       max_len=None, workspace=None, stream=None):
    """k, v [pages, Hkv, page_len, d], score (and pos, int32, with its strides) [S, Hkv, keys], page_table [S, max_pages] i32,
    cache_len [S] i32: sequences of more than `budget` keys keep those with the largest scores, the first n_sink and the
    last n_recent among them, moved together in place.  kept_idx [S, Hkv, budget] i32.  Returns new_len [S] i32."""
    lib = load_library()
    S, Hkv = score.shape[:2]
    if new_len is None:
        new_len = _new(torch.empty, (S,), _I32, score.device, stream)
    fields = _paged_evict_fields(k, v, score, page_table, budget, n_sink, n_recent, max_len)
    if pos is not None and (pos.dtype is not _I32 or pos.shape != score.shape or pos.stride() != score.stride()):
        raise ValueError("pos: int32, shape and strides of score")
    dev = _gpu(k)
    if v.get_device() != dev or score.get_device() != dev or page_table.get_device() != dev:
        raise ValueError("all tensors have to be on the current GPU")
    desc = _pack_paged_evict(*fields)
    ws, ws_bytes = _scratch(lib.reform_paged_evict_workspace, desc, dev, workspace, k, stream)
    rc = lib.reform_paged_evict(desc, k.data_ptr(), v.data_ptr(), score.data_ptr(), _at(pos, dev), page_table.data_ptr(),
                                _i32(cache_len, S, dev, "cache_len"), _i32(kept_idx, S * Hkv * budget, dev, "kept_idx"),
                                _i32(new_len, S, dev, "new_len"), ws, ws_bytes, _stream_of(stream, dev))
    _check(rc, "reform_paged_evict")
    return new_len


def window_workspace_bytes(desc):
    return load_library().reform_window_attend_workspace(ctypes.byref(desc))


def paged_workspace_bytes(desc):
    return load_library().reform_paged_attend_workspace(ctypes.byref(desc))


def paged_evict_workspace_bytes(desc):
    return load_library().reform_paged_evict_workspace(ctypes.byref(desc))


def prompt_workspace_bytes(desc):
    return load_library().reform_prompt_attend_workspace(ctypes.byref(desc))


def tree_workspace_bytes(desc):
    return load_library().reform_tree_attend_workspace(ctypes.byref(desc))


def pooled_desc(emb, qry, budget, pool_window=129, n_head_keep=0, n_tail_keep=0, eps=1e-8):
    N, D = emb.shape
    nq, D2 = qry.shape
    assert D == D2 and emb.dtype == qry.dtype
    return PooledDesc(ctypes.sizeof(PooledDesc), _dtype_code(emb), N, D, nq, int(budget),
                      int(pool_window), int(n_head_keep), int(n_tail_keep), float(eps))


def reform_gather_pooled(emb, qry, budget, pool_window=129, n_head_keep=0, n_tail_keep=0, eps=1e-8,
                         sel_idx=None, pooled=None, workspace=None, stream=None):
    """Returns (sel_idx [budget] i32 ascending, pooled [N] f32)."""
    lib = load_library()
    assert emb.is_contiguous() and qry.is_contiguous()
    dev = emb.device
    if sel_idx is None:
        sel_idx = torch.empty((budget,), dtype=torch.int32, device=dev)
    if pooled is None:
        pooled = torch.empty((emb.shape[0],), dtype=torch.float32, device=dev)
    desc = pooled_desc(emb, qry, budget, pool_window, n_head_keep, n_tail_keep, eps)
    ws, ws_bytes = _workspace(lib.reform_gather_pooled_workspace, ctypes.byref(desc), dev, workspace, stream)
    rc = lib.reform_gather_pooled(ctypes.byref(desc), _ptr(emb), _ptr(qry), _ptr(sel_idx), _ptr(pooled),
                                  ws, ws_bytes, _stream(stream))
    _check(rc, "reform_gather_pooled")
    return sel_idx, pooled


def pooled_workspace_bytes(desc):
    return load_library().reform_gather_pooled_workspace(ctypes.byref(desc))


def attend_workspace_bytes(desc):
    return load_library().reform_chunk_attend_score_workspace(ctypes.byref(desc))


def evict_workspace_bytes(desc):
    return load_library().reform_evict_topk_compact_workspace(ctypes.byref(desc))


def gather_workspace_bytes(desc):
    return load_library().reform_gather_topk_workspace(ctypes.byref(desc))


def probe_mfma_bf16(operands, sink, iters, workgroups, stream=None):
    """Measurement aid: a pure bf16 MFMA loop; returns the flop it executes."""
    assert operands.numel() * operands.element_size() >= 65536 and sink.numel() * sink.element_size() >= 16
    rc = load_library().reform_probe_mfma_bf16(_ptr(operands), _ptr(sink), int(iters), int(workgroups),
                                               _stream(stream))
    _check(rc, "reform_probe_mfma_bf16")
    return float(workgroups) * 8 * iters * 16 * 16384


def probe_stream(src, dst, sink, stream=None):
    """Measurement aid: read src (and copy it to dst unless dst is None); returns the bytes moved."""
    nbytes = src.numel() * src.element_size()
    assert src.is_contiguous() and (dst is None or (dst.is_contiguous() and dst.numel() * dst.element_size() >= nbytes))
    rc = load_library().reform_probe_stream(_ptr(src), _ptr(dst), nbytes, _ptr(sink), _stream(stream))
    _check(rc, "reform_probe_stream")
    return float(nbytes) * (1 if dst is None else 2)
