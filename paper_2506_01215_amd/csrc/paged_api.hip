// C ABI of the calls on sliding windows and on caches in pages (see include/reform.h).  Host-side validation and kernel
// launches; nothing here allocates device memory or synchronises.
#include "../../include/reform.h"
#include "common.h"
#include "serving_checks.h"

#include <cmath>
#include <cstring>

namespace reform {
hipError_t window_attend_launch(const WindowParams &p, bool bf16, hipStream_t st);
void paged_plan_bf16(PagedParams &p);
void paged_plan_f32(PagedParams &p);
hipError_t paged_attend_bf16(const PagedParams &p, hipStream_t st);
hipError_t paged_attend_f32_launch(const PagedParams &p, hipStream_t st);
size_t tree_part_dim(bool bf16, int D);
void paged_evict_plan(PagedEvictParams &p);
size_t paged_evict_stage_bytes(const PagedEvictParams &p);
hipError_t paged_evict_launch(const PagedEvictParams &p, hipStream_t st);
}  // namespace reform

using namespace reform;

namespace {

constexpr int64_t kMaxPagedKeys = (1ll << 31) - 65536;   // keys are counted in 32-bit signed integers, some tiles or chunks past the last one
inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// An output that is another output or an input, where it is given at all.  (The workspace is asked for before the whole tensors are compared.)
bool shared(std::initializer_list<const void *> outs, std::initializer_list<const void *> ins)
{
    for (const void *const *x = outs.begin(); x != outs.end(); ++x) {
        if (!*x) continue;
        for (const void *const *y = x + 1; y != outs.end(); ++y)
            if (*x == *y) return true;
        for (const void *y : ins)
            if (*x == y) return true;
    }
    return false;
}

// ---------------------------------------------------------------------------------------
reform_status check_window(const reform_window_desc *d)
{
    if (!d || d->struct_size != sizeof(reform_window_desc) || d->reserved != 0) return REFORM_ERR_INVALID_ARG;
    const reform_status rc = check_heads(d->dtype, d->n_q_heads, d->n_kv_heads, d->head_dim, d->scale);
    if (rc == REFORM_ERR_INVALID_ARG) return rc;
    if (d->n_seq < 0 || d->n_q_rows < 0 || d->n_k_rows < 0 || d->window < 1 || d->n_sink < 0) return REFORM_ERR_INVALID_ARG;
    const int64_t strides[8] = {d->q_head_stride, d->q_row_stride, d->k_head_stride, d->k_row_stride,
                                d->v_head_stride, d->v_row_stride, d->o_head_stride, d->o_row_stride};
    const int64_t es = elt_size(d->dtype);
    for (int64_t s : strides)
        if (s < 0 || (s * es) % 16) return REFORM_ERR_INVALID_ARG;
    if (bad_out_strides(d->head_dim, {{d->n_q_heads, d->o_head_stride}, {d->n_q_rows, d->o_row_stride}})) return REFORM_ERR_INVALID_ARG;
    if (rc != REFORM_OK) return rc;
    if (d->n_seq > 65536 || (int64_t)d->n_kv_heads * d->n_k_rows >= (1ll << 30)) return REFORM_ERR_UNSUPPORTED;
    if ((double)d->n_q_heads * d->n_q_rows / 16.0 + (double)d->n_kv_heads * d->n_seq > kMaxGroups) return REFORM_ERR_UNSUPPORTED;
    if (d->k_row_stride >= kMaxRowStride || d->v_row_stride >= kMaxRowStride) return REFORM_ERR_UNSUPPORTED;
    return REFORM_OK;
}

WindowParams window_sizes(const reform_window_desc *d)
{
    WindowParams p;
    std::memset(&p, 0, sizeof(p));
    p.Hq = d->n_q_heads; p.Hkv = d->n_kv_heads; p.G = p.Hq / p.Hkv; p.D = d->head_dim;
    p.n_seq = d->n_seq; p.n_q = d->n_q_rows; p.n_k = d->n_k_rows;
    p.q_hs = d->q_head_stride; p.q_rs = d->q_row_stride; p.k_hs = d->k_head_stride; p.k_rs = d->k_row_stride;
    p.v_hs = d->v_head_stride; p.v_rs = d->v_row_stride; p.o_hs = d->o_head_stride; p.o_rs = d->o_row_stride;
    p.scale = d->scale;
    p.units = compute_units();
    // beyond the number of keys neither says more, and the kernels' sums with them stay within 32 bits
    p.window = d->window < d->n_k_rows ? d->window : d->n_k_rows > 0 ? d->n_k_rows : 1;
    p.n_sink = d->n_sink < d->n_k_rows ? d->n_sink : d->n_k_rows;
    // Where all blocks have as many tiles as the window shows, their order says nothing, and finding it takes 0.1 us and more (15 sequences
    // of together 4400 rows behind 4977 keys each, window 3, 32/8 heads of 64: 27.4 us sorted, 25.3 not; 17 of together 4000 rows, window 3743, 28/4: 23.2, 27.2).
    p.sorted = 2 * (int64_t)p.window * p.n_seq > p.n_k;
    return p;
}

// ---------------------------------------------------------------------------------------
// What the calls on a pool of pages have in common.
template <class DESC>
reform_status check_pool(const DESC *d)
{
    if (d->n_seq < 0 || d->page_len < 1 || d->n_pages < 0 || d->max_pages < 0 || d->max_len < 0 || d->n_sink < 0) return REFORM_ERR_INVALID_ARG;
    if ((int64_t)d->max_len > (int64_t)d->max_pages * d->page_len) return REFORM_ERR_INVALID_ARG;
    if (d->kv_page_stride < 0 || d->kv_head_stride < 0 || d->kv_row_stride < 0) return REFORM_ERR_INVALID_ARG;
    if (d->table_stride < 0 || d->score_seq_stride < 0 || d->score_head_stride < 0) return REFORM_ERR_INVALID_ARG;
    return REFORM_OK;
}

template <class DESC>
bool pool_too_large(const DESC *d)
{
    return (int64_t)d->n_pages * d->page_len >= (1ll << 31) || d->max_len > kMaxPagedKeys || d->kv_row_stride >= kMaxRowStride;
}

template <class DESC>
PagedPool pool_of(const DESC *d, const int32_t *page_table)
{
    PagedPool p;
    p.table = page_table;
    p.table_stride = d->table_stride;
    p.n_pages = (unsigned)d->n_pages;
    p.page_len = (unsigned)d->page_len;
    p.page_stride = d->kv_page_stride; p.head_stride = d->kv_head_stride; p.row_stride = d->kv_row_stride;
    // x / page_len by a product with 2^(32 + shift) / page_len rounded up, of which 2^32 is added as x itself: exact for x below 2^31
    p.shift = 0;
    while ((1ll << p.shift) < d->page_len) ++p.shift;
    const uint64_t one = 1ull << (32 + p.shift);
    p.magic = (unsigned)((one + (uint64_t)d->page_len - 1) / (uint64_t)d->page_len - (1ull << 32));
    return p;
}

template <class DESC>
Area pool_area(const DESC *d, const void *x)
{
    return area_of(x, elt_size(d->dtype), d->head_dim, {{d->n_pages, d->kv_page_stride}, {d->n_kv_heads, d->kv_head_stride}, {d->page_len, d->kv_row_stride}});
}

template <class DESC>
Area table_area(const DESC *d, const int32_t *x) { return area_of(x, 4, d->max_pages, {{d->n_seq, d->table_stride}}); }

// Of score, or of what has its strides.
template <class DESC>
Area score_area(const DESC *d, const void *x)
{
    return area_of(x, 4, d->max_len, {{d->n_seq, d->score_seq_stride}, {d->n_kv_heads, d->score_head_stride}});
}

reform_status check_paged(const reform_paged_desc *d)
{
    if (!d || d->struct_size != sizeof(reform_paged_desc) || d->reserved != 0) return REFORM_ERR_INVALID_ARG;
    reform_status rc = check_heads(d->dtype, d->n_q_heads, d->n_kv_heads, d->head_dim, d->scale);
    if (rc == REFORM_ERR_INVALID_ARG) return rc;
    if (check_pool(d) != REFORM_OK || d->window < 0) return REFORM_ERR_INVALID_ARG;
    if ((d->want_score != 0 && d->want_score != 1) || (d->accumulate != 0 && d->accumulate != 1)) return REFORM_ERR_INVALID_ARG;
    const int64_t strides[7] = {d->q_seq_stride, d->q_head_stride, d->o_seq_stride, d->o_head_stride,
                                d->kv_page_stride, d->kv_head_stride, d->kv_row_stride};
    const int64_t es = elt_size(d->dtype);
    for (int64_t s : strides)
        if (s < 0 || (s * es) % 16) return REFORM_ERR_INVALID_ARG;
    if (bad_out_strides(d->head_dim, {{d->n_seq, d->o_seq_stride}, {d->n_q_heads, d->o_head_stride}})) return REFORM_ERR_INVALID_ARG;
    if (d->want_score && bad_out_strides(d->max_len, {{d->n_seq, d->score_seq_stride}, {d->n_kv_heads, d->score_head_stride}}))
        return REFORM_ERR_INVALID_ARG;
    if (rc != REFORM_OK) return rc;
    if (pool_too_large(d) || (double)d->n_seq * d->n_q_heads > 4194304.0) return REFORM_ERR_UNSUPPORTED;
    // the list of all key tiles is counted in 32 bits (tree_list.h)
    const double blocks = std::ceil((double)(d->n_q_heads / d->n_kv_heads) / 16.0);
    if ((double)d->n_seq * d->n_kv_heads * blocks * ((double)d->max_len / 16.0 + 64.0) >= 2147483648.0) return REFORM_ERR_UNSUPPORTED;
    return REFORM_OK;
}

PagedParams paged_sizes(const reform_paged_desc *d, const int32_t *page_table)
{
    PagedParams p;
    std::memset(&p, 0, sizeof(p));
    p.pool = pool_of(d, page_table);
    p.n_seq = d->n_seq; p.Hq = d->n_q_heads; p.Hkv = d->n_kv_heads; p.G = p.Hq / p.Hkv; p.D = d->head_dim;
    p.max_len = d->max_len; p.window = d->window; p.n_sink = d->n_sink; p.accumulate = d->accumulate;
    p.q_ss = d->q_seq_stride; p.q_hs = d->q_head_stride; p.o_ss = d->o_seq_stride; p.o_hs = d->o_head_stride;
    p.score_ss = d->score_seq_stride; p.score_hs = d->score_head_stride;
    p.scale = d->scale;
    p.units = compute_units();
    if (d->dtype == REFORM_BF16) paged_plan_bf16(p);
    else paged_plan_f32(p);
    return p;
}

// The workspace's parts, in this order: pieces and their sums, then with a score the logits and the rows' sums.
struct PagedRoom {
    size_t part_o, part_ml, logits, row_ml;
    size_t all() const { return part_o + part_ml + logits + row_ml; }
};
PagedRoom paged_room(const reform_paged_desc *d, const PagedParams &p)
{
    const size_t rows = (size_t)2 * p.shares * p.row_blocks * p.part_rows, heads = (size_t)p.n_seq * p.Hq;
    PagedRoom r;
    r.part_o = align_up(rows * tree_part_dim(d->dtype == REFORM_BF16, p.D) * sizeof(float));
    r.part_ml = align_up(rows * sizeof(float2));
    r.logits = d->want_score ? align_up(heads * p.logit_keys * sizeof(float)) : 0;
    r.row_ml = d->want_score ? align_up(heads * sizeof(float2)) : 0;
    return r;
}

reform_status check_paged_evict(const reform_paged_evict_desc *d)
{
    if (!d || d->struct_size != sizeof(reform_paged_evict_desc) || !known_dtype(d->dtype)) return REFORM_ERR_INVALID_ARG;
    if (check_pool(d) != REFORM_OK || d->n_kv_heads <= 0 || d->head_dim <= 0) return REFORM_ERR_INVALID_ARG;
    if (d->budget < 1 || d->n_recent < 0 || (int64_t)d->n_sink + d->n_recent > d->budget) return REFORM_ERR_INVALID_ARG;
    if (bad_out_strides(d->head_dim, {{d->n_pages, d->kv_page_stride}, {d->n_kv_heads, d->kv_head_stride}, {d->page_len, d->kv_row_stride}}))
        return REFORM_ERR_INVALID_ARG;
    if (bad_out_strides(d->max_len, {{d->n_seq, d->score_seq_stride}, {d->n_kv_heads, d->score_head_stride}})) return REFORM_ERR_INVALID_ARG;
    const int64_t es = elt_size(d->dtype);
    if ((d->head_dim * es) % 16 || d->head_dim * es > 4096) return REFORM_ERR_UNSUPPORTED;
    if ((d->kv_page_stride * es) % 16 || (d->kv_head_stride * es) % 16 || (d->kv_row_stride * es) % 16) return REFORM_ERR_UNSUPPORTED;
    // workgroups of 1024 threads, two for each 128 bytes of a row and two more (evict_paged.hip)
    if (pool_too_large(d) || (double)d->n_seq * d->n_kv_heads * (d->head_dim * es / 64.0 + 4.0) > kMaxGroups / 2) return REFORM_ERR_UNSUPPORTED;
    return REFORM_OK;
}

PagedEvictParams evict_sizes(const reform_paged_evict_desc *d, const int32_t *page_table)
{
    PagedEvictParams p;
    std::memset(&p, 0, sizeof(p));
    p.pool = pool_of(d, page_table);
    p.n_seq = d->n_seq; p.Hkv = d->n_kv_heads; p.max_len = d->max_len;
    p.budget = d->budget; p.n_sink = d->n_sink; p.n_recent = d->n_recent;
    p.units = compute_units();
    p.elt = (int)elt_size(d->dtype);
    p.row_bytes = d->head_dim * p.elt;
    p.score_ss = d->score_seq_stride; p.score_hs = d->score_head_stride;
    paged_evict_plan(p);
    return p;
}

// The workspace's parts: kept keys, first rows that move, staged rows.
struct EvictRoom {
    size_t list, first, stage;
    size_t all() const { return list + first + stage; }
};
EvictRoom evict_room(const PagedEvictParams &p)
{
    if (p.max_len <= p.budget) return {0, 0, 0};         // nobody outgrows the budget
    const size_t items = (size_t)p.n_seq * p.Hkv;
    return {align_up(items * p.budget * sizeof(int32_t)), align_up(items * sizeof(int32_t)), align_up(paged_evict_stage_bytes(p))};
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------------------------------
size_t reform_window_attend_workspace(const reform_window_desc *d)
{
    return 0;
}

reform_status reform_window_attend(const reform_window_desc *d, const void *q, const void *k, const void *v, const int32_t *cu_q,
                                   const int32_t *cu_k, void *out, float *lse, void *workspace, size_t workspace_bytes,
                                   void *hip_stream)
{
    const reform_status rc = check_window(d);
    if (rc != REFORM_OK) return rc;
    if (d->n_q_rows == 0 || d->n_seq == 0) return REFORM_OK;
    if (!q || !out || !cu_q || (d->n_k_rows > 0 && (!k || !v))) return REFORM_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return REFORM_ERR_INVALID_ARG;
    if (shared({out, lse}, {q, k, v, cu_q, cu_k})) return REFORM_ERR_INVALID_ARG;
    WindowParams p = window_sizes(d);
    p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse; p.cu_q = cu_q; p.cu_k = cu_k;
    const int64_t es = elt_size(d->dtype), dim = d->head_dim;
    if (mixed({area_of(out, es, dim, {{p.Hq, p.o_hs}, {p.n_q, p.o_rs}}), area_of(lse, 4, (int64_t)p.Hq * p.n_q, {})},
              {area_of(q, es, dim, {{p.Hq, p.q_hs}, {p.n_q, p.q_rs}}), area_of(k, es, dim, {{p.Hkv, p.k_hs}, {p.n_k, p.k_rs}}),
               area_of(v, es, dim, {{p.Hkv, p.v_hs}, {p.n_k, p.v_rs}}), area_of(cu_q, 4, p.n_seq + 1, {}), area_of(cu_k, 4, p.n_seq + 1, {})}))
        return REFORM_ERR_INVALID_ARG;
    return window_attend_launch(p, d->dtype == REFORM_BF16, (hipStream_t)hip_stream) == hipSuccess ? REFORM_OK : REFORM_ERR_RUNTIME;
}

// ---------------------------------------------------------------------------------------
size_t reform_paged_attend_workspace(const reform_paged_desc *d)
{
    if (check_paged(d) != REFORM_OK || d->n_seq == 0) return 0;
    return paged_room(d, paged_sizes(d, nullptr)).all();
}

reform_status reform_paged_attend(const reform_paged_desc *d, const void *q, const void *k, const void *v, const int32_t *page_table,
                                  const int32_t *cache_len, float *score, void *out, float *lse, void *workspace,
                                  size_t workspace_bytes, void *hip_stream)
{
    const reform_status rc = check_paged(d);
    if (rc != REFORM_OK) return rc;
    if (d->n_seq == 0) return REFORM_OK;
    if (!q || !out || !cache_len || (d->want_score != 0) != (score != nullptr)) return REFORM_ERR_INVALID_ARG;
    if ((d->n_pages > 0 && (!k || !v)) || (d->max_pages > 0 && !page_table)) return REFORM_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return REFORM_ERR_INVALID_ARG;
    if (shared({out, lse, score}, {q, k, v, page_table, cache_len})) return REFORM_ERR_INVALID_ARG;
    PagedParams p = paged_sizes(d, page_table);
    p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse; p.score = score; p.cache_len = cache_len;
    const PagedRoom room = paged_room(d, p);
    if (room.all()) {
        if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < room.all()) return REFORM_ERR_WORKSPACE;
        char *at = (char *)workspace;
        p.part_o = (float *)at;
        p.part_ml = (float2 *)(at + room.part_o);
        p.logits = room.logits ? (float *)(at + room.part_o + room.part_ml) : nullptr;
        p.row_ml = room.row_ml ? (float2 *)(at + room.part_o + room.part_ml + room.logits) : nullptr;
    }
    const int64_t es = elt_size(d->dtype);
    if (mixed({area_of(out, es, p.D, {{p.n_seq, p.o_ss}, {p.Hq, p.o_hs}}), area_of(lse, 4, (int64_t)p.n_seq * p.Hq, {}), score_area(d, score)},
              {area_of(q, es, p.D, {{p.n_seq, p.q_ss}, {p.Hq, p.q_hs}}), pool_area(d, k), pool_area(d, v), table_area(d, page_table),
               area_of(cache_len, 4, p.n_seq, {})}))
        return REFORM_ERR_INVALID_ARG;
    hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = d->dtype == REFORM_BF16 ? paged_attend_bf16(p, st) : paged_attend_f32_launch(p, st);
    return e == hipSuccess ? REFORM_OK : REFORM_ERR_RUNTIME;
}

// ---------------------------------------------------------------------------------------
size_t reform_paged_evict_workspace(const reform_paged_evict_desc *d)
{
    if (check_paged_evict(d) != REFORM_OK || d->n_seq == 0) return 0;
    return evict_room(evict_sizes(d, nullptr)).all();
}

reform_status reform_paged_evict(const reform_paged_evict_desc *d, void *k, void *v, float *score, int32_t *pos,
                                 const int32_t *page_table, const int32_t *cache_len, int32_t *kept_idx, int32_t *new_len,
                                 void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const reform_status rc = check_paged_evict(d);
    if (rc != REFORM_OK) return rc;
    if (d->n_seq == 0) return REFORM_OK;
    if (!cache_len || (d->max_len > 0 && !score) || (d->n_pages > 0 && (!k || !v)) || (d->max_pages > 0 && !page_table)) return REFORM_ERR_INVALID_ARG;
    if (shared({k, v, score, pos, kept_idx, new_len}, {page_table, cache_len})) return REFORM_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v)) return REFORM_ERR_UNSUPPORTED;
    PagedEvictParams p = evict_sizes(d, page_table);
    p.k = k; p.v = v; p.score = score; p.pos = pos; p.kept = kept_idx; p.new_len = new_len; p.cache_len = cache_len;
    const EvictRoom room = evict_room(p);
    if (room.all()) {
        if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < room.all()) return REFORM_ERR_WORKSPACE;
        char *at = (char *)workspace;
        if (!p.kept) p.kept = (int32_t *)at;
        p.first = (int32_t *)(at + room.list);
        p.stage = at + room.list + room.first;
    }
    const int64_t items = (int64_t)p.n_seq * p.Hkv;
    if (mixed({pool_area(d, k), pool_area(d, v), score_area(d, score), score_area(d, pos), area_of(kept_idx, 4, items * p.budget, {}),
               area_of(new_len, 4, p.n_seq, {})},
              {table_area(d, page_table), area_of(cache_len, 4, p.n_seq, {})}))
        return REFORM_ERR_INVALID_ARG;
    return paged_evict_launch(p, (hipStream_t)hip_stream) == hipSuccess ? REFORM_OK : REFORM_ERR_RUNTIME;
}

}  // extern "C"
