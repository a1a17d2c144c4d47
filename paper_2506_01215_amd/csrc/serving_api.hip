// C ABI of the serving calls (see include/reform.h): rotary positions, packed prompts, drafted trees.  Host-side
// validation and kernel launches; nothing here allocates device memory or synchronises.
#include "../../include/reform.h"
#include "common.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

namespace reform {
hipError_t rotary_embed_launch(const RotaryParams &p, bool bf16, bool adjacent, hipStream_t st);
hipError_t tree_accept_launch(const AcceptParams &p, hipStream_t st);
void prompt_plan_bf16(PromptParams &p);
void prompt_plan_f32(PromptParams &p);
hipError_t prompt_attend_bf16(const PromptParams &p, hipStream_t st);
hipError_t prompt_attend_f32_launch(const PromptParams &p, hipStream_t st);
void tree_plan_bf16(TreeParams &p, int compute_units);
void tree_plan_f32(TreeParams &p, int compute_units);
hipError_t tree_attend_bf16(const TreeParams &p, hipStream_t st);
hipError_t tree_attend_f32_launch(const TreeParams &p, hipStream_t st);
size_t tree_part_dim(bool bf16, int D);
}  // namespace reform

using namespace reform;

namespace {

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
inline int64_t elt_size(int dtype) { return dtype == REFORM_BF16 ? 2 : 4; }
inline bool known_dtype(int dtype) { return dtype == REFORM_F32 || dtype == REFORM_BF16; }

struct Walk {
    int64_t n, step;
};

// Strides of something that is written: its pieces of `extent` elements, at every combination of the walks' steps, must not
// overlap.  Sorted by their steps, each walk's step has to pass over all that the ones before it cover.
bool bad_out_strides(int64_t extent, std::initializer_list<Walk> walks)
{
    Walk w[4];
    int n = 0;
    for (const Walk &x : walks) {
        if (x.step < 0) return true;
        if (x.n > 1) w[n++] = x;
    }
    std::sort(w, w + n, [](const Walk &x, const Walk &y) { return x.step < y.step; });
    double covered = (double)extent;
    for (int i = 0; i < n; ++i) {
        if ((double)w[i].step < covered) return true;
        covered += (double)(w[i].n - 1) * (double)w[i].step;
    }
    return false;
}

// What the attention calls support of types and heads.
reform_status check_heads(int32_t dtype, int32_t n_q, int32_t n_kv, int32_t dim, float scale)
{
    if (!known_dtype(dtype) || n_q <= 0 || n_kv <= 0 || n_q % n_kv || dim <= 0) return REFORM_ERR_INVALID_ARG;
    if (!(scale > 0.f) || !std::isfinite(scale)) return REFORM_ERR_INVALID_ARG;
    if (dtype == REFORM_BF16 ? dim != 64 && dim != 128 : dim % 4 || dim > 256) return REFORM_ERR_UNSUPPORTED;
    return REFORM_OK;
}

constexpr double kMaxGroups = 8388607.0;                 // workgroups of 512 threads in a grid
constexpr int64_t kMaxRowStride = 1 << 24;               // offsets inside a tile of 64 rows stay within 32 bits
// Keys of a sequence, and the row behind the tiles that a loop asks about next (two groups of waves, 64 keys a tile: up to 320 rows
// further), are counted in 32-bit signed integers.
constexpr int64_t kMaxTreeKeys = (1ll << 31) - 512;

reform_status check_prompt(const reform_prompt_desc *d)
{
    if (!d || d->struct_size != sizeof(reform_prompt_desc) || d->reserved != 0) return REFORM_ERR_INVALID_ARG;
    const reform_status rc = check_heads(d->dtype, d->n_q_heads, d->n_kv_heads, d->head_dim, d->scale);
    if (rc == REFORM_ERR_INVALID_ARG) return rc;
    if (d->n_seq < 0 || d->n_q_rows < 0 || d->n_k_rows < 0) return REFORM_ERR_INVALID_ARG;
    const int64_t strides[8] = {d->q_head_stride, d->q_row_stride, d->k_head_stride, d->k_row_stride,
                                d->v_head_stride, d->v_row_stride, d->o_head_stride, d->o_row_stride};
    const int64_t es = elt_size(d->dtype);
    for (int64_t s : strides)
        if (s < 0 || (s * es) % 16) return REFORM_ERR_INVALID_ARG;
    if (bad_out_strides(d->head_dim, {{d->n_q_heads, d->o_head_stride}, {d->n_q_rows, d->o_row_stride}})) return REFORM_ERR_INVALID_ARG;
    if (rc != REFORM_OK) return rc;
    if (d->n_seq > 65536 || (int64_t)d->n_kv_heads * d->n_k_rows >= (1ll << 30)) return REFORM_ERR_UNSUPPORTED;
    // workgroups of up to 512 threads, of which a grid has fewer than 2^32
    if ((double)d->n_q_heads * d->n_q_rows / 16.0 + (double)d->n_kv_heads * d->n_seq > kMaxGroups) return REFORM_ERR_UNSUPPORTED;
    if (d->k_row_stride >= kMaxRowStride || d->v_row_stride >= kMaxRowStride) return REFORM_ERR_UNSUPPORTED;
    return REFORM_OK;
}

int compute_units()
{
    const int n = device_compute_units();
    return n > 0 ? n : 256;
}

PromptParams prompt_sizes(const reform_prompt_desc *d)
{
    PromptParams p;
    std::memset(&p, 0, sizeof(p));
    p.Hq = d->n_q_heads; p.Hkv = d->n_kv_heads; p.G = p.Hq / p.Hkv; p.D = d->head_dim;
    p.n_seq = d->n_seq; p.n_q = d->n_q_rows; p.n_k = d->n_k_rows;
    p.q_hs = d->q_head_stride; p.q_rs = d->q_row_stride; p.k_hs = d->k_head_stride; p.k_rs = d->k_row_stride;
    p.v_hs = d->v_head_stride; p.v_rs = d->v_row_stride; p.o_hs = d->o_head_stride; p.o_rs = d->o_row_stride;
    p.scale = d->scale;
    p.units = compute_units();
    if (d->dtype == REFORM_BF16) prompt_plan_bf16(p);
    else prompt_plan_f32(p);
    return p;
}

size_t prompt_part_rows(const PromptParams &p) { return (size_t)2 * p.shares * p.part_rows; }

TreeParams tree_sizes(const reform_tree_desc *d)
{
    TreeParams p;
    std::memset(&p, 0, sizeof(p));
    p.n_seq = d->n_seq; p.Hq = d->n_q_heads; p.Hkv = d->n_kv_heads; p.G = p.Hq / p.Hkv; p.D = d->head_dim;
    p.T = d->n_nodes; p.max_len = d->max_cache_len;
    p.q_ss = d->q_seq_stride; p.q_hs = d->q_head_stride; p.q_rs = d->q_row_stride;
    p.o_ss = d->o_seq_stride; p.o_hs = d->o_head_stride; p.o_rs = d->o_row_stride;
    p.kv_ss = d->kv_seq_stride; p.kv_hs = d->kv_head_stride;
    p.scale = d->scale;
    if (d->dtype == REFORM_BF16) tree_plan_bf16(p, compute_units());
    else tree_plan_f32(p, compute_units());
    return p;
}

reform_status check_tree(const reform_tree_desc *d)
{
    if (!d || d->struct_size != sizeof(reform_tree_desc)) return REFORM_ERR_INVALID_ARG;
    const reform_status rc = check_heads(d->dtype, d->n_q_heads, d->n_kv_heads, d->head_dim, d->scale);
    if (rc == REFORM_ERR_INVALID_ARG) return rc;
    if (d->n_seq < 0 || d->n_nodes < 1 || d->max_cache_len < 0 || (int64_t)d->max_cache_len + d->n_nodes > d->capacity)
        return REFORM_ERR_INVALID_ARG;
    const int64_t strides[8] = {d->q_seq_stride, d->q_head_stride, d->q_row_stride, d->o_seq_stride,
                                d->o_head_stride, d->o_row_stride, d->kv_seq_stride, d->kv_head_stride};
    const int64_t es = elt_size(d->dtype);
    for (int64_t s : strides)
        if (s < 0 || (s * es) % 16) return REFORM_ERR_INVALID_ARG;
    if (rc != REFORM_OK) return rc;
    if (d->n_nodes > 64 || (int64_t)d->max_cache_len + d->n_nodes > kMaxTreeKeys) return REFORM_ERR_UNSUPPORTED;
    // the list of all key tiles is counted in 32 bits (tree_list.h): 16 rows and 16 keys are the smallest blocks and tiles
    if ((double)d->n_seq * d->n_q_heads * d->n_nodes > 4194304.0) return REFORM_ERR_UNSUPPORTED;
    const double blocks = std::ceil((double)d->n_nodes * (d->n_q_heads / d->n_kv_heads) / 16.0);
    if ((double)d->n_seq * d->n_kv_heads * blocks * (((double)d->max_cache_len + d->n_nodes) / 16.0 + 64.0) >= 2147483648.0)
        return REFORM_ERR_UNSUPPORTED;
    if (bad_out_strides(d->head_dim, {{d->n_seq, d->o_seq_stride}, {d->n_q_heads, d->o_head_stride}, {d->n_nodes, d->o_row_stride}}))
        return REFORM_ERR_INVALID_ARG;
    return REFORM_OK;
}

size_t tree_part_rows(const TreeParams &p) { return (size_t)2 * p.shares * p.row_blocks * p.part_rows; }

}  // namespace

extern "C" {

// ---------------------------------------------------------------------------------------
size_t reform_prompt_attend_workspace(const reform_prompt_desc *d)
{
    if (check_prompt(d) != REFORM_OK || d->n_seq == 0 || d->n_q_rows == 0) return 0;
    const PromptParams p = prompt_sizes(d);
    return prompt_part_rows(p) * (tree_part_dim(d->dtype == REFORM_BF16, p.D) * sizeof(float) + sizeof(float2));
}

reform_status reform_prompt_attend(const reform_prompt_desc *d, const void *q, const void *k, const void *v,
                                   const int32_t *cu_q, const int32_t *cu_k, void *out, float *lse, void *workspace,
                                   size_t workspace_bytes, void *hip_stream)
{
    const reform_status rc = check_prompt(d);
    if (rc != REFORM_OK) return rc;
    if (d->n_q_rows == 0 || d->n_seq == 0) return REFORM_OK;
    if (!q || !out || !cu_q || (d->n_k_rows > 0 && (!k || !v))) return REFORM_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return REFORM_ERR_INVALID_ARG;
    PromptParams p = prompt_sizes(d);
    p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse; p.cu_q = cu_q; p.cu_k = cu_k;
    if (p.shares) {
        const size_t row = tree_part_dim(d->dtype == REFORM_BF16, p.D) * sizeof(float);
        if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < prompt_part_rows(p) * (row + sizeof(float2)))
            return REFORM_ERR_WORKSPACE;
        p.part_o = (float *)workspace;
        p.part_ml = (float2 *)((char *)workspace + prompt_part_rows(p) * row);
    }
    hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = d->dtype == REFORM_BF16 ? prompt_attend_bf16(p, st) : prompt_attend_f32_launch(p, st);
    return e == hipSuccess ? REFORM_OK : REFORM_ERR_RUNTIME;
}

// ---------------------------------------------------------------------------------------
size_t reform_tree_attend_workspace(const reform_tree_desc *d)
{
    if (check_tree(d) != REFORM_OK || d->n_seq == 0) return 0;
    const TreeParams p = tree_sizes(d);
    return tree_part_rows(p) * (tree_part_dim(d->dtype == REFORM_BF16, p.D) * sizeof(float) + sizeof(float2));
}

reform_status reform_tree_attend(const reform_tree_desc *d, const void *q, const void *k, const void *v,
                                 const int32_t *cache_len, const int32_t *parent, const int32_t *node_count, void *out,
                                 float *lse, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const reform_status rc = check_tree(d);
    if (rc != REFORM_OK) return rc;
    if (d->n_seq == 0) return REFORM_OK;
    if (!q || !k || !v || !out || !cache_len) return REFORM_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return REFORM_ERR_INVALID_ARG;
    TreeParams p = tree_sizes(d);
    p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse; p.cache_len = cache_len; p.parent = parent; p.node_count = node_count;
    if (p.shares) {
        const size_t row = tree_part_dim(d->dtype == REFORM_BF16, p.D) * sizeof(float);
        if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < tree_part_rows(p) * (row + sizeof(float2)))
            return REFORM_ERR_WORKSPACE;
        p.part_o = (float *)workspace;
        p.part_ml = (float2 *)((char *)workspace + tree_part_rows(p) * row);
    }
    hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = d->dtype == REFORM_BF16 ? tree_attend_bf16(p, st) : tree_attend_f32_launch(p, st);
    return e == hipSuccess ? REFORM_OK : REFORM_ERR_RUNTIME;
}

// ---------------------------------------------------------------------------------------
reform_status reform_rotary_embed(const reform_rotary_desc *d, const void *q, const void *k, const void *v,
                                  const int32_t *pos, const int32_t *slot, void *q_out, void *k_out, void *v_out,
                                  void *hip_stream)
{
    if (!d || d->struct_size != sizeof(reform_rotary_desc) || !known_dtype(d->dtype)) return REFORM_ERR_INVALID_ARG;
    if (d->n_tokens < 0 || d->n_q_heads < 0 || d->n_kv_heads < 0 || d->head_dim <= 0) return REFORM_ERR_INVALID_ARG;
    if (d->rotary_dim < 0 || d->rotary_dim > d->head_dim || d->rotary_dim % 2) return REFORM_ERR_INVALID_ARG;
    if ((d->pairs != REFORM_PAIRS_HALVES && d->pairs != REFORM_PAIRS_ADJACENT) || (d->inverse != 0 && d->inverse != 1) ||
        d->scaling < REFORM_ROPE_PLAIN || d->scaling > REFORM_ROPE_BANDS)
        return REFORM_ERR_INVALID_ARG;
    if (!(d->theta > 1.0) || !std::isfinite(d->theta)) return REFORM_ERR_INVALID_ARG;
    if (!(d->magnitude > 0.f) || !std::isfinite(d->magnitude)) return REFORM_ERR_INVALID_ARG;
    if (d->scaling != REFORM_ROPE_PLAIN && (!(d->factor >= 1.0) || !std::isfinite(d->factor))) return REFORM_ERR_INVALID_ARG;
    if (d->scaling == REFORM_ROPE_BASE && d->rotary_dim == 2) return REFORM_ERR_INVALID_ARG;
    if (d->scaling == REFORM_ROPE_PARTS || d->scaling == REFORM_ROPE_BANDS) {
        if (d->original_len < 1 || !(d->turns_low > 0.0) || !(d->turns_high > d->turns_low) || !std::isfinite(d->turns_high))
            return REFORM_ERR_INVALID_ARG;
    }
    const bool has_q = d->n_q_heads > 0, has_k = d->n_kv_heads > 0, has_v = v != nullptr;
    const bool work = d->n_tokens > 0 && (has_q || has_k);
    if (work) {
        if (!pos || has_q != (q != nullptr) || has_q != (q_out != nullptr) || has_k != (k != nullptr) ||
            has_k != (k_out != nullptr) || has_v != (v_out != nullptr) || (has_v && !has_k))
            return REFORM_ERR_INVALID_ARG;
    }
    const int64_t strides[10] = {d->q_head_stride, d->q_row_stride, d->k_head_stride, d->k_row_stride, d->v_head_stride,
                                 d->v_row_stride, d->q_out_head_stride, d->q_out_row_stride, d->kv_out_head_stride,
                                 d->kv_out_row_stride};
    for (int64_t s : strides)
        if (s < 0) return REFORM_ERR_INVALID_ARG;
    const int64_t es = elt_size(d->dtype);
    if (has_q && bad_out_strides(d->head_dim, {{d->n_q_heads, d->q_out_head_stride}, {d->n_tokens, d->q_out_row_stride}}))
        return REFORM_ERR_INVALID_ARG;
    if (has_k && slot) {
        if (d->block_len < 1 || d->n_blocks < 1 || d->block_stride < 0) return REFORM_ERR_INVALID_ARG;
        if ((int64_t)d->block_len * d->n_blocks >= (1ll << 31)) return REFORM_ERR_UNSUPPORTED;
        if (bad_out_strides(d->head_dim, {{d->n_blocks, d->block_stride}, {d->n_kv_heads, d->kv_out_head_stride}, {d->block_len, d->kv_out_row_stride}}))
            return REFORM_ERR_INVALID_ARG;
        if ((d->block_stride * es) % 16) return REFORM_ERR_UNSUPPORTED;
    } else if (has_k && bad_out_strides(d->head_dim, {{d->n_kv_heads, d->kv_out_head_stride}, {d->n_tokens, d->kv_out_row_stride}})) {
        return REFORM_ERR_INVALID_ARG;
    }
    // in place: the same tensor in the same layout
    const bool same_q = q && q == q_out, same_k = k && k == k_out, same_v = v && v == v_out;
    if (same_q && (d->q_head_stride != d->q_out_head_stride || d->q_row_stride != d->q_out_row_stride)) return REFORM_ERR_INVALID_ARG;
    if (same_k && (slot || d->k_head_stride != d->kv_out_head_stride || d->k_row_stride != d->kv_out_row_stride))
        return REFORM_ERR_INVALID_ARG;
    if (same_v && (slot || d->v_head_stride != d->kv_out_head_stride || d->v_row_stride != d->kv_out_row_stride))
        return REFORM_ERR_INVALID_ARG;
    const int64_t unit = d->pairs == REFORM_PAIRS_HALVES ? 32 : 16;
    if ((d->head_dim * es) % 16 || d->head_dim > kRotaryMaxDim || (d->rotary_dim * es) % unit) return REFORM_ERR_UNSUPPORTED;
    for (int64_t s : strides)
        if ((s * es) % 16) return REFORM_ERR_UNSUPPORTED;
    for (const void *x : {q, k, v, (const void *)q_out, (const void *)k_out, (const void *)v_out})
        if (!aligned16(x)) return REFORM_ERR_UNSUPPORTED;
    if ((int64_t)d->n_q_heads + 2 * (int64_t)d->n_kv_heads > 65535) return REFORM_ERR_UNSUPPORTED;
    if ((double)d->n_tokens * (d->head_dim * es / 16) >= 2147483648.0) return REFORM_ERR_UNSUPPORTED;     // a thread for two pieces at least
    if (!work) return REFORM_OK;
    if ((q_out && (q_out == k_out || q_out == v_out)) || (k_out && k_out == v_out)) return REFORM_ERR_INVALID_ARG;
    RotaryParams p;
    std::memset(&p, 0, sizeof(p));
    const void *src[3] = {q, k, v};
    void *dst[3] = {q_out, k_out, v_out};
    for (int i = 0; i < 3; ++i) {
        p.src[i] = src[i];
        p.dst[i] = dst[i];
        p.src_hs[i] = strides[2 * i] * es;
        p.src_rs[i] = strides[2 * i + 1] * es;
        p.dst_hs[i] = (i ? d->kv_out_head_stride : d->q_out_head_stride) * es;
        p.dst_rs[i] = (i ? d->kv_out_row_stride : d->q_out_row_stride) * es;
        p.skip_rest[i] = src[i] == dst[i];
    }
    p.heads[0] = d->n_q_heads;
    p.heads[1] = d->n_kv_heads;
    p.heads[2] = has_v ? d->n_kv_heads : 0;
    p.pos = pos;
    p.n = d->n_tokens;
    p.rot = d->rotary_dim;
    p.elts = d->head_dim;
    p.inverse = d->inverse;
    p.magnitude = d->magnitude;
    if (has_k && slot) {
        p.slot = slot;
        p.block_len = d->block_len;
        p.n_slots = (unsigned)(d->block_len * d->n_blocks);
        p.block_bytes = d->block_stride * es;
    }
    p.scale = d->scaling == REFORM_ROPE_LINEAR ? 1.0 / d->factor : 1.0;
    if (d->rotary_dim) {
        const double rot = d->rotary_dim;
        double log2_theta = std::log2(d->theta);
        if (d->scaling == REFORM_ROPE_BASE) log2_theta += std::log2(d->factor) * rot / (rot - 2.0);
        p.neg2_log2_theta_over_rot = -2.0 * log2_theta / rot;
        const double two_pi = 6.283185307179586;
        if (d->scaling == REFORM_ROPE_PARTS) {
            const double at_high = rot * std::log(d->original_len / (two_pi * d->turns_high)) / (2.0 * std::log(d->theta));
            const double at_low = rot * std::log(d->original_len / (two_pi * d->turns_low)) / (2.0 * std::log(d->theta));
            const double low = std::fmin(std::fmax(std::floor(at_high), 0.0), rot - 1.0);
            const double high = std::fmin(std::fmax(std::ceil(at_low), 0.0), rot - 1.0);
            p.ramp = 1;
            p.ramp_at = low;
            p.ramp_inv = 1.0 / std::fmax(high - low, 0.001);
            p.ramp_low = 1.0 / d->factor;
        } else if (d->scaling == REFORM_ROPE_BANDS) {
            p.ramp = 2;
            p.turns = d->original_len / 4.0;             // frequencies are in quarter turns per position
            p.ramp_at = d->turns_high;
            p.ramp_inv = -1.0 / (d->turns_high - d->turns_low);
            p.ramp_low = 1.0 / d->factor;
        }
    }
    return rotary_embed_launch(p, d->dtype == REFORM_BF16, d->pairs == REFORM_PAIRS_ADJACENT, (hipStream_t)hip_stream) ==
                   hipSuccess ? REFORM_OK : REFORM_ERR_RUNTIME;
}

// ---------------------------------------------------------------------------------------
reform_status reform_tree_accept(const reform_accept_desc *d, const int32_t *parent, const int32_t *drafted,
                                 const int32_t *target, const int32_t *cache_len, const int32_t *node_count, void *k,
                                 void *v, int32_t *path, int32_t *accepted, int32_t *next_token, int32_t *new_len,
                                 void *hip_stream)
{
    if (!d || d->struct_size != sizeof(reform_accept_desc) || !known_dtype(d->dtype)) return REFORM_ERR_INVALID_ARG;
    if (d->n_seq < 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->n_layers <= 0) return REFORM_ERR_INVALID_ARG;
    if (d->n_nodes < 1 || d->capacity < d->n_nodes) return REFORM_ERR_INVALID_ARG;
    if ((k == nullptr) != (v == nullptr)) return REFORM_ERR_INVALID_ARG;
    if (d->n_seq > 0 && (!drafted || !target || !cache_len)) return REFORM_ERR_INVALID_ARG;
    // every workgroup of a sequence reads the inputs, one of them writes the outputs
    const int32_t *const in[5] = {parent, drafted, target, cache_len, node_count}, *const outs[4] = {path, accepted, next_token, new_len};
    for (int i = 0; i < 4 && d->n_seq > 0; ++i) {
        for (const int32_t *x : in)
            if (outs[i] && outs[i] == x) return REFORM_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (outs[i] && outs[i] == outs[j]) return REFORM_ERR_INVALID_ARG;
    }
    const int64_t es = elt_size(d->dtype), cache = (int64_t)d->capacity * d->head_dim;
    if (k) {
        if (k == v) return REFORM_ERR_INVALID_ARG;
        if (d->kv_seq_stride < 0 || d->kv_head_stride < 0 || d->kv_layer_stride < 0) return REFORM_ERR_INVALID_ARG;
    }
    if (d->n_nodes > 64) return REFORM_ERR_UNSUPPORTED;
    if ((d->head_dim * es) % 16 || d->head_dim * es > 4096) return REFORM_ERR_UNSUPPORTED;
    if (k && ((d->kv_seq_stride * es) % 16 || (d->kv_head_stride * es) % 16 || (d->kv_layer_stride * es) % 16 ||
              !aligned16(k) || !aligned16(v)))
        return REFORM_ERR_UNSUPPORTED;
    if (k && bad_out_strides(cache, {{d->n_layers, d->kv_layer_stride}, {d->n_seq, d->kv_seq_stride}, {d->n_kv_heads, d->kv_head_stride}}))
        return REFORM_ERR_INVALID_ARG;
    if ((double)d->n_layers * d->n_seq * d->n_kv_heads > 4194304.0) return REFORM_ERR_UNSUPPORTED;
    AcceptParams p;
    std::memset(&p, 0, sizeof(p));
    p.parent = parent; p.drafted = drafted; p.target = target; p.cache_len = cache_len; p.node_count = node_count;
    p.k = k; p.v = v; p.path = path; p.accepted = accepted; p.next_token = next_token; p.new_len = new_len;
    p.n_seq = d->n_seq; p.n_kv = d->n_kv_heads; p.n_nodes = d->n_nodes; p.n_layers = d->n_layers;
    p.capacity = d->capacity;
    p.row_bytes = (int)(d->head_dim * es);
    p.seq_bytes = d->kv_seq_stride * es; p.head_bytes = d->kv_head_stride * es; p.layer_bytes = d->kv_layer_stride * es;
    return tree_accept_launch(p, (hipStream_t)hip_stream) == hipSuccess ? REFORM_OK : REFORM_ERR_RUNTIME;
}

}  // extern "C"
