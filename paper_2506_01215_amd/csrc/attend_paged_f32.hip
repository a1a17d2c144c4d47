// One new token of each sequence over caches in pages, fp32 (see reform_paged_attend in reform.h), on v_mfma_f32_16x16x4f32 as
// attend_seq_f32.hip: 16 heads of a KV group to a workgroup, whose eight waves take every eighth 16-key tile; both products' operands
// come straight from memory, 16 bytes a lane.  Lane l % 16 looks up the row of that key of the tile, a tile ahead of its use.
//
// Bound: reading K and V once: 1073 MB of one cache of 131072 keys, 8 KV heads of 128, in 175 us (the call): 6.1 TB/s.
#include "paged_list.h"

namespace reform {

namespace {

constexpr int kRows = 16, kKeys = 16, kWaves = 8;

template <int DP>
struct PagedSumsF32 {
    float o[kWaves / 2][kRows][DP + 4];
    float m[kWaves][kRows], l[kWaves][kRows];
    float2 row[kRows];
};

// As paged_segment of the bf16 form; D <= DP elements a row.  STREAM: V goes past the caches' order of replacement; pieces of K's lines are read
// by different loads, so K does not (us without, V, both: 655 MB 129.0, 121.4, 122.9; 131 MB in heads of 64 33.4, 30.3; 65 MB of 256 27.9, 29.6).
template <int DP, bool STREAM>
__device__ __forceinline__ void paged_segment_f32(const PagedParams &p, int b, int kvh, int len, int row0, int t0, int t1, float *po, float2 *pml,
                                                  PagedSumsF32<DP> &sh)
{
    // V^T's operand of a product is element l % 16 of a row of 16; which 16 of the head's elements these are is free.  A lane takes VEC
    // adjacent ones for as many products, with one load.
    constexpr int NA = DP / 16, VEC = NA < 4 ? NA : 4, NV = NA / VEC;
    typedef float quadlet __attribute__((ext_vector_type(VEC)));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ln = lane & 15, lg = lane >> 4, D = p.D, rows = p.G - row0;
    const PagedSpan<kKeys> span(p, len);
    const float *const K = (const float *)p.k + (size_t)kvh * p.pool.head_stride, *const V = (const float *)p.v + (size_t)kvh * p.pool.head_stride;
    const int32_t *table = p.pool.table + (size_t)b * p.pool.table_stride;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    // where the row of key l % 16 of tile u is, -1 where it is not seen
    auto look = [&](int u) {
        if (u >= t1) return -1l;
        const int j = span.tile(u) * kKeys + ln;
        return span.seen(j) ? pool_row(p.pool, table, j) : -1l;
    };
    // elements behind the head's last one count as 0
    auto quad = [&](const float *from, int a) { return 16 * a + 4 * lg < D ? *(const f32x4 *)(from + 16 * a + 4 * lg) : zero; };
    f32x4 q[NA], o[NA];
    {
        const float *src = (const float *)p.q + (size_t)b * p.q_ss + (size_t)(kvh * p.G + row0 + min(ln, rows - 1)) * p.q_hs;
#pragma unroll
        for (int a = 0; a < NA; ++a) {
            q[a] = quad(src, a);
            o[a] = zero;
        }
    }
    float m = -INFINITY, l = 0.f;
    const float c = p.scale * kLog2e;
    float *const logits = p.logits && ln < rows ? p.logits + ((size_t)b * p.Hq + (size_t)kvh * p.G + row0 + ln) * p.logit_keys + 4 * lg : nullptr;
    // K of the next tile and V of this one are on their way while the tile's logits are formed (rows of up to 128 elements: there
    // are no registers for it beyond)
    constexpr bool AHEAD = DP <= 128;
    f32x4 k[NA];
    auto load_keys = [&](long at) {
#pragma unroll
        for (int a = 0; a < NA; ++a) k[a] = zero;
        if (at < 0) return;
#pragma unroll
        for (int a = 0; a < NA; ++a) k[a] = quad(K + at, a);
    };
    int u = t0 + wave;
    long here = look(u), next = look(u + kWaves);
    if (AHEAD) load_keys(here);
    // Q has to be there before the loop: a wait inside it would be one for the next tile's loads as well, in every trip
#pragma unroll
    for (int a = 0; a < NA; ++a) asm volatile("" : "+v"(q[a]));
    for (; u < t1; u += kWaves) {
        if (!AHEAD) load_keys(here);
        quadlet v[4][NV];
        auto load_values = [&](int e) {
            const int from = 4 * lg + e;                 // lane of the key's place
            const long at = ((long)__shfl((int)(here >> 32), from) << 32) | (unsigned)__shfl((int)here, from);
#pragma unroll
            for (int a = 0; a < NV; ++a) {
                v[e][a] = (quadlet)(0.f);
                if (at >= 0 && VEC * (16 * a + ln) < D) {
                    const quadlet *from = (const quadlet *)(V + at + VEC * (16 * a + ln));
                    v[e][a] = STREAM ? __builtin_nontemporal_load(from) : *from;
                }
            }
        };
        if (AHEAD) {
#pragma unroll
            for (int e = 0; e < 4; ++e) load_values(e);
        }
        f32x4 x = zero;
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x4f32(k[a][e], q[a][e], x, 0, 0, 0);
        const unsigned seen = (unsigned)__builtin_amdgcn_ballot_w64(here >= 0) & 0xffffu;
        const long after = look(u + 2 * kWaves);
        if (AHEAD) load_keys(next);
        if (seen != 0xffffu) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!((seen >> (4 * lg + e)) & 1u)) x[e] = -INFINITY;
        }
        if (logits) *(f32x4 *)(logits + (size_t)u * kKeys) = x;
        float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m, mx);
        const float ref = m_new == -INFINITY ? 0.f : m_new * c;             // -inf: no key yet
        const float alpha = __builtin_amdgcn_exp2f(fmaf(m, c, -ref));
        m = m_new;
        f32x4 pr;
#pragma unroll
        for (int e = 0; e < 4; ++e) pr[e] = __builtin_amdgcn_exp2f(fmaf(x[e], c, -ref));
        l = fmaf(l, alpha, (pr[0] + pr[1]) + (pr[2] + pr[3]));
#pragma unroll
        for (int a = 0; a < NA; ++a) o[a] *= alpha;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!AHEAD) load_values(e);
#pragma unroll
            for (int a = 0; a < NA; ++a) o[a] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][a / VEC][a % VEC], pr[e], o[a], 0, 0, 0);
        }
        here = next;
        next = after;
    }
    // the waves' sums, as in seq_segment
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (lg == 0) { sh.m[wave][ln] = m; sh.l[wave][ln] = l; }
    __syncthreads();
    float m_all = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m_all = fmaxf(m_all, sh.m[w][ln]);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_all) * c);
#pragma unroll
    for (int a = 0; a < NA; ++a) o[a] *= f;
    // element e of product a is element VEC (16 (a / VEC) + 4 lg + e) + a % VEC of the head
    auto meet = [&](float *row, bool add) {
#pragma unroll
        for (int a = 0; a < NV; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                quadlet *const to = (quadlet *)(row + VEC * (16 * a + 4 * lg + e));
                quadlet y = add ? *to : (quadlet)(0.f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) y[i] += o[a * VEC + i][e];
                *to = y;
            }
    };
    if (wave >= kWaves / 2) meet(sh.o[wave - kWaves / 2][ln], false);
    __syncthreads();
    if (wave < kWaves / 2) meet(sh.o[wave][ln], true);
    __syncthreads();
    for (int i = threadIdx.x; i < min(kRows, rows) * (DP / 4); i += kWaves * 64) {
        const int row = i / (DP / 4), c4 = i % (DP / 4) * 4;
        f32x4 y = *(const f32x4 *)&sh.o[0][row][c4];
#pragma unroll
        for (int w = 1; w < kWaves / 2; ++w) y += *(const f32x4 *)&sh.o[w][row][c4];
        float m_row = -INFINITY, l_row = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m_row = fmaxf(m_row, sh.m[w][row]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w)                 // multiplied, not left out: NaN logits alone leave -inf and a NaN sum
            l_row += sh.l[w][row] * (sh.m[w][row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((sh.m[w][row] - m_row) * c));
        if (pml) {
            *(f32x4 *)(po + (size_t)row * DP + c4) = y;
            if (c4 == 0) pml[row] = make_float2(m_row * c, l_row);
            continue;
        }
        const int head = kvh * p.G + row0 + row;
        const float inv = l_row == 0.f ? 0.f : 1.0f / l_row;                // 0: the row sees no key
        if (c4 < D) *(f32x4 *)((float *)p.out + (size_t)b * p.o_ss + (size_t)head * p.o_hs + c4) = y * inv;
        if (c4 == 0) {
            if (p.lse) p.lse[(size_t)b * p.Hq + head] = (m_row * c + __builtin_amdgcn_logf(l_row)) * kLn2;
            if (paged_scores_alone(p)) sh.row[row] = score_row(m_row * c, l_row);
            else if (p.row_ml) p.row_ml[(size_t)b * p.Hq + head] = make_float2(m_row * c, l_row);
        }
    }
    if (paged_scores_alone(p)) {
        __syncthreads();                                 // rows and logits are there
        int counter = 0;
        paged_score<kKeys>(p, b, kvh, len, t0, t1, counter, wave, kWaves, [&](int) { return sh.row[min(lane, rows - 1)]; });
    }
}

template <int DP, bool STREAM>
__global__ __launch_bounds__(kWaves * 64, 2) void paged_attend_f32(PagedParams p)
{
    __shared__ PagedSumsF32<DP> sh;
    list_walk<kRows, kKeys>(p, [&](int b, const TreeSeq &seq, int kvh, int rb, int t0, int t1, long slot) {
        paged_segment_f32<DP, STREAM>(p, b, kvh, seq.len, rb * kRows, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * DP,
                              slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, sh);
    });
}

template <int DP>
hipError_t launch(const PagedParams &p, hipStream_t st)
{
    const unsigned grid = (unsigned)(p.shares ? p.shares : p.n_seq * p.Hkv) * p.row_blocks;
    if (p.stream) hipLaunchKernelGGL((paged_attend_f32<DP, true>), dim3(grid), dim3(kWaves * 64), 0, st, p);
    else hipLaunchKernelGGL((paged_attend_f32<DP, false>), dim3(grid), dim3(kWaves * 64), 0, st, p);
    paged_join_launch<DP, kRows, kKeys, false>(p, st);
    return hipGetLastError();
}

}  // namespace

// Keys that a workgroup takes whole: fitted to 22 batches of 1 to 48 caches of up to 3000 keys, with scores and without, in heads of 64 and
// 128, each whole and shared out: 1.01 times the better of the two in the mean, at worst 1.08.  Narrower heads in proportion, wider ones by two batches
// of 109 and 149 keys (whole 16.2 and 18.5 us, shared out 19.4 and 22.6).
//
// Shares: as many as run at once, two a compute unit in up to 128 registers and one beyond (heads of 128, two / one, us: 2 caches of 4000 keys, 8 KV
// heads, 31.6 / 22.0, 4 of 20000 128.6 / 122.7; of 256: 8 of 4000, 2 KV heads, 60.1 / 43.3; of 64: 8 of 4000, 8 KV heads, 33.4 / 34.4; of 32: 36.1 / 43.3).
void paged_plan_f32(PagedParams &p)
{
    const int whole = p.D <= 32 ? 900 : p.D <= 64 ? 450 : p.D <= 128 ? 250 : 175;
    paged_plan(p, kRows, kKeys, whole, kWaves, p.D <= 64 ? 2 * p.units : p.units);
}

hipError_t paged_attend_f32_launch(const PagedParams &p, hipStream_t st)
{
    if (p.D <= 32) return launch<32>(p, st);
    if (p.D <= 64) return launch<64>(p, st);
    if (p.D <= 128) return launch<128>(p, st);
    return launch<256>(p, st);
}

}  // namespace reform
