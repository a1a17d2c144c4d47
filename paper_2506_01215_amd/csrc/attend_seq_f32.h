// fp32 attention of a block of 16 query rows over a range of one sequence's keys, on v_mfma_f32_16x16x4f32: fp32 operands, products
// and sums.
//
// A workgroup has 16 query rows, counted over the query rows and the heads of a KV group, and its eight waves
// take every eighth 16-key tile.  S^T = K Q^T: A[m][k]: lane l holds m = l % 16, k = l / 16; B[k][n]: n = l % 16,
// same k; C[m][n]: n = l % 16, m = 4 (l / 16) + e.  The contraction over the head takes its elements in the order
// 16 a + 4 (l / 16) + b, so a lane reads 16 bytes of a row at once; a lane then owns one query and the keys
// 4 (l / 16) + e, which is the B operand of O^T = V^T P^T for the contraction over those four keys, and V's
// operand is an element of row 4 (l / 16) + e for each l % 16: both straight from global memory, no LDS.
#pragma once
#include "attend_seq.h"

namespace reform {

constexpr int kF32Rows = 16, kF32Keys = 16, kF32Waves = 8;

template <int DP>
struct F32Sums {
    float o[kF32Waves / 2][kF32Rows][DP + 4];
    float m[kF32Waves][kF32Rows], l[kF32Waves][kF32Rows];
};

// As seq_segment: key tiles [t0, t1) of 16 keys for the 16 rows from r.row0 on; D <= DP elements a row.
template <int DP, bool TREE, class KEYS>
__device__ __forceinline__ void f32_segment(const SeqRows &r, const KEYS &s, int D, float scale, int t0, int t1, float *po,
                                            float2 *pml, F32Sums<DP> &sh)
{
    constexpr bool WINDOW = std::is_same<KEYS, WindowKeys>::value;
    // V^T's operand of a product is element l % 16 of a row of 16; which 16 of the head's elements these are is free.  A lane takes VEC
    // adjacent ones for as many products, with one load (element by element / so, us: prompts of 864 rows, 24/8 heads of 64, 35.7 / 32.6, 8/2 of 256
    // 51.8 / 46.7; 8 nodes over three caches, 32/8 of 128, 36.9 / 33.2; 512 rows with a window, 16/2 of 128, 28.3 / 25.3).
    constexpr int NA = DP / 16, VEC = NA < 4 ? NA : 4, NV = NA / VEC;
    typedef float quadlet __attribute__((ext_vector_type(VEC)));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ln = lane & 15, lg = lane >> 4;
    unsigned long long line = 0ull;
    if (TREE && t1 * kF32Keys > s.open) line = tree_line(s.parent, s.nodes);
    const int row = min(r.row0 + ln, r.rows - 1), at = row / r.G;
    const int lim = s.shift + at;
    if (TREE) line = ((unsigned long long)(unsigned)__shfl((int)(line >> 32), at) << 32) | (unsigned)__shfl((int)line, at);
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    // elements behind the head's last one count as 0: loaded from the row's start, so that no load hangs on a branch
    auto quad = [&](const float *from, int a) {
        const bool in = 16 * a + 4 * lg < D;
        const f32x4 x = *(const f32x4 *)(from + (in ? 16 * a : -4 * lg));
        return in ? x : zero;
    };
    f32x4 q[NA], o[NA];
    {
        const float *src = (const float *)r.q + (size_t)(row % r.G) * r.q_hs + (size_t)at * r.q_rs + 4 * lg;
#pragma unroll
        for (int a = 0; a < NA; ++a) {
            q[a] = quad(src, a);
            o[a] = zero;
        }
    }
    float m = -INFINITY, l = 0.f;
    const float c = scale * kLog2e;
    // K of the next tile and V of this one are on their way while the tile's logits are formed (rows of up to 128
    // elements: there are no registers for it beyond)
    constexpr bool AHEAD = DP <= 128;
    f32x4 k[NA];
    auto load_keys = [&](int u) {
        const float *kr = (const float *)s.k + (size_t)min(key_of(s, u * kF32Keys + ln), s.n - 1) * s.k_rs + 4 * lg;
#pragma unroll
        for (int a = 0; a < NA; ++a) k[a] = quad(kr, a);
    };
    int t = t0 + wave;
    if (AHEAD && t < t1) load_keys(t);
    // as in seq_segment: Q has to be there before the loop
#pragma unroll
    for (int a = 0; a < NA; ++a) asm volatile("" : "+v"(q[a]));
    int behind = -1, stay = 0;                           // as in seq_segment
    if constexpr (WINDOW) {
        behind = __builtin_amdgcn_readlane(lim, 15) - s.window;
        stay = s.stay;
    }
    for (; t < t1; t += kF32Waves) {
        const int j0 = key_start<kF32Keys>(s, t);
        if (!AHEAD) load_keys(t);
        quadlet v[4][NV];
        auto load_values = [&](int e) {
            const float *vr = (const float *)s.v + (size_t)min(key_of(s, t * kF32Keys + 4 * lg + e), s.n - 1) * s.v_rs;
#pragma unroll
            for (int a = 0; a < NV; ++a) {
                const int from = VEC * (16 * a + ln);
                const quadlet x = *(const quadlet *)(vr + (from < D ? from : 0));
                v[e][a] = from < D ? x : (quadlet)(0.f);
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
        if (AHEAD && t + kF32Waves < t1) load_keys(t + kF32Waves);
        if (j0 + kF32Keys - 1 >= s.open || (WINDOW && j0 <= behind && j0 + kF32Keys > stay)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = key_of(s, t * kF32Keys + 4 * lg + e), node = j - s.open;
                bool seen = TREE ? node < 0 || (node < 64 && ((line >> (node & 63)) & 1ull)) : j <= lim;
                if constexpr (WINDOW) seen = seen && (j > lim - s.window || j < stay);
                if (!seen) x[e] = -INFINITY;
            }
        }
        float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m, mx);
        const float ref = m_new == -INFINITY ? 0.f : m_new * c;             // -inf: the row sees no key yet
        const float alpha = __builtin_amdgcn_exp2f(fmaf(m, c, -ref));
        m = m_new;
        f32x4 p;
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(x[e], c, -ref));
        l = fmaf(l, alpha, (p[0] + p[1]) + (p[2] + p[3]));
#pragma unroll
        for (int a = 0; a < NA; ++a) o[a] *= alpha;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!AHEAD) load_values(e);
#pragma unroll
            for (int a = 0; a < NA; ++a) o[a] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][a / VEC][a % VEC], p[e], o[a], 0, 0, 0);
        }
    }
    // the waves' sums, as in seq_segment
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (lg == 0) { sh.m[wave][ln] = m; sh.l[wave][ln] = l; }
    __syncthreads();
    float m_all = -INFINITY;
#pragma unroll
    for (int w = 0; w < kF32Waves; ++w) m_all = fmaxf(m_all, sh.m[w][ln]);
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
    if (wave >= kF32Waves / 2) meet(sh.o[wave - kF32Waves / 2][ln], false);
    __syncthreads();
    if (wave < kF32Waves / 2) meet(sh.o[wave][ln], true);
    __syncthreads();
    const int rows_here = min(kF32Rows, r.rows - r.row0);
    for (int i = threadIdx.x; i < rows_here * (DP / 4); i += kF32Waves * 64) {
        const int ri = i / (DP / 4), c4 = i % (DP / 4) * 4;
        f32x4 y = *(const f32x4 *)&sh.o[0][ri][c4];
#pragma unroll
        for (int w = 1; w < kF32Waves / 2; ++w) y += *(const f32x4 *)&sh.o[w][ri][c4];
        float m_row = -INFINITY, l_row = 0.f;
#pragma unroll
        for (int w = 0; w < kF32Waves; ++w) m_row = fmaxf(m_row, sh.m[w][ri]);
#pragma unroll
        for (int w = 0; w < kF32Waves; ++w)              // multiplied, not left out: NaN logits alone leave -inf and a NaN sum
            l_row += sh.l[w][ri] * (sh.m[w][ri] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((sh.m[w][ri] - m_row) * c));
        if (pml) {
            *(f32x4 *)(po + (size_t)ri * DP + c4) = y;
            if (c4 == 0) pml[ri] = make_float2(m_row * c, l_row);
            continue;
        }
        const int qr = (r.row0 + ri) / r.G, head = (r.row0 + ri) % r.G;
        const float inv = l_row == 0.f ? 0.f : 1.0f / l_row;                // 0: the row sees no key
        if (c4 < D) *(f32x4 *)((float *)r.out + (size_t)head * r.o_hs + (size_t)qr * r.o_rs + c4) = y * inv;
        if (c4 == 0 && r.lse) r.lse[(size_t)head * r.lse_hs + qr] = (m_row * c + __builtin_amdgcn_logf(l_row)) * kLn2;
    }
}

}  // namespace reform
