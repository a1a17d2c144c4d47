// fp32 attention of packed prompts and of drafted tokens (see reform_prompt_attend and reform_tree_attend in
// reform.h), on v_mfma_f32_16x16x4f32: fp32 operands, products and sums.
//
// A workgroup has 16 query rows, counted over the query rows and the heads of a KV group, and its eight waves
// take every eighth 16-key tile.  S^T = K Q^T: A[m][k]: lane l holds m = l % 16, k = l / 16; B[k][n]: n = l % 16,
// same k; C[m][n]: n = l % 16, m = 4 (l / 16) + e.  The contraction over the head takes its elements in the order
// 16 a + 4 (l / 16) + b, so a lane reads 16 bytes of a row at once; a lane then owns one query and the keys
// 4 (l / 16) + e, which is the B operand of O^T = V^T P^T for the contraction over those four keys, and V's
// operand is element l % 16 of row 4 (l / 16) + e: both straight from global memory, no LDS.
//
// Bound: the fp32 matrix pipe (0.15 PFLOP/s, of which it reaches 0.32 to 0.48: 2048 rows, 32/8 heads of 128, 534 us; 4096, 32/8 of 64, 926; 8 x 1000, 32/8 of 128, 1341) and,
// at the sizes of checks, latency (three prompts of up to 301 rows, 4 heads of 64: 11 us).  32 rows to a workgroup, so that K and V are read half
// as often: the same time for large batches, twice as long for small ones (60 batches, 1.27).
#include "attend_seq.h"
#include "prompt_share.h"

namespace reform {

constexpr int kF32Rows = 16, kF32Keys = 16, kF32Waves = 8;

template <int DP>
struct F32Sums {
    float o[kF32Waves / 2][kF32Rows][DP + 4];
    float m[kF32Waves][kF32Rows], l[kF32Waves][kF32Rows];
};

// As seq_segment: key tiles [t0, t1) of 16 keys for the 16 rows from r.row0 on; D <= DP elements a row.
template <int DP, bool TREE>
__device__ __forceinline__ void f32_segment(const SeqRows &r, const SeqKeys &s, int D, float scale, int t0, int t1, float *po,
                                            float2 *pml, F32Sums<DP> &sh)
{
    constexpr int NA = DP / 16;
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
    auto load_keys = [&](int t) {
        const float *kr = (const float *)s.k + (size_t)min(t * kF32Keys + ln, s.n - 1) * s.k_rs + 4 * lg;
#pragma unroll
        for (int a = 0; a < NA; ++a) k[a] = quad(kr, a);
    };
    int t = t0 + wave;
    if (AHEAD && t < t1) load_keys(t);
    // as in seq_segment: Q has to be there before the loop
#pragma unroll
    for (int a = 0; a < NA; ++a) asm volatile("" : "+v"(q[a]));
    for (; t < t1; t += kF32Waves) {
        const int j0 = t * kF32Keys;
        if (!AHEAD) load_keys(t);
        float v[4][NA];
        auto load_values = [&](int e) {
            const float *vr = (const float *)s.v + (size_t)min(j0 + 4 * lg + e, s.n - 1) * s.v_rs + ln;
#pragma unroll
            for (int a = 0; a < NA; ++a) {
                const bool in = 16 * a + ln < D;
                const float x = vr[in ? 16 * a : -ln];
                v[e][a] = in ? x : 0.f;
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
        if (j0 + kF32Keys - 1 >= s.open) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = j0 + 4 * lg + e, node = j - s.open;
                const bool seen = TREE ? node < 0 || (node < 64 && ((line >> (node & 63)) & 1ull)) : j <= lim;
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
            for (int a = 0; a < NA; ++a) o[a] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][a], p[e], o[a], 0, 0, 0);
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
    for (int a = 0; a < NA; ++a) {
        o[a] *= f;
        if (wave >= kF32Waves / 2) *(f32x4 *)&sh.o[wave - kF32Waves / 2][ln][16 * a + 4 * lg] = o[a];
    }
    __syncthreads();
    if (wave < kF32Waves / 2) {
#pragma unroll
        for (int a = 0; a < NA; ++a) *(f32x4 *)&sh.o[wave][ln][16 * a + 4 * lg] += o[a];
    }
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

template <int DP>
__global__ __launch_bounds__(kF32Waves * 64, 2) void prompt_attend_f32(PromptParams p)
{
    __shared__ F32Sums<DP> sh;
    const int kvh = blockIdx.x % p.Hkv;
    const PromptBlock blk = prompt_block<kF32Rows, kF32Keys>(p, blockIdx.x / p.Hkv);
    if (blk.rb < 0) return;
    SeqRows r;
    SeqKeys k;
    prompt_block_operands<float>(p, blk, kvh, blk.rb * kF32Rows, r, k);
    f32_segment<DP, false>(r, k, p.D, p.scale, 0, blk.tiles, nullptr, nullptr, sh);
}

template <int DP>
__global__ __launch_bounds__(kF32Waves * 64, 2) void prompt_attend_f32_shared(PromptParams p)
{
    __shared__ F32Sums<DP> sh;
    prompt_walk<float, kF32Rows, kF32Keys>(p, [&](const SeqRows &r, const SeqKeys &k, int t0, int t1, long slot) {
        f32_segment<DP, false>(r, k, p.D, p.scale, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * DP,
                               slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, sh);
    });
}

template <int DP>
__global__ __launch_bounds__(kF32Waves * 64, 2) void tree_attend_f32(TreeParams p)
{
    __shared__ F32Sums<DP> sh;
    tree_walk<float, kF32Rows, kF32Keys>(p, [&](const SeqRows &r, const SeqKeys &k, int t0, int t1, long slot) {
        f32_segment<DP, true>(r, k, p.D, p.scale, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * DP,
                              slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, sh);
    });
}

namespace {

template <int DP>
hipError_t launch_prompt(const PromptParams &p, hipStream_t st)
{
    if (p.shares) {
        hipLaunchKernelGGL((prompt_attend_f32_shared<DP>), dim3(p.shares), dim3(kF32Waves * 64), 0, st, p);
        prompt_merge_launch<DP, kF32Rows, kF32Keys, false>(p, st);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((prompt_attend_f32<DP>), dim3(prompt_grid(p, kF32Rows)), dim3(kF32Waves * 64), 0, st, p);
    return hipGetLastError();
}

template <int DP>
hipError_t launch_tree(const TreeParams &p, hipStream_t st)
{
    const unsigned grid = (unsigned)(p.shares ? p.shares : p.n_seq * p.Hkv) * p.row_blocks;
    hipLaunchKernelGGL((tree_attend_f32<DP>), dim3(grid), dim3(kF32Waves * 64), 0, st, p);
    if (p.shares) tree_merge_launch<DP, kF32Rows, kF32Keys, false>(p, st);
    return hipGetLastError();
}

}  // namespace

// A step is eight tiles of 16 keys by the waves of a workgroup, some 0.03 us for each element of a row (3.7 us at 128, 1.9 at 64), whether the chip
// is full or not.  What sharing out saves is the longest block's chain, for some 8 us; but where a sequence's blocks are then at different keys, each
// brings them from memory (ten rows, 12/4 heads of 96 behind 16000 keys 430 -> 48 us; 282 rows, 12/4 of 256 behind 4 x 3000 221 -> 396).
// 80 batches of 1 to 50 sequences behind up to 16000 keys each: 0.62 of the time without sharing, at worst 1.26 (three rows behind 200, 8/4 of 256).
void prompt_plan_f32(PromptParams &p)
{
    const double step = 0.03 * (p.D <= 32 ? 32 : p.D <= 64 ? 64 : p.D <= 128 ? 128 : 256), keys = (double)p.n_k / p.n_seq;
    const double blocks = ((double)p.n_q * p.G / kF32Rows + p.n_seq) * p.Hkv, full = blocks * (keys / 128.0 + 1.0) * step / p.units;
    const double alone = keys / 128.0 * step, memory = blocks * keys * p.D * 8.0 / 3.5e6;
    if (alone < 8.0 || p.n_seq > 64 || blocks * ((double)p.n_k / kF32Keys + 16.0) >= 33554432.0) return;          // as in prompt_share_rows
    if (std::cbrt(full * full * full + alone * alone * alone) < 8.0 + (full > memory ? full : memory)) return;
    const int rows = p.n_q * p.G;
    p.block = kF32Rows;
    p.part_rows = rows < kF32Rows ? rows : kF32Rows;
    p.least = kF32Waves;
    p.shares = 2 * p.units > kTreeMaxShares ? kTreeMaxShares : 2 * p.units;
}

hipError_t prompt_attend_f32_launch(const PromptParams &p, hipStream_t st)
{
    if (p.D <= 32) return launch_prompt<32>(p, st);
    if (p.D <= 64) return launch_prompt<64>(p, st);
    if (p.D <= 128) return launch_prompt<128>(p, st);
    return launch_prompt<256>(p, st);
}

// Elements of a row of the pieces: heads are padded to the next form.
size_t tree_part_dim(bool bf16, int D) { return bf16 ? D : D <= 32 ? 32 : D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// Fitted as in tree.hip, to 90 batches of 1 to 40 rows over 300 to 3000 keys in heads of 32 to 256: shares of a tile for each wave and more take
// 0.87 of the time that two tiles for each take, whole items of up to 1024 keys up to 4.8 times as much where heads are wide.  70 other batches of 1 to 64
// rows: 0.61 of all whole, at worst 1.21 times (37 rows of 8 x 4 caches of up to 432 keys, 128 wide, 21.7 us whole, 26.2).
void tree_plan_f32(TreeParams &p, int compute_units)
{
    const int whole = p.D <= 32 ? 1200 : p.D <= 64 ? 850 : p.D <= 128 ? 350 : 200;
    tree_plan(p, kF32Rows, kF32Keys, whole, kF32Waves, compute_units, 2 * compute_units);
}

hipError_t tree_attend_f32_launch(const TreeParams &p, hipStream_t st)
{
    if (p.D <= 32) return launch_tree<32>(p, st);
    if (p.D <= 64) return launch_tree<64>(p, st);
    if (p.D <= 128) return launch_tree<128>(p, st);
    return launch_tree<256>(p, st);
}

}  // namespace reform
