// Attention of a block of query rows over a range of one sequence's keys, by one workgroup whose waves share
// out the keys (bf16: also the rows): the short prompts' form and the drafted tokens' share it.
//
// Rows are counted over a sequence's query rows and the G heads of a KV group together (row r is query row
// r / G of head r % G), so K and V are read once for all of them.  Softmax in one pass with a running
// reference maximum and sum; logits, sums and outputs in fp32, the probabilities of P.V rounded to bf16 in
// the bf16 form (the matrix instruction takes nothing wider; 2^-9 of a probability, as in attend_bf16.hip).
#pragma once
#include "attend_tile.h"

#include <atomic>

namespace reform {

// More than the default 64 KB of LDS for a kernel: once per kernel and device, not per launch.
template <auto KERNEL>
inline hipError_t raise_lds(size_t bytes)
{
    static std::atomic<bool> raised[64];
    int dev = 0;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev >= 0 && dev < 64 && raised[dev].load(std::memory_order_acquire)) return hipSuccess;
    const hipError_t f = hipFuncSetAttribute((const void *)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (f == hipSuccess && dev >= 0 && dev < 64) raised[dev].store(true, std::memory_order_release);
    return f;
}

struct SeqRows {
    const void *q;           // first row of the group's first head
    void *out;
    float *lse;              // nullable
    long q_hs, q_rs, o_hs, o_rs, lse_hs;     // elements
    int G, row0, rows;       // first row of the block, rows of the sequence
};

struct SeqKeys {
    const void *k, *v;       // first key of the KV head
    long k_rs, v_rs;         // elements
    int n;                   // keys of the sequence (>= 1 where a range is not empty)
    int open;                // keys below it are seen by every row of the block
    int shift;               // prompts: query row i sees keys j <= i + shift
    const int *parent;       // trees (open = first drafted key): parents of the nodes, null: a chain
    int nodes;
};

// Drafted nodes that node `lane` sees: itself and its ancestors, one bit each, one node per lane of a wave.
// Six doublings: after step m the word holds the 2^m nearest of the line and `up` points 2^m nodes up.
__device__ __forceinline__ unsigned long long tree_line(const int *parent, int nodes)
{
    const int lane = threadIdx.x & 63;
    if (!parent) return lane == 63 ? ~0ull : (2ull << lane) - 1ull;
    int up = -1;
    if (lane < nodes) {
        up = parent[lane];
        if (up >= lane || up < 0) up = -1;
    }
    unsigned lo = lane < 32 ? 1u << lane : 0u, hi = lane < 32 ? 0u : 1u << (lane - 32);
#pragma unroll
    for (int m = 0; m < 6; ++m) {
        const int from = up < 0 ? lane : up;
        lo |= (unsigned)__shfl((int)lo, from);
        hi |= (unsigned)__shfl((int)hi, from);
        const int above = __shfl(up, from);
        up = up < 0 ? -1 : above;
    }
    return ((unsigned long long)hi << 32) | lo;
}

constexpr int kSeqWaves = 8;

// RG waves side by side take RG * 16 NB rows; the KG = 8 / RG groups of them divide the key tiles of TK
// keys.  RG = 1: a wave's tiles are its own, no barrier in the loop.
template <int D, int NB, int RG>
struct SeqShape {
    static constexpr int KG = kSeqWaves / RG, R = 16 * NB * RG, TK = RG == 8 ? 64 : 32, SUB = TK / 32;
    static constexpr int C8 = D / 8, ROW = D + 16, TILE = TK * ROW, GT = 64 * RG;
    static constexpr int PIECES = TK * C8 / GT, BUFS = RG == 1 ? 1 : 2;
    static constexpr int SL = KG > 1 ? KG / 2 : 1, OROW = D + 4;
    static constexpr size_t stage_bytes = sizeof(u16) * (size_t)BUFS * KG * 2 * TILE;
    static constexpr size_t sum_bytes = sizeof(float) * (size_t)SL * R * OROW;
    static constexpr size_t base_bytes = (stage_bytes > sum_bytes ? stage_bytes : sum_bytes);
    static constexpr size_t lds_bytes = base_bytes + sizeof(float) * 2 * kSeqWaves * 16 * NB;
};

// Key tiles [t0, t1) of the sequence (may be empty).  po, pml: null for a final result, else this block's
// unnormalised sums [rows][D] and (reference maximum in log2 units, sum) [rows].
// On entry nothing in `smem` may be in use by any wave.
template <int D, int NB, int RG, bool TREE>
__device__ __forceinline__ void seq_segment(const SeqRows &r, const SeqKeys &s, float scale, int t0, int t1, float *po,
                                            float2 *pml, char *smem)
{
    using S = SeqShape<D, NB, RG>;
    constexpr int KS = D / 32, DB = D / 16, C8 = S::C8, ROW = S::ROW, TILE = S::TILE, KG = S::KG, TK = S::TK;
    float *sm = (float *)(smem + S::base_bytes), *sl = sm + kSeqWaves * 16 * NB;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ln = lane & 15, lg = lane >> 4;
    const int rg = wave % RG, kg = wave / RG, tg = rg * 64 + lane;

    // 16-byte pieces of a tile: piece i of a thread lies in row tg / C8 + i * (GT / C8)
    v4u kreg[S::PIECES], vreg[S::PIECES];
    const uint32_t koff = (uint32_t)((tg / C8) * (int)s.k_rs + tg % C8 * 8) * 2u;
    const uint32_t voff = (uint32_t)((tg / C8) * (int)s.v_rs + tg % C8 * 8) * 2u;
    auto load = [&](int t) {
        const char *kt = (const char *)((const u16 *)s.k + (size_t)t * TK * s.k_rs);
        const char *vt = (const char *)((const u16 *)s.v + (size_t)t * TK * s.v_rs);
        const int last = s.n - 1 - t * TK;
        if (last >= TK - 1) {
#pragma unroll
            for (int i = 0; i < S::PIECES; ++i) {
                kreg[i] = *(const v4u *)(kt + (koff + (uint32_t)(i * (S::GT / C8) * (int)s.k_rs) * 2u));
                vreg[i] = *(const v4u *)(vt + (voff + (uint32_t)(i * (S::GT / C8) * (int)s.v_rs) * 2u));
            }
        } else {                                         // rows past the end repeat the last one
#pragma unroll
            for (int i = 0; i < S::PIECES; ++i) {
                const int row = min(tg / C8 + i * (S::GT / C8), last);
                kreg[i] = *(const v4u *)(kt + (uint32_t)(row * (int)s.k_rs + tg % C8 * 8) * 2u);
                vreg[i] = *(const v4u *)(vt + (uint32_t)(row * (int)s.v_rs + tg % C8 * 8) * 2u);
            }
        }
    };
    auto buffer = [&](int b) { return (u16 *)smem + (size_t)(b * KG + kg) * 2 * TILE; };
    auto store = [&](u16 *dst) {
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i) {
            const int at = (tg / C8 + i * (S::GT / C8)) * ROW + tg % C8 * 8;
            *(v4u *)(dst + at) = kreg[i];
            *(v4u *)(dst + TILE + at) = vreg[i];
        }
    };

    int t = t0 + kg;
    if (t < t1) load(t);
    // Q^T operands, and what the lane's rows see of the keys from s.open on
    v4u qreg[NB][KS];
    int lim[NB];
    unsigned long long line[NB];
    unsigned long long mine = 0ull;
    if (TREE && t1 * TK > s.open) mine = tree_line(s.parent, s.nodes);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int row = min(r.row0 + (rg * NB + nb) * 16 + ln, r.rows - 1), at = row / r.G;
        if (TREE) {
            line[nb] = ((unsigned long long)(unsigned)__shfl((int)(mine >> 32), at) << 32) | (unsigned)__shfl((int)mine, at);
        } else {
            lim[nb] = s.shift + at;
        }
        const u16 *src = (const u16 *)r.q + (size_t)(row % r.G) * r.q_hs + (size_t)at * r.q_rs + 8 * lg;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qreg[nb][ks] = *(const v4u *)(src + ks * 32);
    }
    f32x4 o[NB][DB];
    float m[NB], l[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        m[nb] = -INFINITY;
        l[nb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[nb][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const float c = scale * kLog2e;

    auto compute = [&](const u16 *sk, int j0) {          // 32 keys; V lies one tile behind K
        const u16 *sv = sk + TILE;
        f32x4 x[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) x[nb][0] = x[nb][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const v4u a = *(const v4u *)(sk + (kb * 16 + ln) * ROW + 8 * lg + ks * 32);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) x[nb][kb] = mfma16(a, qreg[nb][ks], x[nb][kb]);
            }
        if (j0 + 31 >= s.open) {
            asm volatile("; mask path" ::: "memory");
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = j0 + (e >> 2) * 16 + 4 * lg + (e & 3), node = j - s.open;
                    const bool seen = TREE ? node < 0 || (node < 64 && ((line[nb] >> (node & 63)) & 1ull)) : j <= lim[nb];
                    if (!seen) x[nb][e >> 2][e & 3] = -INFINITY;
                }
        }
        // against the reference so far, and anew with the true maximum where a row outgrew it (or has none yet)
        v4u pb[NB];
        float rs[NB];
        bool big = false;
        auto probabilities = [&](int nb, float ref) {
            float pv[8];
            rs[nb] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                pv[e] = __builtin_amdgcn_exp2f(fmaf(x[nb][e >> 2][e & 3], c, -ref));
                rs[nb] += pv[e];
            }
            pb[nb] = (v4u){pack_bf16x2(pv[0], pv[1]), pack_bf16x2(pv[2], pv[3]), pack_bf16x2(pv[4], pv[5]),
                           pack_bf16x2(pv[6], pv[7])};
        };
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            probabilities(nb, m[nb] * c);
            big = big || !(rs[nb] < kBigSum);
        }
        if (__builtin_amdgcn_ballot_w64(big) != 0ull) {
            asm volatile("; rescale path" ::: "memory");
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float mx = -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; ++e) mx = fmaxf(mx, x[nb][e >> 2][e & 3]);
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m_new = fmaxf(m[nb], mx);
                const float ref = m_new == -INFINITY ? 0.f : m_new * c;     // -inf: the row sees no key yet
                const float alpha = __builtin_amdgcn_exp2f(fmaf(m[nb], c, -ref));
                m[nb] = m_new;
                l[nb] *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db) o[nb][db] *= alpha;
                probabilities(nb, ref);
            }
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) l[nb] += rs[nb];
        const u16 *vf = sv + (4 * lg + (ln >> 2)) * ROW + 4 * (ln & 3);      // see lds_read_tr16
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const v2u lo = lds_read_tr16(vf + 16 * db), hi = lds_read_tr16(vf + 16 * ROW + 16 * db);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) o[nb][db] = mfma16((v4u){lo.x, lo.y, hi.x, hi.y}, pb[nb], o[nb][db]);
        }
    };

    if constexpr (RG == 1) {
        for (; t < t1; t += KG) {
            store(buffer(0));
            const int j0 = t * TK;
            if (t + KG < t1) load(t + KG);
            compute(buffer(0), j0);
        }
    } else {
        // the groups' tiles in step: stage i of group kg is tile t0 + i KG + kg, in the buffer i % 2
        const int stages = (t1 - t0 + KG - 1) / KG;
        if (t < t1) store(buffer(0));
        if (t + KG < t1) load(t + KG);
        __syncthreads();
        for (int i = 0; i < stages; ++i, t += KG) {
            if (t < t1) {
#pragma unroll
                for (int sub = 0; sub < S::SUB; ++sub) {
                    const int j0 = t * TK + sub * 32;
                    if (sub == 0 || j0 < s.n) compute(buffer(i & 1) + sub * 32 * ROW, j0);
                }
            }
            if (t + KG < t1) store(buffer((i + 1) & 1));
            if (t + 2 * KG < t1) load(t + 2 * KG);
            __syncthreads();
        }
    }

    // the waves' sums: scaled to the common maximum, the upper half's handed to the lower half's, and those
    // added up on the way out
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        l[nb] += __shfl_xor(l[nb], 16);
        l[nb] += __shfl_xor(l[nb], 32);
        if (lg == 0) { sm[(wave * NB + nb) * 16 + ln] = m[nb]; sl[(wave * NB + nb) * 16 + ln] = l[nb]; }
    }
    __syncthreads();                                     // also: the last tiles have been read
    float *so = (float *)smem;
    auto place = [&](int slot, int nb) { return so + ((size_t)slot * S::R + (rg * NB + nb) * 16 + ln) * S::OROW + 4 * lg; };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        if constexpr (KG > 1) {
            float m_all = -INFINITY;
#pragma unroll
            for (int w = 0; w < KG; ++w) m_all = fmaxf(m_all, sm[((w * RG + rg) * NB + nb) * 16 + ln]);
            const float f = m[nb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[nb] - m_all) * c);
#pragma unroll
            for (int db = 0; db < DB; ++db) o[nb][db] *= f;
        }
        if (KG == 1 || kg >= KG / 2) {
#pragma unroll
            for (int db = 0; db < DB; ++db) *(f32x4 *)(place(KG == 1 ? 0 : kg - KG / 2, nb) + db * 16) = o[nb][db];
        }
    }
    __syncthreads();
    if constexpr (KG > 1) {
        if (kg < KG / 2) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int db = 0; db < DB; ++db) *(f32x4 *)(place(kg, nb) + db * 16) += o[nb][db];
        }
        __syncthreads();
    }
    const int rows_here = min(S::R, r.rows - r.row0);
    for (int i = threadIdx.x; i < rows_here * (D / 4); i += kSeqWaves * 64) {
        const int row = i / (D / 4), c4 = i % (D / 4) * 4, rr = row / (16 * NB), ri = row % (16 * NB);
        f32x4 y = *(const f32x4 *)(so + (size_t)row * S::OROW + c4);
#pragma unroll
        for (int w = 1; w < S::SL; ++w) y += *(const f32x4 *)(so + ((size_t)w * S::R + row) * S::OROW + c4);
        float m_row = -INFINITY, l_row = 0.f;
#pragma unroll
        for (int w = 0; w < KG; ++w) m_row = fmaxf(m_row, sm[(w * RG + rr) * 16 * NB + ri]);
#pragma unroll
        for (int w = 0; w < KG; ++w) {                   // multiplied, not left out: NaN logits alone leave -inf and a NaN sum
            const float mw = sm[(w * RG + rr) * 16 * NB + ri];
            l_row += sl[(w * RG + rr) * 16 * NB + ri] * (mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - m_row) * c));
        }
        if (pml) {
            *(f32x4 *)(po + (size_t)row * D + c4) = y;
            if (c4 == 0) pml[row] = make_float2(m_row * c, l_row);
            continue;
        }
        const int at = (r.row0 + row) / r.G, head = (r.row0 + row) % r.G;
        const float inv = l_row == 0.f ? 0.f : 1.0f / l_row;                // 0: the row sees no key
        v2u w;
        w.x = pack_bf16x2(y[0] * inv, y[1] * inv);
        w.y = pack_bf16x2(y[2] * inv, y[3] * inv);
        *(v2u *)((u16 *)r.out + (size_t)head * r.o_hs + (size_t)at * r.o_rs + c4) = w;
        if (c4 == 0 && r.lse) r.lse[(size_t)head * r.lse_hs + at] = (m_row * c + __builtin_amdgcn_logf(l_row)) * kLn2;
    }
}

}  // namespace reform
