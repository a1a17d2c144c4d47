// Attention of a block of query rows over a range of one sequence's keys, by one workgroup whose waves share
// out the keys (bf16: also the rows): the short prompts' form and the drafted tokens' share it.
//
// Rows are counted over a sequence's query rows and the G heads of a KV group together (row r is query row
// r / G of head r % G), so K and V are read once for all of them.  Softmax in one pass with a running
// reference maximum and sum; logits, sums and outputs in fp32.  In the bf16 form the probabilities of P.V are
// rounded to bf16, by up to 2^-8 of each, while their sum adds them unrounded: the matrix instruction takes bf16 on both
// sides, and a second product for what the rounding leaves would double P.V where the matrix pipe is the bound (prompts, wide
// trees).  The forms bound by memory could hide it; they do without it too, so that all forms compute alike, and as
// reform_chunk_attend_score does.  Outputs are off by 0.0017 to 0.0024 of their norm (up to 16640 keys), 0.0017 of it by
// their own rounding.
#pragma once
#include "attend_tile.h"

#include <type_traits>

namespace reform {

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

// Prompts with a sliding window: query row i, at key t = i + shift, sees j <= t with j > t - window or j < sinks.  A block goes through
// two runs of keys, the first ones and those that its rows' windows show, counted through: places below `cut` are the keys of these
// numbers, those from there on the keys `skip` further.  Tiles are cut from the places, so that few keys of them are not seen by any row:
// one tile may have keys of both runs, and only there rows are addressed one by one.
struct WindowKeys : SeqKeys {
    int window, cut, skip;   // skip = 0: cut = 0
    int stay;                // keys below it that lie in a tile are seen by all rows, unless they are behind the row's own
};

// Tile u of TK places: its first key (with keys of both runs: as if all were of the second), whether it has keys of both, and the key
// of a place.
template <int TK, class KEYS>
__device__ __forceinline__ int key_start(const KEYS &k, int u)
{
    if constexpr (std::is_same<KEYS, WindowKeys>::value) return u * TK + (u * TK + TK > k.cut ? k.skip : 0);
    else return u * TK;
}
template <int TK, class KEYS>
__device__ __forceinline__ bool key_split(const KEYS &k, int u)
{
    if constexpr (std::is_same<KEYS, WindowKeys>::value) return u * TK < k.cut && u * TK + TK > k.cut;
    else return false;
}
template <class KEYS>
__device__ __forceinline__ int key_of(const KEYS &k, int place)
{
    if constexpr (std::is_same<KEYS, WindowKeys>::value) return place + (place < k.cut ? 0 : k.skip);
    else return place;
}

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

// NW waves of 16 NB rows, all the same ones; each takes every NW-th tile of 32 keys, through LDS of its own, without a
// barrier before the sums meet.
template <int D, int NB, int NW>
struct SeqShape {
    static constexpr int R = 16 * NB, TK = 32;
    static constexpr int C8 = D / 8, ROW = D + 16, TILE = TK * ROW;
    static constexpr int PIECES = TK * C8 / 64;
    static constexpr int SL = NW / 2, OROW = D + 4;
    static constexpr size_t stage_bytes = sizeof(u16) * (size_t)NW * 2 * TILE;
    static constexpr size_t sum_bytes = sizeof(float) * (size_t)SL * R * OROW;
    static constexpr size_t base_bytes = (stage_bytes > sum_bytes ? stage_bytes : sum_bytes);
    static constexpr size_t line_at = base_bytes + sizeof(float) * 2 * NW * R;
    static constexpr size_t lds_bytes = line_at + sizeof(unsigned long long) * 64;
};

// Key tiles [t0, t1) of the sequence (may be empty).  po, pml: null for a final result, else this block's
// unnormalised sums [rows][D] and (reference maximum in log2 units, sum) [rows].
// On entry nothing in `smem` may be in use by any wave.
template <int D, int NB, int NW, bool TREE, class KEYS>
__device__ __forceinline__ void seq_segment(const SeqRows &r, const KEYS &s, float scale, int t0, int t1, float *po,
                                            float2 *pml, char *smem)
{
    using S = SeqShape<D, NB, NW>;
    constexpr bool WINDOW = std::is_same<KEYS, WindowKeys>::value;
    constexpr int KS = D / 32, DB = D / 16, C8 = S::C8, ROW = S::ROW, TILE = S::TILE, TK = S::TK;
    float *sm = (float *)(smem + S::base_bytes), *sl = sm + NW * S::R;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ln = lane & 15, lg = lane >> 4;

    // 16-byte pieces of a tile: piece i of a lane lies in row lane / C8 + i * (64 / C8)
    v4u kreg[S::PIECES], vreg[S::PIECES];
    const uint32_t koff = (uint32_t)((lane / C8) * (int)s.k_rs + lane % C8 * 8) * 2u;
    const uint32_t voff = (uint32_t)((lane / C8) * (int)s.v_rs + lane % C8 * 8) * 2u;
    auto load = [&](int u) {
        const int j0 = key_start<TK>(s, u);
        const char *kt = (const char *)((const u16 *)s.k + (size_t)j0 * s.k_rs);
        const char *vt = (const char *)((const u16 *)s.v + (size_t)j0 * s.v_rs);
        const int last = s.n - 1 - j0;
        if (key_split<TK>(s, u)) {
#pragma unroll
            for (int i = 0; i < S::PIECES; ++i) {
                const size_t row = min(key_of(s, u * TK + lane / C8 + i * (64 / C8)), s.n - 1);
                kreg[i] = *(const v4u *)((const u16 *)s.k + row * s.k_rs + lane % C8 * 8);
                vreg[i] = *(const v4u *)((const u16 *)s.v + row * s.v_rs + lane % C8 * 8);
            }
        } else if (last >= TK - 1) {
#pragma unroll
            for (int i = 0; i < S::PIECES; ++i) {
                kreg[i] = *(const v4u *)(kt + (koff + (uint32_t)(i * (64 / C8) * (int)s.k_rs) * 2u));
                vreg[i] = *(const v4u *)(vt + (voff + (uint32_t)(i * (64 / C8) * (int)s.v_rs) * 2u));
            }
        } else {                                         // rows past the end repeat the last one
#pragma unroll
            for (int i = 0; i < S::PIECES; ++i) {
                const int row = min(lane / C8 + i * (64 / C8), last);
                kreg[i] = *(const v4u *)(kt + (uint32_t)(row * (int)s.k_rs + lane % C8 * 8) * 2u);
                vreg[i] = *(const v4u *)(vt + (uint32_t)(row * (int)s.v_rs + lane % C8 * 8) * 2u);
            }
        }
    };
    u16 *const mine = (u16 *)smem + (size_t)wave * 2 * TILE;
    auto store = [&] {
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i) {
            const int at = (lane / C8 + i * (64 / C8)) * ROW + lane % C8 * 8;
            *(v4u *)(mine + at) = kreg[i];
            *(v4u *)(mine + TILE + at) = vreg[i];
        }
    };

    // Q^T operands
    v4u qreg[NB][KS];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int row = min(r.row0 + nb * 16 + ln, r.rows - 1), at = row / r.G;
        const u16 *src = (const u16 *)r.q + (size_t)(row % r.G) * r.q_hs + (size_t)at * r.q_rs + 8 * lg;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qreg[nb][ks] = *(const v4u *)(src + ks * 32);
    }
    int t = t0 + wave;
    if (t < t1) load(t);
    // what every node sees of the drafted keys: every wave writes all of it for itself (the same words)
    unsigned long long *lines = (unsigned long long *)(smem + S::line_at);
    if (TREE && t1 * TK > s.open) lines[lane] = tree_line(s.parent, s.nodes);
    // Q has to be there before the loop: a wait inside it would be one for the next tile's loads as well, in every trip
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qreg[nb][ks]));
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
    int behind = -1, stay = 0;                           // windows: some row does not see keys up to here; see WindowKeys
    int own[NB];                                         // and the key of the lane's own rows, less its first key of a tile
    if constexpr (WINDOW) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) own[nb] = s.shift + min(r.row0 + nb * 16 + ln, r.rows - 1) / r.G - 4 * lg;
        behind = __builtin_amdgcn_readlane(own[NB - 1], 15) - s.window;          // of the block's last row
        stay = s.stay;
    }

    for (; t < t1; t += NW) {
        store();
        const int j0 = key_start<TK>(s, t);
        if (t + NW < t1) load(t + NW);
        const u16 *sk = mine, *sv = mine + TILE;
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
        if constexpr (WINDOW) {
            // of the lane's keys 16 kb + e: seen up to its rows' own, and from behind their windows' ends or below the first keys'
            if (j0 + 31 >= s.open) {
                asm volatile("; mask path" ::: "memory");
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if ((e >> 2) * 16 + (e & 3) > own[nb] - j0) x[nb][e >> 2][e & 3] = -INFINITY;
            }
            if (j0 <= behind && j0 + TK > stay) {
                asm volatile("; mask path" ::: "memory");
                const int front = stay - j0 - 4 * lg;
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int key = (e >> 2) * 16 + (e & 3);
                        if (key <= own[nb] - j0 - s.window && key >= front) x[nb][e >> 2][e & 3] = -INFINITY;
                    }
            }
        } else if (j0 + 31 >= s.open) {
            asm volatile("; mask path" ::: "memory");
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                // formed here, from values that the compiler cannot relate to the other uses: kept, they cost registers in the loop
                int G = r.G, x0 = lane;
                asm volatile("" : "+s"(G), "+v"(x0));
                const int at = min(r.row0 + nb * 16 + (x0 & 15), r.rows - 1) / G, first = 4 * (x0 >> 4);
                unsigned seen;                           // of the tile's keys 4 lg + e (bit e) and 16 + 4 lg + e (bit 16 + e)
                if (TREE) {
                    const int node = j0 - s.open;        // what the tile's first key is
                    const unsigned long long line = lines[at];
                    if (node >= 0) seen = node < 64 ? (unsigned)(line >> node) : 0u;
                    else seen = (unsigned)(line << -node) | ((1u << -node) - 1u);        // -31 <= node
                    seen >>= first;
                } else {
                    const int more = s.shift + at - j0 - first;    // keys behind the lane's first that are seen
                    seen = more >= 31 ? ~0u : more < 0 ? 0u : (2u << more) - 1u;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!((seen >> ((e >> 2) * 16 + (e & 3))) & 1u)) x[nb][e >> 2][e & 3] = -INFINITY;
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
    }

    // the waves' sums: scaled to the common maximum, the upper half's handed to the lower half's, and those
    // added up on the way out
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        l[nb] += __shfl_xor(l[nb], 16);
        l[nb] += __shfl_xor(l[nb], 32);
        if (lg == 0) { sm[wave * S::R + nb * 16 + ln] = m[nb]; sl[wave * S::R + nb * 16 + ln] = l[nb]; }
    }
    __syncthreads();                                     // also: the last tiles have been read
    float *so = (float *)smem;
    auto place = [&](int slot, int nb) { return so + (slot * S::R + nb * 16 + ln) * S::OROW + 4 * lg; };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        float m_all = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, sm[w * S::R + nb * 16 + ln]);
        const float f = m[nb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[nb] - m_all) * c);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            o[nb][db] *= f;
            if (wave >= NW / 2) *(f32x4 *)(place(wave - NW / 2, nb) + db * 16) = o[nb][db];
        }
    }
    __syncthreads();
    if (wave < NW / 2) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int db = 0; db < DB; ++db) *(f32x4 *)(place(wave, nb) + db * 16) += o[nb][db];
    }
    __syncthreads();
    const int rows_here = min(S::R, r.rows - r.row0);
    for (int i = threadIdx.x; i < rows_here * (D / 4); i += NW * 64) {
        const int row = i / (D / 4), c4 = i % (D / 4) * 4;
        f32x4 y = *(const f32x4 *)(so + row * S::OROW + c4);
#pragma unroll
        for (int w = 1; w < S::SL; ++w) y += *(const f32x4 *)(so + (w * S::R + row) * S::OROW + c4);
        float m_row = -INFINITY, l_row = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) m_row = fmaxf(m_row, sm[w * S::R + row]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {                   // multiplied, not left out: NaN logits alone leave -inf and a NaN sum
            const float mw = sm[w * S::R + row];
            l_row += sl[w * S::R + row] * (mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - m_row) * c));
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
