// One new token of each sequence over caches in pages, bf16 (see reform_paged_attend in reform.h).
//
// Bound: reading K and V once.  The rows of a block are up to 16 heads of a KV group; the keys are shared out over the whole chip
// (paged_list.h), and every wave has tiles of 32 keys of its own, without a barrier before the sums meet: S^T = K Q^T, so that a
// lane owns one head's logits, which are the B operand of O^T = V^T P^T as they stand, as in attend_seq.h.  The matrix pipe waits for
// memory, so P.V is done twice, with the probabilities rounded to bf16 and with what that leaves of them: together 16 bits, and
// outputs are off by their own rounding (0.0017 of their norm; 0.0023 with one product).
//
// What pages add: a tile's rows lie anywhere.  Where page_len is a multiple of 16 (HALVES), each half of a tile lies in one page:
// lane l looks up half l % 2 of the wave's tile l / 2, 32 tiles in one go, and a tile's two bases are read from the lanes into scalar
// registers, so that its loads cost what they do in one piece of memory.  Else every key's row is looked up by a lane of its own, a
// tile ahead, and handed to the lanes that load it.
#include "paged_list.h"

namespace reform {

namespace {

template <int D, int NW>
struct PagedShape {
    static constexpr int R = 16, TK = 32;
    static constexpr int C8 = D / 8, ROW = D + 16, TILE = TK * ROW;      // as SeqShape
    static constexpr int PIECES = TK * C8 / 64;
    static constexpr int SL = NW / 2, OROW = D + 4;
    static constexpr size_t stage_bytes = sizeof(u16) * (size_t)NW * 2 * TILE;
    static constexpr size_t sum_bytes = sizeof(float) * (size_t)SL * R * OROW;
    static constexpr size_t base_bytes = stage_bytes > sum_bytes ? stage_bytes : sum_bytes;
    static constexpr size_t row_at = base_bytes + sizeof(float) * 2 * NW * R;
    static constexpr size_t lds_bytes = row_at + sizeof(float2) * R;
};

__device__ __forceinline__ long lane_value(long x, int lane)
{
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned long)x, lane);
    const unsigned hi = (unsigned)__builtin_amdgcn_readlane((int)((unsigned long)x >> 32), lane);
    return (long)(((unsigned long)hi << 32) | lo);
}

// K and V that are read once go past the caches' usual order of replacement (paged_plan).
template <bool STREAM>
__device__ __forceinline__ v4u load16(const void *p)
{
    return STREAM ? __builtin_nontemporal_load((const v4u *)p) : *(const v4u *)p;
}

// Virtual tiles [t0, t1) of sequence b's KV head for the heads from row0 on.  po, pml: as in seq_segment.
template <int D, int NW, bool HALVES, bool STREAM>
__device__ __forceinline__ void paged_segment(const PagedParams &p, int b, int kvh, int len, int row0, int t0, int t1, float *po, float2 *pml, char *smem)
{
    using S = PagedShape<D, NW>;
    constexpr int KS = D / 32, DB = D / 16, C8 = S::C8, ROW = S::ROW, TILE = S::TILE, TK = S::TK, STEP = 64 / C8;
    float *sm = (float *)(smem + S::base_bytes), *sl = sm + NW * S::R;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ln = lane & 15, lg = lane >> 4;
    const PagedSpan<TK> span(p, len);
    const u16 *const K = (const u16 *)p.k + (size_t)kvh * p.pool.head_stride, *const V = (const u16 *)p.v + (size_t)kvh * p.pool.head_stride;
    const int32_t *table = p.pool.table + (size_t)b * p.pool.table_stride;
    const int rows = p.G - row0;                         // heads from row0 on

    // Where key j's row is, -1 where it is not seen.
    auto place = [&](int j) { return span.seen(j) ? pool_row(p.pool, table, j) : -1l; };
    long ahead = -1l;                                    // HALVES: of half lane % 2 of tile `from` + NW (lane / 2); else of key lane % 32
    int from = 0;
    auto look = [&](int u) {
        if (HALVES) {
            // a half is there if its page is, and has a seen key; which ones are seen is told by their numbers
            const int v = u + NW * (lane >> 1), j = span.tile(v) * TK + 16 * (lane & 1);
            ahead = v < t1 && j < span.n ? pool_row(p.pool, table, j) : -1l;
            from = u;
        } else {
            ahead = u < t1 ? place(span.tile(u) * TK + (lane & 31)) : -1l;
        }
    };
    // 16-byte pieces of a tile: piece i of a lane lies in row lane / C8 + i * STEP
    v4u kreg[S::PIECES], vreg[S::PIECES];
    unsigned mask = 0u;                                  // keys of the loaded tile that are seen
    const uint32_t lane_off = (uint32_t)((lane / C8) * (int)p.pool.row_stride + lane % C8 * 8) * 2u;
    auto load = [&](int u) {
        const int j0 = span.tile(u) * TK;
        if (HALVES) {
            if (u - from >= 32 * NW) look(u);
            const int at = (u - from) / NW * 2;
            const long a = lane_value(ahead, at), b1 = lane_value(ahead, at + 1);
            const int j = j0 + (lane & 31);
            mask = (unsigned)__builtin_amdgcn_ballot_w64(span.seen(j) && ((lane & 16) ? b1 : a) >= 0);
            if (mask == ~0u) {
#pragma unroll
                for (int i = 0; i < S::PIECES; ++i) {
                    const long half = i < S::PIECES / 2 ? a : b1;
                    const uint32_t off = lane_off + (uint32_t)((i % (S::PIECES / 2)) * STEP * (int)p.pool.row_stride) * 2u;
                    kreg[i] = load16<STREAM>((const char *)(K + half) + off);
                    vreg[i] = load16<STREAM>((const char *)(V + half) + off);
                }
            } else {
#pragma unroll
                for (int i = 0; i < S::PIECES; ++i) {
                    const long half = i < S::PIECES / 2 ? a : b1;
                    const uint32_t off = lane_off + (uint32_t)((i % (S::PIECES / 2)) * STEP * (int)p.pool.row_stride) * 2u;
                    kreg[i] = vreg[i] = (v4u){0u, 0u, 0u, 0u};           // weights of 0 meet zeros, whatever lies there
                    if ((mask >> (lane / C8 + i * STEP)) & 1u) {
                        kreg[i] = load16<STREAM>((const char *)(K + half) + off);
                        vreg[i] = load16<STREAM>((const char *)(V + half) + off);
                    }
                }
            }
        } else {
            mask = (unsigned)__builtin_amdgcn_ballot_w64(ahead >= 0);
#pragma unroll
            for (int i = 0; i < S::PIECES; ++i) {
                const int row = lane / C8 + i * STEP;
                const long at = ((long)__shfl((int)(ahead >> 32), row) << 32) | (unsigned)__shfl((int)ahead, row);
                kreg[i] = vreg[i] = (v4u){0u, 0u, 0u, 0u};
                if (at >= 0) {
                    kreg[i] = load16<STREAM>(K + at + lane % C8 * 8);
                    vreg[i] = load16<STREAM>(V + at + lane % C8 * 8);
                }
            }
            look(u + NW);
        }
    };
    u16 *const mine = (u16 *)smem + (size_t)wave * 2 * TILE;
    auto store = [&] {
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i) {
            const int at = (lane / C8 + i * STEP) * ROW + lane % C8 * 8;
            *(v4u *)(mine + at) = kreg[i];
            *(v4u *)(mine + TILE + at) = vreg[i];
        }
    };

    v4u qreg[KS];                                        // Q^T operand; columns behind the last head repeat it
    {
        const u16 *src = (const u16 *)p.q + (size_t)b * p.q_ss + (size_t)(kvh * p.G + row0 + min(ln, rows - 1)) * p.q_hs + 8 * lg;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qreg[ks] = *(const v4u *)(src + ks * 32);
    }
    int u = t0 + wave;
    look(u);
    if (u < t1) load(u);
    // Q has to be there before the loop: a wait inside it would be one for the next tile's loads as well, in every trip
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qreg[ks]));
    f32x4 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const float c = p.scale * kLog2e;
    float *const logits = p.logits && ln < rows ? p.logits + ((size_t)b * p.Hq + (size_t)kvh * p.G + row0 + ln) * p.logit_keys + 4 * lg : nullptr;

    for (; u < t1; u += NW) {
        store();
        const unsigned seen = mask;
        if (u + NW < t1) load(u + NW);
        const u16 *sk = mine, *sv = mine + TILE;
        f32x4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) x[kb] = mfma16(*(const v4u *)(sk + (kb * 16 + ln) * ROW + 8 * lg + ks * 32), qreg[ks], x[kb]);
        if (seen != ~0u) {
            const unsigned mine_seen = seen >> (4 * lg);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!((mine_seen >> ((e >> 2) * 16 + (e & 3))) & 1u)) x[e >> 2][e & 3] = -INFINITY;
        }
        if (logits) {
            *(f32x4 *)(logits + (size_t)u * TK) = x[0];
            *(f32x4 *)(logits + (size_t)u * TK + 16) = x[1];
        }
        // against the reference so far, and anew with the true maximum where a row outgrew it (or has none yet)
        v4u pb, pl;                                      // rounded to bf16, and what that leaves, rounded
        float rs;
        auto probabilities = [&](float ref) {
            float pv[8];
            rs = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                pv[e] = __builtin_amdgcn_exp2f(fmaf(x[e >> 2][e & 3], c, -ref));
                rs += pv[e];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                pb[i] = pack_bf16x2(pv[2 * i], pv[2 * i + 1]);
                pl[i] = pack_bf16x2(pv[2 * i] - __uint_as_float(pb[i] << 16), pv[2 * i + 1] - __uint_as_float(pb[i] & 0xffff0000u));
            }
        };
        probabilities(m * c);
        if (__builtin_amdgcn_ballot_w64(!(rs < kBigSum)) != 0ull) {
            asm volatile("; rescale path" ::: "memory");
            float mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, x[e >> 2][e & 3]);
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new * c;    // -inf: no key yet
            const float alpha = __builtin_amdgcn_exp2f(fmaf(m, c, -ref));
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db] *= alpha;
            probabilities(ref);
        }
        l += rs;
        const u16 *vf = sv + (4 * lg + (ln >> 2)) * ROW + 4 * (ln & 3);          // see lds_read_tr16
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const v2u lo = lds_read_tr16(vf + 16 * db), hi = lds_read_tr16(vf + 16 * ROW + 16 * db);
            o[db] = mfma16((v4u){lo.x, lo.y, hi.x, hi.y}, pb, o[db]);
            o[db] = mfma16((v4u){lo.x, lo.y, hi.x, hi.y}, pl, o[db]);
        }
    }

    // the waves' sums, as in seq_segment
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (lg == 0) { sm[wave * S::R + ln] = m; sl[wave * S::R + ln] = l; }
    __syncthreads();
    float *so = (float *)smem;
    auto spot = [&](int slot) { return so + (slot * S::R + ln) * S::OROW + 4 * lg; };
    float m_all = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) m_all = fmaxf(m_all, sm[w * S::R + ln]);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - m_all) * c);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        o[db] *= f;
        if (wave >= NW / 2) *(f32x4 *)(spot(wave - NW / 2) + db * 16) = o[db];
    }
    __syncthreads();
    if (wave < NW / 2) {
#pragma unroll
        for (int db = 0; db < DB; ++db) *(f32x4 *)(spot(wave) + db * 16) += o[db];
    }
    __syncthreads();
    float2 *const row_ml = (float2 *)(smem + S::row_at);
    for (int i = threadIdx.x; i < min(S::R, rows) * (D / 4); i += NW * 64) {
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
        const int head = kvh * p.G + row0 + row;
        const float inv = l_row == 0.f ? 0.f : 1.0f / l_row;                     // 0: the row sees no key
        *(v2u *)((u16 *)p.out + (size_t)b * p.o_ss + (size_t)head * p.o_hs + c4) =
            (v2u){pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv)};
        if (c4 == 0) {
            if (p.lse) p.lse[(size_t)b * p.Hq + head] = (m_row * c + __builtin_amdgcn_logf(l_row)) * kLn2;
            if (paged_scores_alone(p)) row_ml[row] = score_row(m_row * c, l_row);
            else if (p.row_ml) p.row_ml[(size_t)b * p.Hq + head] = make_float2(m_row * c, l_row);
        }
    }
    if (paged_scores_alone(p)) {
        __syncthreads();                                 // rows and logits are there
        int counter = 0;
        paged_score<TK>(p, b, kvh, len, t0, t1, counter, wave, NW, [&](int) { return row_ml[min(lane, rows - 1)]; });
    }
}

template <int D, int NW, bool HALVES, bool STREAM>
__global__ __launch_bounds__(NW * 64, 2) void paged_attend(PagedParams p)
{
    using S = PagedShape<D, NW>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    list_walk<S::R, S::TK>(p, [&](int b, const TreeSeq &seq, int kvh, int rb, int t0, int t1, long slot) {
        paged_segment<D, NW, HALVES, STREAM>(p, b, kvh, seq.len, rb * S::R, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * D,
                                     slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, smem);
    });
}

template <int D, int NW, bool HALVES, bool STREAM>
hipError_t launch(const PagedParams &p, hipStream_t st)
{
    using S = PagedShape<D, NW>;
    const hipError_t e = raise_lds<paged_attend<D, NW, HALVES, STREAM>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    const unsigned grid = (unsigned)(p.shares ? p.shares : p.n_seq * p.Hkv) * p.row_blocks;
    hipLaunchKernelGGL((paged_attend<D, NW, HALVES, STREAM>), dim3(grid), dim3(NW * 64), S::lds_bytes, st, p);
    paged_join_launch<D, S::R, S::TK, true>(p, st);
    return hipGetLastError();
}

}  // namespace

// Keys that a workgroup takes whole: fitted to 88 batches of 1 to 48 caches of 150 to 6000 keys, half of them with scores, each whole and
// shared out: 1.004 times the better of the two in the mean, at worst 1.10 (2000 and 1600 keys 1.02, 1.34).  As many
// shares as run at once, of 128 keys at least (heads of 64, 256 / 128, us: 1 cache of 1258 keys, 28/4 heads, 10.8 / 10.0; 4 of 1221, 16/2, 11.2 / 10.1; 4 with
// windows of 5761, 16/2, 12.7 / 13.4; heads of 128: 2 with windows of 2204, 16/4, 13.4 / 12.2).
void paged_plan_bf16(PagedParams &p)
{
    paged_plan(p, 16, 32, 1000, 128 / 32, (p.D == 64 ? 2 : 1) * p.units);
}

namespace {

template <int D, int NW>
hipError_t launch_form(const PagedParams &p, hipStream_t st)
{
    if (p.pool.page_len % 16) return p.stream ? launch<D, NW, false, true>(p, st) : launch<D, NW, false, false>(p, st);
    return p.stream ? launch<D, NW, true, true>(p, st) : launch<D, NW, true, false>(p, st);
}

}  // namespace

hipError_t paged_attend_bf16(const PagedParams &p, hipStream_t st)
{
    return p.D == 64 ? launch_form<64, 4>(p, st) : launch_form<128, 8>(p, st);
}

}  // namespace reform
