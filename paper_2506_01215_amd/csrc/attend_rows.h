// Attention of a block of many query rows over a range of one sequence's keys: every wave has 32 rows of its own, and
// all go through the same key tiles of 64 keys together (attend_seq.h has the form for few rows).
//
// It computes S^T = K Q^T with v_mfma_f32_16x16x32_bf16 (operand layouts in attend_bf16.hip), so that a
// lane owns one query column of each of its wave's two 16-row blocks, its softmax statistics are scalars, and the
// probabilities are the B operand of O^T = V^T P^T as they stand.  K and V tiles of 64 keys go from memory
// straight into LDS (global_load_lds, 16 bytes a lane), one tile ahead of the one that is computed (two ahead: no faster where
// it was tried, with one group of eight waves: 52 batches of prompts and of 20 to 64 nodes, geometric mean 69.7 us against
// 69.4; not tried with two groups of two waves).
//
// Addresses, strides and the list's state take more than the scalar registers there are: the compiler keeps 78 to 148 of them in
// lanes of vector registers in the shared-out forms (8 to 32 in prompt_attend) and reads some back in every tile.
//
// LDS: the 64 lanes of such a load land in 1024 adjacent bytes, so rows cannot be padded one by one.  Instead a load
// takes rows that no read takes together: rows c, c + 16, c + 32, c + 48 at head_dim 128 (at 64 rows c and c + 8 of
// every 16), and the loads' places ("chunks") lie 1024 + 32 bytes apart.  K's fragments (16 rows x 32 bytes per half
// wave, free of conflicts where they differ modulo 512 bytes) and V's transposing reads (8 rows x 32 bytes, modulo 256)
// then find their rows 32 bytes apart, and every fragment of a tile is at a constant distance from the lane's first.
#pragma once
#include "attend_seq.h"

#include <type_traits>

namespace reform {

constexpr int kRowsKeys = 64;

// KG groups of NW waves each: the groups have the same rows and take every KG-th tile.  THIN: 16 rows instead of 32 for the upper half
// of eight waves.
template <int D, int NW, int KG, bool THIN = false>
struct RowsShape {
    static_assert(!THIN || NW == 8, "two waves to a SIMD");
    static constexpr int ROWS = THIN ? 192 : NW * 32, BN = kRowsKeys, C8 = D / 8;
    static constexpr int CHUNKS = BN * D / 512, PITCH = 512 + 16, TILE = CHUNKS * PITCH;      // elements
    static constexpr int LOADS = CHUNKS / NW;            // of a wave, for K and for V
    static constexpr bool LAG = NW == 8;                 // the upper half of the waves runs P.V one tile late
    static_assert(!LAG || KG == 1, "two waves to a SIMD");
    static constexpr int KSLOTS = 2, VSLOTS = 2 + LAG;   // tiles of K and V in LDS
    static constexpr int GROUP = (KSLOTS + VSLOTS) * TILE;                   // of one group of waves
    static constexpr int OROW = D + 4;                   // floats of a row of the groups' sums
    static constexpr size_t line_at = sizeof(u16) * (size_t)KG * GROUP;      // bytes
    static_assert(sizeof(float) * (size_t)(KG - 1) * ROWS * (OROW + 2) <= line_at, "the groups' sums replace their tiles");
    static constexpr size_t lds_bytes = line_at + sizeof(unsigned long long) * 64;
    static constexpr int KS = D / 32, DB = D / 16, NK = 4 * KS, NV = 2 * DB;
    // offset inside a tile of row 16 kb + x, x < 16: part that depends on x, part that depends on kb
    __device__ static __forceinline__ int row_at(int x) { return D == 128 ? x * PITCH : (x & 7) * PITCH + (x >> 3) * 128; }
    __device__ static constexpr int block_at(int kb) { return D == 128 ? kb * 128 : (kb & 1) * 64 + (kb >> 1) * 256; }
    // row that lane l fetches for chunk c: c + this
    __device__ static __forceinline__ int lane_row(int l)
    {
        const int i = l / C8;
        return D == 128 ? 16 * i : 16 * ((i & 1) + 2 * (i >> 2)) + 8 * ((i >> 1) & 1);
    }
};

__device__ __forceinline__ void load_to_lds(const char *from, u16 *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// What a wave carries over the key tiles.
template <int D>
struct RowsWave {
    static constexpr int KS = D / 32, DB = D / 16;
    v4u q[2][KS];
    f32x4 o[2][DB];
    float m[2], l[2];
    v4u pb[2][2];            // probabilities of a tile
    int kat, vat;            // the lane's first fragment inside a K and a V tile (elements)
};

// What a wave does while a tile's successor is on its way: nothing (it needs no more keys), Q.K^T and softmax of
// the tile, P.V of the tile (in step) or of the one before (lagging waves), in this order.
enum RowsStep { kRowsIdle, kRowsAll, kRowsFirst, kRowsLag, kRowsLast };

// The pointers are to different tiles of the LDS; `next_*` are the ones that the loads under way fill.  That
// they are different is what lets the compiler read the others without waiting for these loads.
template <int D, int NW, int KG, int STEP, int NB, class MASK>
__device__ __forceinline__ void rows_tile(RowsWave<D> &w, const u16 *__restrict__ tk, const u16 *__restrict__ tv,
                                            u16 *__restrict__ next_k, u16 *__restrict__ next_v, const char *from_k, const char *from_v,
                                            size_t step_k, size_t step_v, bool loads, float c, MASK mask_tile)
{
    using S = RowsShape<D, NW, KG>;
    constexpr int DB = S::DB, NK = S::NK, NV = S::NV, kWin = 4;
    if (loads) {
#pragma unroll
        for (int i = 0; i < S::LOADS; ++i) {
            load_to_lds(from_k + i * step_k, next_k + i * NW * S::PITCH);
            load_to_lds(from_v + i * step_v, next_v + i * NW * S::PITCH);
        }
    }
    const u16 *ak = tk + w.kat, *av = tv + w.vat;
    auto kfrag = [&](int i) -> v4u { return *(const v4u *)(ak + S::block_at(i & 3) + (i >> 2) * 32); };    // i = 4 ks + kb
    auto vfrag = [&](int i) -> v4u {                     // i = DB kp + db
        const int kp = i / DB, db = i % DB;
        const v2u lo = lds_read_tr16(av + S::block_at(2 * kp) + 16 * db), hi = lds_read_tr16(av + S::block_at(2 * kp + 1) + 16 * db);
        return (v4u){lo.x, lo.y, hi.x, hi.y};
    };
    // fragments stream through a window of kWin register quads, each feeding the MFMAs of both row blocks; it is
    // refilled with the first fragments of the product that comes next while the last MFMAs of the one before run
    v4u fw[kWin];
    if constexpr (STEP == kRowsLag || STEP == kRowsLast) {
#pragma unroll
        for (int i = 0; i < kWin; ++i) fw[i] = vfrag(i);
#pragma unroll
        for (int f = 0; f < NV; ++f) {
            w.o[0][f % DB] = mfma16(fw[f % kWin], w.pb[0][f / DB], w.o[0][f % DB]);
            if (NB == 2) w.o[1][f % DB] = mfma16(fw[f % kWin], w.pb[1][f / DB], w.o[1][f % DB]);
            const int g = f + kWin;
            if (g < NV) fw[f % kWin] = vfrag(g);
            else if (STEP == kRowsLag) fw[f % kWin] = kfrag(g - NV);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * kWin, 0);
#pragma unroll
        for (int f = 0; f < NV - kWin; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, NB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);               // a V^T fragment is two reads
        }
#pragma unroll
        for (int f = NV - kWin; f < NV; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, NB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, STEP == kRowsLag ? 1 : 0, 0);
        }
    }
    if constexpr (STEP == kRowsAll || STEP == kRowsFirst || STEP == kRowsLag) {
        if (STEP != kRowsLag) {
#pragma unroll
            for (int i = 0; i < kWin; ++i) fw[i] = kfrag(i);
        }
        f32x4 s[NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) s[nb][kb] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < NK; ++f) {
            s[0][f & 3] = mfma16(fw[f % kWin], w.q[0][f >> 2], s[0][f & 3]);
            if (NB == 2) s[1][f & 3] = mfma16(fw[f % kWin], w.q[1][f >> 2], s[1][f & 3]);
            const int g = f + kWin;
            if (g < NK) fw[f % kWin] = kfrag(g);
            else if (STEP == kRowsAll) fw[f % kWin] = vfrag(g - NK);
        }
        if (STEP != kRowsLag) __builtin_amdgcn_sched_group_barrier(0x100, kWin, 0);
#pragma unroll
        for (int f = 0; f < NK - kWin; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, NB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
#pragma unroll
        for (int f = NK - kWin; f < NK; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, NB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, STEP == kRowsAll ? 2 : 0, 0);
        }
        mask_tile(s);
        float rs[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) rs[nb] = softmax_row(s[nb], c, w.m[nb] * c, w.pb[nb]);
        if (__builtin_amdgcn_ballot_w64(!(rs[0] < kBigSum) || !(rs[NB - 1] < kBigSum)) != 0ull) {
            asm volatile("; rescale path" ::: "memory");
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float mx = s[nb][0][0];
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[nb][kb][e]);
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m_new = fmaxf(w.m[nb], mx);
                const float ref = m_new == -INFINITY ? 0.f : m_new * c;     // -inf: the row sees no key yet
                const float alpha = __builtin_amdgcn_exp2f(fmaf(w.m[nb], c, -ref));
                w.m[nb] = m_new;
                w.l[nb] *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int e = 0; e < 4; ++e) w.o[nb][db][e] *= alpha;
                rs[nb] = softmax_row(s[nb], c, ref, w.pb[nb]);
            }
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) w.l[nb] += rs[nb];
    }
    if constexpr (STEP == kRowsAll) {
#pragma unroll
        for (int f = 0; f < NV; ++f) {
            w.o[0][f % DB] = mfma16(fw[f % kWin], w.pb[0][f / DB], w.o[0][f % DB]);
            if (NB == 2) w.o[1][f % DB] = mfma16(fw[f % kWin], w.pb[1][f / DB], w.o[1][f % DB]);
            if (f + kWin < NV) fw[f % kWin] = vfrag(f + kWin);
        }
#pragma unroll
        for (int f = 0; f < NV - kWin; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, NB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
    }
}

// Key tiles [t0, t1) of the sequence for the block of ROWS rows from r.row0 on, as seq_segment.  by_head: how the rows are dealt to
// the waves.
template <int D, int NW, int KG, bool TREE, bool THIN = false>
__device__ __forceinline__ void rows_segment(const SeqRows &r, SeqKeys k, bool by_head, float scale, int t0, int t1, float *po,
                                             float2 *pml, u16 *lds)
{
    using S = RowsShape<D, NW, KG, THIN>;
    constexpr int BN = S::BN, TILE = S::TILE, KS = S::KS, DB = S::DB, C8 = S::C8;
    // keys are counted from the range's first one
    k.k = (const u16 *)k.k + (size_t)t0 * BN * k.k_rs;
    k.v = (const u16 *)k.v + (size_t)t0 * BN * k.v_rs;
    k.n -= t0 * BN;
    k.open -= t0 * BN;
    k.shift -= t0 * BN;

    const int lane = threadIdx.x & 63, wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ln = lane & 15, lg = lane >> 4, kg = wave_all / NW, wave = wave_all % NW;
    u16 *ldsK = lds + kg * S::GROUP, *ldsV = ldsK + S::KSLOTS * TILE;        // [KSLOTS][TILE], [VSLOTS][TILE]
    // the wave's 32 rows: by_head (G divides the waves): consecutive query rows of one head, else consecutive rows
    const int slab = by_head ? wave / r.G : wave, rstep = by_head ? r.G : 1;
    const bool thin = THIN && wave >= NW / 2;            // then the second 16 rows do not exist, and nothing of theirs is computed or stored
    const int row0 = r.row0 + (thin ? 128 + (wave - NW / 2) * 16 : slab * 32 * rstep + (by_head ? wave % r.G : 0));
    // formed where needed, from values that the compiler cannot relate to the other uses: kept, they cost registers in the loop
    auto locate = [&](int nb, int &at, int &head) {
        int G = r.G, l = lane;
        asm volatile("" : "+s"(G), "+v"(l));
        const int x = min(row0 + rstep * (16 * nb + (l & 15)), r.rows - 1);
        at = x / G;
        head = x - at * G;
    };
    RowsWave<D> w;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
        int at, head;
        locate(nb, at, head);
        const u16 *src = (const u16 *)r.q + (size_t)head * r.q_hs + (size_t)at * r.q_rs + 8 * lg;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) w.q[nb][ks] = *(const v4u *)(src + ks * 32);
        w.m[nb] = -INFINITY;
        w.l[nb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) w.o[nb][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    w.kat = S::row_at(ln) + 8 * lg;
    w.vat = S::row_at(4 * lg + (ln >> 2)) + 4 * (ln & 3);        // see lds_read_tr16
    const float c = scale * kLog2e;
    const int ntiles = t1 - t0, M = k.shift;
    // tile t of the group is tile KG t + kg of the range; all groups go through as many steps
    const int steps = (ntiles + KG - 1) / KG;
    int tl = -1;                                         // last tile of the group that the wave needs
    if (row0 < r.rows) {
        const int last = TREE ? k.n - 1 : M + min(row0 + 31 * rstep, r.rows - 1) / r.G;       // prompts have no thin waves
        if (last >= kg * BN && kg < ntiles) tl = (min(last / BN, ntiles - 1) - kg) / KG;       // a range may have fewer tiles than groups
    }
    const int open = TREE ? k.open : M + row0 / r.G + 1; // keys below it are seen by all of the wave's rows
    unsigned long long *lines = (unsigned long long *)((char *)lds + S::line_at);
    if (TREE && ntiles * BN > k.open) lines[lane] = tree_line(k.parent, k.nodes);      // every wave the same words

    // this lane's 16 bytes of the wave's first load, and how far apart its loads are
    const int lr = wave + S::lane_row(lane);
    const uint32_t koff = (uint32_t)(lr * (int)k.k_rs + lane % C8 * 8) * 2u, voff = (uint32_t)(lr * (int)k.v_rs + lane % C8 * 8) * 2u;
    const size_t step_k = (size_t)NW * k.k_rs * 2, step_v = (size_t)NW * k.v_rs * 2;
    const bool lag = S::LAG && wave >= NW / 2;
    u16 *const wk = ldsK + wave * S::PITCH, *const wv = ldsV + wave * S::PITCH;        // where it lands in a tile
    // a tile that ends behind the last key: rows past it repeat the last one (they are masked)
    auto load_end = [&](int t, u16 *to_k, u16 *to_v) {
        int l = lane;
        asm volatile("" : "+v"(l));                      // as in locate
#pragma unroll
        for (int i = 0; i < S::LOADS; ++i) {
            const int row = min((t * KG + kg) * BN + wave + S::lane_row(l) + i * NW, k.n - 1);
            load_to_lds((const char *)((const u16 *)k.k + (size_t)row * k.k_rs + l % C8 * 8), to_k + i * NW * S::PITCH);
            load_to_lds((const char *)((const u16 *)k.v + (size_t)row * k.v_rs + l % C8 * 8), to_v + i * NW * S::PITCH);
        }
    };
    if (kg < ntiles) load_end(0, wk, wv);
    // Q has to be there before the loops: a wait inside them would be one for the next tile's loads as well
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(w.q[nb][ks]));
    int t = 0, kslot = 0, vslot = 0;                     // the slots of tile t: t mod KSLOTS, t mod VSLOTS
    auto mask_tile = [&](auto &s) {
        constexpr int NB = sizeof(s) / sizeof(s[0]);
        const int j0 = (t * KG + kg) * BN;
        if (j0 + BN > open) {
            asm volatile("; mask path" ::: "memory");
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                int at, head;
                locate(nb, at, head);
                int l = lane;
                asm volatile("" : "+v"(l));
                unsigned long long seen;                 // of the tile's keys 4 lg + 16 kb + e: bit 16 kb + e
                if (TREE) {
                    const int node = j0 - open;          // what the tile's first key is
                    const unsigned long long line = lines[at];
                    if (node >= 0) seen = node < 64 ? line >> node : 0ull;
                    else seen = (line << -node) | ((1ull << -node) - 1ull);              // -63 <= node
                    seen >>= 4 * (l >> 4);
                } else {
                    const int more = M + at - j0 - 4 * (l >> 4);         // keys behind the lane's first that are seen
                    seen = more >= 63 ? ~0ull : more < 0 ? 0ull : (2ull << more) - 1ull;
                }
                const unsigned half[2] = {(unsigned)seen, (unsigned)(seen >> 32)};
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!((half[kb >> 1] >> ((kb & 1) * 16 + e)) & 1u)) s[nb][kb][e] = -INFINITY;
            }
        }
    };
    // one tile for every wave of the workgroup, whatever it does with it
    constexpr int LAG_NB = THIN ? 1 : 2;
    auto step = [&](auto what) {
        constexpr int STEP = decltype(what)::value, NB = STEP == kRowsFirst || STEP == kRowsLag || STEP == kRowsLast ? LAG_NB : 2;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // the wave's part of tile t is there ...
        __builtin_amdgcn_s_barrier();                    // ... everyone's is, and the tiles that are loaded over have been read
        asm volatile("" ::: "memory");
        auto after = [](int slot, int by, int slots) { const int x = slot + by; return x >= slots ? x - slots : x; };
        const int next = (t + 1) * KG + kg;
        const bool more = next < ntiles, whole = (next + 1) * BN <= k.n;
        u16 *const nk = wk + (kslot ^ 1) * TILE, *const nv = wv + after(vslot, 1, S::VSLOTS) * TILE;
        if (more && !whole) load_end(t + 1, nk, nv);
        const size_t j1 = (size_t)next * BN;
        const int vread = STEP == kRowsLag || STEP == kRowsLast ? after(vslot, S::VSLOTS - 1, S::VSLOTS) : vslot;
        rows_tile<D, NW, KG, STEP, NB>(w, ldsK + kslot * TILE, ldsV + vread * TILE, nk, nv,
                                      (const char *)((const u16 *)k.k + j1 * k.k_rs) + koff, (const char *)((const u16 *)k.v + j1 * k.v_rs) + voff,
                                      step_k, step_v, more && whole, c, mask_tile);
        kslot ^= 1;
        vslot = after(vslot, 1, S::VSLOTS);
        ++t;
    };
    // Two waves share a SIMD (w and w + 4), and the barrier per tile keeps them in step; the upper half's P.V one tile
    // late puts one wave's MFMAs beside the other's softmax (V has a slot more then).  Loops of their own: with the
    // choice inside one loop the accumulators change registers in every trip.
    if (!lag) {
        while (t <= tl) step(std::integral_constant<int, kRowsAll>());
    } else if (tl >= 0) {
        step(std::integral_constant<int, kRowsFirst>());
        while (t <= tl) step(std::integral_constant<int, kRowsLag>());
        if (t < steps) {
            step(std::integral_constant<int, kRowsLast>());
        } else {
            rows_tile<D, NW, KG, kRowsLast, LAG_NB>(w, ldsK, ldsV + (vslot == 0 ? S::VSLOTS - 1 : vslot - 1) * TILE, wk, wv, nullptr, nullptr, 0, 0, false,
                                            c, mask_tile);
        }
    }
    while (t < steps) step(std::integral_constant<int, kRowsIdle>());
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
        w.l[nb] += __shfl_xor(w.l[nb], 16);
        w.l[nb] += __shfl_xor(w.l[nb], 32);
    }
    if constexpr (KG > 1) {
        // the other groups leave their sums to the first one
        float *so = (float *)lds;
        float2 *sml = (float2 *)(so + (KG - 1) * S::ROWS * S::OROW);
        __syncthreads();                                 // the tiles have been read
        if (kg > 0) {
#pragma unroll
            for (int nb = 0; nb < 2; ++nb) {
                const int at = (kg - 1) * S::ROWS + wave * 32 + 16 * nb + ln;
#pragma unroll
                for (int db = 0; db < DB; ++db) *(f32x4 *)(so + at * S::OROW + db * 16 + 4 * lg) = w.o[nb][db];
                if (lg == 0) sml[at] = make_float2(w.m[nb], w.l[nb]);
            }
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int g = 0; g < KG - 1; ++g)
#pragma unroll
            for (int nb = 0; nb < 2; ++nb) {
                const int at = g * S::ROWS + wave * 32 + 16 * nb + ln;
                const float2 ml = sml[at];
                const float m = fmaxf(w.m[nb], ml.x), ref = m == -INFINITY ? 0.f : m * c;
                const float mine = __builtin_amdgcn_exp2f(fmaf(w.m[nb], c, -ref)), other = __builtin_amdgcn_exp2f(fmaf(ml.x, c, -ref));
                w.m[nb] = m;
                w.l[nb] = w.l[nb] * mine + ml.y * other;
#pragma unroll
                for (int db = 0; db < DB; ++db) w.o[nb][db] = w.o[nb][db] * mine + *(const f32x4 *)(so + at * S::OROW + db * 16 + 4 * lg) * other;
            }
    }
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
        const float l = w.l[nb];
        const int row = row0 + rstep * (16 * nb + ln);
        if (row >= r.rows || (thin && nb == 1)) continue;
        if (pml) {
#pragma unroll
            for (int db = 0; db < DB; ++db) *(f32x4 *)(po + (size_t)(row - r.row0) * D + db * 16 + 4 * lg) = w.o[nb][db];
            if (lg == 0) pml[row - r.row0] = make_float2(w.m[nb] * c, l);
            continue;
        }
        int at, head;
        locate(nb, at, head);
        const float inv = l == 0.f ? 0.f : 1.0f / l;     // 0: the row sees no key
        u16 *dst = (u16 *)r.out + (size_t)head * r.o_hs + (size_t)at * r.o_rs;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            v2u y;
            y.x = pack_bf16x2(w.o[nb][db][0] * inv, w.o[nb][db][1] * inv);
            y.y = pack_bf16x2(w.o[nb][db][2] * inv, w.o[nb][db][3] * inv);
            *(v2u *)(dst + db * 16 + 4 * lg) = y;
        }
        if (lg == 0 && r.lse) r.lse[(size_t)head * r.lse_hs + at] = (w.m[nb] * c + __builtin_amdgcn_logf(l)) * kLn2;
    }
}

}  // namespace reform
