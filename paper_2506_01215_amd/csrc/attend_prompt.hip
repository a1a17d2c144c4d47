// Causal attention over packed prompts, bf16 (see reform_prompt_attend in reform.h).
//
//   prompt_attend<D,NW>   a workgroup takes a block of 32 NW rows of one KV head (counted over query rows and the
//                         heads of the group) over all keys that the block sees
//   prompt_attend_short   blocks of 32 rows whose eight waves divide the keys (attend_seq.h), for batches that
//                         have too few rows to fill the chip otherwise
//
// prompt_attend computes S^T = K Q^T with v_mfma_f32_16x16x32_bf16 (operand layouts in attend_bf16.hip), so that a
// lane owns one query column of each of its wave's two 16-row blocks, its softmax statistics are scalars, and the
// probabilities are the B operand of O^T = V^T P^T as they stand.  K and V tiles of 64 keys go from memory
// straight into LDS (global_load_lds, 16 bytes a lane), one tile ahead of the one that is computed.
//
// LDS: the 64 lanes of such a load land in 1024 adjacent bytes, so rows cannot be padded one by one.  Instead a load
// takes rows that no read takes together: rows c, c + 16, c + 32, c + 48 at head_dim 128 (at 64 rows c and c + 8 of
// every 16), and the loads' places ("chunks") lie 1024 + 32 bytes apart.  K's fragments (16 rows x 32 bytes per half
// wave, free of conflicts where they differ modulo 512 bytes) and V's transposing reads (8 rows x 32 bytes, modulo 256)
// then find their rows 32 bytes apart, and every fragment of a tile is at a constant distance from the lane's first.
//
// Bound: the matrix pipe, and the power it draws (attend_bf16.hip); short batches: latency.
#include "attend_seq.h"
#include "prompt_blocks.h"

#include <type_traits>

namespace reform {

constexpr int kPromptKeys = 64;

template <int D, int NW>
struct PromptShape {
    static constexpr int ROWS = NW * 32, BN = kPromptKeys, C8 = D / 8;
    static constexpr int CHUNKS = BN * D / 512, PITCH = 512 + 16, TILE = CHUNKS * PITCH;      // elements
    static constexpr int LOADS = CHUNKS / NW;            // of a wave, for K and for V
    static constexpr bool LAG = NW == 8;                 // the upper half of the waves runs P.V one tile late
    static constexpr int VSLOTS = LAG ? 3 : 2;
    static constexpr size_t lds_bytes = sizeof(u16) * (size_t)(2 + VSLOTS) * TILE;
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
struct PromptWave {
    static constexpr int KS = D / 32, DB = D / 16;
    v4u q[2][KS];
    f32x4 o[2][DB];
    float m[2], l[2];
    v4u pb[2][2];            // probabilities of a tile
    int kat, vat;            // the lane's first fragment inside a K and a V tile (elements)
};

// What a wave does while a tile's successor is on its way: nothing (it needs no more keys), Q.K^T and softmax of
// the tile, P.V of the tile (in step) or of the one before (lagging waves), in this order.
enum PromptStep { kPromptIdle, kPromptAll, kPromptFirst, kPromptLag, kPromptLast };

// The pointers are to different tiles of the LDS; `next_*` are the ones that the loads under way fill.  That
// they are different is what lets the compiler read the others without waiting for these loads.
template <int D, int NW, int STEP, class MASK>
__device__ __forceinline__ void prompt_tile(PromptWave<D> &w, const u16 *__restrict__ tk, const u16 *__restrict__ tv,
                                            u16 *__restrict__ next_k, u16 *__restrict__ next_v, const char *from_k, const char *from_v,
                                            size_t step_k, size_t step_v, bool loads, float c, MASK mask_tile)
{
    using S = PromptShape<D, NW>;
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
    if constexpr (STEP == kPromptLag || STEP == kPromptLast) {
#pragma unroll
        for (int i = 0; i < kWin; ++i) fw[i] = vfrag(i);
#pragma unroll
        for (int f = 0; f < NV; ++f) {
            w.o[0][f % DB] = mfma16(fw[f % kWin], w.pb[0][f / DB], w.o[0][f % DB]);
            w.o[1][f % DB] = mfma16(fw[f % kWin], w.pb[1][f / DB], w.o[1][f % DB]);
            const int g = f + kWin;
            if (g < NV) fw[f % kWin] = vfrag(g);
            else if (STEP == kPromptLag) fw[f % kWin] = kfrag(g - NV);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * kWin, 0);
#pragma unroll
        for (int f = 0; f < NV - kWin; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);               // a V^T fragment is two reads
        }
#pragma unroll
        for (int f = NV - kWin; f < NV; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, STEP == kPromptLag ? 1 : 0, 0);
        }
    }
    if constexpr (STEP == kPromptAll || STEP == kPromptFirst || STEP == kPromptLag) {
        if (STEP != kPromptLag) {
#pragma unroll
            for (int i = 0; i < kWin; ++i) fw[i] = kfrag(i);
        }
        f32x4 s[2][4];
#pragma unroll
        for (int nb = 0; nb < 2; ++nb)
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) s[nb][kb] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < NK; ++f) {
            s[0][f & 3] = mfma16(fw[f % kWin], w.q[0][f >> 2], s[0][f & 3]);
            s[1][f & 3] = mfma16(fw[f % kWin], w.q[1][f >> 2], s[1][f & 3]);
            const int g = f + kWin;
            if (g < NK) fw[f % kWin] = kfrag(g);
            else if (STEP == kPromptAll) fw[f % kWin] = vfrag(g - NK);
        }
        if (STEP != kPromptLag) __builtin_amdgcn_sched_group_barrier(0x100, kWin, 0);
#pragma unroll
        for (int f = 0; f < NK - kWin; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
#pragma unroll
        for (int f = NK - kWin; f < NK; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, STEP == kPromptAll ? 2 : 0, 0);
        }
        mask_tile(s);
        float rs[2];
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) rs[nb] = softmax_row(s[nb], c, w.m[nb] * c, w.pb[nb]);
        if (__builtin_amdgcn_ballot_w64(!(rs[0] < kBigSum) || !(rs[1] < kBigSum)) != 0ull) {
            asm volatile("; rescale path" ::: "memory");
#pragma unroll
            for (int nb = 0; nb < 2; ++nb) {
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
        w.l[0] += rs[0];
        w.l[1] += rs[1];
    }
    if constexpr (STEP == kPromptAll) {
#pragma unroll
        for (int f = 0; f < NV; ++f) {
            w.o[0][f % DB] = mfma16(fw[f % kWin], w.pb[0][f / DB], w.o[0][f % DB]);
            w.o[1][f % DB] = mfma16(fw[f % kWin], w.pb[1][f / DB], w.o[1][f % DB]);
            if (f + kWin < NV) fw[f % kWin] = vfrag(f + kWin);
        }
#pragma unroll
        for (int f = 0; f < NV - kWin; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
    }
}

template <int D, int NW>
__global__ __launch_bounds__(NW * 64, 2) void prompt_attend(PromptParams p)
{
    using S = PromptShape<D, NW>;
    constexpr int BN = S::BN, TILE = S::TILE, KS = S::KS, DB = S::DB, C8 = S::C8;
    extern __shared__ __attribute__((aligned(16))) u16 lds[];
    u16 *ldsK = lds, *ldsV = lds + 2 * TILE;             // [2][TILE], [VSLOTS][TILE]
    const int kvh = blockIdx.x % p.Hkv;
    const PromptBlock blk = prompt_block<S::ROWS, BN>(p, blockIdx.x / p.Hkv);
    if (blk.rb < 0) return;
    SeqRows r;
    SeqKeys k;
    prompt_block_operands<u16>(p, blk, kvh, blk.rb * S::ROWS, r, k);

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ln = lane & 15, lg = lane >> 4;
    // the wave's 32 rows: p.by_head (G divides the waves): consecutive query rows of one head, else consecutive rows
    const int slab = p.by_head ? wave / p.G : wave, rstep = p.by_head ? p.G : 1;
    const int row0 = r.row0 + slab * 32 * rstep + (p.by_head ? wave % p.G : 0);
    // formed where needed, from values that the compiler cannot relate to the other uses: kept, they cost registers in the loop
    auto locate = [&](int nb, int &at, int &head) {
        int G = p.G, l = lane;
        asm volatile("" : "+s"(G), "+v"(l));
        const int x = min(row0 + rstep * (16 * nb + (l & 15)), r.rows - 1);
        at = x / G;
        head = x - at * G;
    };
    PromptWave<D> w;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
        int at;
        int head;
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
    const float c = p.scale * kLog2e;
    const int ntiles = blk.tiles, M = k.shift;
    const int wave_last_key = row0 < r.rows ? M + min(row0 + 31 * rstep, r.rows - 1) / p.G : -1;
    const int tl = wave_last_key >= 0 ? wave_last_key / BN : -1;            // last tile that the wave needs
    const int wave_open = M + row0 / p.G;                // keys up to it are seen by all of the wave's rows

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
            const int row = min(t * BN + wave + S::lane_row(l) + i * NW, k.n - 1);
            load_to_lds((const char *)((const u16 *)k.k + (size_t)row * k.k_rs + l % C8 * 8), to_k + i * NW * S::PITCH);
            load_to_lds((const char *)((const u16 *)k.v + (size_t)row * k.v_rs + l % C8 * 8), to_v + i * NW * S::PITCH);
        }
    };
    if (ntiles > 0) load_end(0, wk, wv);
    int t = 0, vslot = 0;                                // vslot: t mod VSLOTS
    auto mask_tile = [&](f32x4 (&s)[2][4]) {
        const int j0 = t * BN;
        if (j0 + BN - 1 > wave_open) {
            asm volatile("; mask path" ::: "memory");
#pragma unroll
            for (int nb = 0; nb < 2; ++nb) {
                int at;
                int head;
                locate(nb, at, head);
                int l = lane;
                asm volatile("" : "+v"(l));
                const int lim = M + at - j0 - 4 * (l >> 4);  // of the lane's first key
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (kb * 16 + e > lim) s[nb][kb][e] = -INFINITY;
            }
        }
    };
    // one tile for every wave of the workgroup, whatever it does with it
    auto step = [&](auto what) {
        constexpr int STEP = decltype(what)::value;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // the wave's part of tile t is there
        __builtin_amdgcn_s_barrier();                    // everyone's is, and the tiles that are loaded over have been read
        asm volatile("" ::: "memory");
        const int vnext = vslot == S::VSLOTS - 1 ? 0 : vslot + 1, vprev = vslot == 0 ? S::VSLOTS - 1 : vslot - 1;
        const bool more = t + 1 < ntiles, whole = (t + 2) * BN <= k.n;
        u16 *const nk = wk + ((t + 1) & 1) * TILE, *const nv = wv + vnext * TILE;
        if (more && !whole) load_end(t + 1, nk, nv);
        const size_t j1 = (size_t)(t + 1) * BN;
        prompt_tile<D, NW, STEP>(w, ldsK + (t & 1) * TILE, ldsV + (STEP == kPromptLag || STEP == kPromptLast ? vprev : vslot) * TILE, nk, nv,
                                 (const char *)((const u16 *)k.k + j1 * k.k_rs) + koff, (const char *)((const u16 *)k.v + j1 * k.v_rs) + voff,
                                 step_k, step_v, more && whole, c, mask_tile);
        vslot = vnext;
        ++t;
    };
    // Two waves share a SIMD (w and w + 4), and the barrier per tile keeps them in step; the upper half's P.V one tile
    // late puts one wave's MFMAs beside the other's softmax (V has three places then).  Loops of their own: with the
    // choice inside one loop the accumulators change registers in every trip.
    if (!lag) {
        while (t <= tl) step(std::integral_constant<int, kPromptAll>());
    } else if (tl >= 0) {
        step(std::integral_constant<int, kPromptFirst>());
        while (t <= tl) step(std::integral_constant<int, kPromptLag>());
        if (t < ntiles) {
            step(std::integral_constant<int, kPromptLast>());
        } else {
            prompt_tile<D, NW, kPromptLast>(w, ldsK, ldsV + (vslot == 0 ? S::VSLOTS - 1 : vslot - 1) * TILE, wk, wv, nullptr, nullptr, 0, 0, false,
                                            c, mask_tile);
        }
    }
    while (t < ntiles) step(std::integral_constant<int, kPromptIdle>());
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
        float l = w.l[nb] + __shfl_xor(w.l[nb], 16);
        l += __shfl_xor(l, 32);
        if (row0 + rstep * (16 * nb + ln) >= r.rows) continue;
        int at;
        int head;
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

template <int D>
__global__ __launch_bounds__(kSeqWaves * 64, 2) void prompt_attend_short(PromptParams p)
{
    using S = SeqShape<D, 2, 1>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int kvh = blockIdx.x % p.Hkv;
    const PromptBlock blk = prompt_block<S::R, S::TK>(p, blockIdx.x / p.Hkv);
    if (blk.rb < 0) return;
    SeqRows r;
    SeqKeys k;
    prompt_block_operands<u16>(p, blk, kvh, blk.rb * S::R, r, k);
    seq_segment<D, 2, 1, false>(r, k, p.scale, 0, blk.tiles, nullptr, nullptr, smem);
}

namespace {

template <int D, int NW>
hipError_t launch_long(PromptParams p, hipStream_t st)
{
    using S = PromptShape<D, NW>;
    const hipError_t e = raise_lds<prompt_attend<D, NW>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    p.by_head = NW % p.G == 0;
    hipLaunchKernelGGL((prompt_attend<D, NW>), dim3(prompt_grid(p, S::ROWS)), dim3(NW * 64), S::lds_bytes, st, p);
    return hipGetLastError();
}

template <int D>
hipError_t launch_short(const PromptParams &p, hipStream_t st)
{
    using S = SeqShape<D, 2, 1>;
    const hipError_t e = raise_lds<prompt_attend_short<D>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((prompt_attend_short<D>), dim3(prompt_grid(p, S::R)), dim3(kSeqWaves * 64), S::lds_bytes, st, p);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const PromptParams &p, hipStream_t st)
{
    const long rows = (long)p.n_q * p.G * p.Hkv;
    if (rows <= 16384) return launch_short<D>(p, st);
    if (rows <= 65536) return launch_long<D, 4>(p, st);
    return launch_long<D, 8>(p, st);
}

}  // namespace

hipError_t prompt_attend_bf16(const PromptParams &p, hipStream_t st)
{
    return p.D == 64 ? launch<64>(p, st) : launch<128>(p, st);
}

}  // namespace reform
