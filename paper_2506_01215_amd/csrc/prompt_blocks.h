// Which rows of a batch of packed prompts a workgroup takes (see reform_prompt_attend in reform.h).
//
// A sequence's rows, counted over its query rows and the G heads of a KV group, are cut into blocks of ROWS.  The
// lengths are on the device, so the host launches as many workgroups as there can be blocks, and workgroup number i
// takes the i-th longest block: causal blocks differ by the length of their sequence, and the chip is filled
// evenly to the end only if the long ones begin first.  (The search is 2.2 us of a block's time at 12 sequences; three thresholds side by side, half
// as many steps, changed no batch.)
#pragma once
#include "attend_seq.h"

namespace reform {

constexpr int kPromptSorted = 64;        // sequences whose blocks are sorted, one to a lane
// Beyond so many, counting the blocks in front of its own costs a workgroup more than the empty workgroups of places that are found by
// a search (8 heads of 128 over 2; counted / searched, us): 512 prompts of 32 rows 32 / 48, 2048 of 32 202 / 176, 8192 of 8 1085 / 255.
constexpr int kPromptCounted = 1024;

struct PromptBlock {
    int rb;                  // block of the sequence, -1: none is left
    int q0, nq, k0, nk;      // the sequence's rows
    int tiles;               // key tiles that the block sees
};

struct PromptSeq {
    int q0, nq, k0, nk, blocks;
};

template <int ROWS>
__device__ __forceinline__ PromptSeq prompt_seq(const PromptParams &p, int s)
{
    PromptSeq x;
    const int32_t *cu_k = p.cu_k ? p.cu_k : p.cu_q;
    x.q0 = min(max(p.cu_q[s], 0), p.n_q);
    x.nq = max(min(max(p.cu_q[s + 1], 0), p.n_q) - x.q0, 0);
    x.k0 = min(max(cu_k[s], 0), p.n_k);
    x.nk = max(min(max(cu_k[s + 1], 0), p.n_k) - x.k0, 0);
    x.blocks = (x.nq * p.G + ROWS - 1) / ROWS;
    return x;
}

// Blocks of a sequence that see at least `tiles` tiles of TK keys.
template <int ROWS, int TK>
__device__ __forceinline__ int prompt_blocks_with(const PromptParams &p, const PromptSeq &s, int tiles)
{
    if (tiles <= 0) return s.blocks;
    // the last row r of the block has to see key TK (tiles - 1): r >= x
    const int x = max(TK * (tiles - 1) - (s.nk - s.nq), 0);
    if (x >= s.nq) return 0;
    return s.blocks - p.G * x / ROWS;
}

template <int ROWS, int TK>
__device__ __forceinline__ PromptBlock prompt_block(const PromptParams &p, int idx)
{
    const int lane = threadIdx.x & 63;
    PromptSeq s = {0, 0, 0, 0, 0};
    int rb;
    if (p.n_seq == 1) {                                  // late (long) ones first
        s = prompt_seq<ROWS>(p, 0);
        rb = s.blocks - 1 - idx;
        if (rb < 0) return {-1, 0, 0, 0, 0, 0};
    } else if (p.n_seq <= kPromptSorted) {
        if (lane < p.n_seq) s = prompt_seq<ROWS>(p, lane);
        auto count = [&](int tiles, int &mine) {
            mine = prompt_blocks_with<ROWS, TK>(p, s, tiles);
            return __builtin_amdgcn_readlane(wave_incl_scan(mine), 63);
        };
        int mine, above;
        if (idx >= count(0, mine)) return {-1, 0, 0, 0, 0, 0};
        // the idx-th longest block sees `lo` tiles: more than idx blocks see at least lo, at most idx more than lo
        int lo = 0, hi = (p.n_k + TK - 1) / TK + 1;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (count(mid, mine) > idx) lo = mid;
            else hi = mid;
        }
        const int rest = idx - count(lo + 1, above);
        mine = prompt_blocks_with<ROWS, TK>(p, s, lo);
        const int exact = mine - above, incl = wave_incl_scan(exact);
        const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(rest < incl));
        rb = s.blocks - mine + rest - (incl - exact);
        rb = __builtin_amdgcn_readlane(rb, l);
        s = {__builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.nq, l), __builtin_amdgcn_readlane(s.k0, l),
             __builtin_amdgcn_readlane(s.nk, l), 0};
    } else if (p.n_seq <= kPromptCounted) {              // so many sequences fill the chip in any order: theirs
        int sum = 0;
        for (int s0 = 0;; s0 += 64) {
            if (s0 >= p.n_seq) return {-1, 0, 0, 0, 0, 0};
            s = {0, 0, 0, 0, 0};
            if (s0 + lane < p.n_seq) s = prompt_seq<ROWS>(p, s0 + lane);
            const int incl = wave_incl_scan(s.blocks), all = __builtin_amdgcn_readlane(incl, 63);
            if (idx < sum + all) {
                const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(idx < sum + incl));
                rb = sum + __builtin_amdgcn_readlane(incl, l) - 1 - idx;         // late ones first
                s = {__builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.nq, l),
                     __builtin_amdgcn_readlane(s.k0, l), __builtin_amdgcn_readlane(s.nk, l), 0};
                break;
            }
            sum += all;
        }
    } else {
        // sequence s has the places from front(s) on, at least as many as its rows can make blocks: found by 64 lanes at a time
        auto front = [&](int x) { return min(max(p.cu_q[x], 0), p.n_q) * p.G / ROWS + x; };
        int at = 0;
        for (int step = p.n_seq > 4096 ? 4096 : 64; step > 0; step /= 64) {
            const int x = at + lane * step;
            const int fit = __builtin_popcountll(__builtin_amdgcn_ballot_w64(x < p.n_seq && front(min(x, p.n_seq - 1)) <= idx));
            at += step * (max(fit, 1) - 1);
        }
        s = prompt_seq<ROWS>(p, at);
        rb = s.blocks - 1 - (idx - front(at));           // late ones first
        if (rb < 0 || rb >= s.blocks) return {-1, 0, 0, 0, 0, 0};
    }
    const int last = s.nk - s.nq + (min((rb + 1) * ROWS, s.nq * p.G) - 1) / p.G;         // last key that the block sees
    // the same in every lane; said here, since the compiler would keep them and all that follows in vector registers
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    return {uniform(rb), uniform(s.q0), uniform(s.nq), uniform(s.k0), uniform(s.nk), uniform(last < 0 ? 0 : last / TK + 1)};
}

template <class T>
__device__ __forceinline__ void prompt_block_operands(const PromptParams &p, const PromptBlock &b, int kvh, int row0, SeqRows &r,
                                                      SeqKeys &k)
{
    r.q = (const T *)p.q + (size_t)kvh * p.G * p.q_hs + (size_t)b.q0 * p.q_rs;
    r.out = (T *)p.out + (size_t)kvh * p.G * p.o_hs + (size_t)b.q0 * p.o_rs;
    r.lse = p.lse ? p.lse + (size_t)kvh * p.G * p.n_q + b.q0 : nullptr;
    r.q_hs = p.q_hs; r.q_rs = p.q_rs; r.o_hs = p.o_hs; r.o_rs = p.o_rs; r.lse_hs = p.n_q;
    r.G = p.G; r.row0 = row0; r.rows = b.nq * p.G;
    k.k = (const T *)p.k + (size_t)kvh * p.k_hs + (size_t)b.k0 * p.k_rs;
    k.v = (const T *)p.v + (size_t)kvh * p.v_hs + (size_t)b.k0 * p.v_rs;
    k.k_rs = p.k_rs; k.v_rs = p.v_rs;
    k.n = b.nk;
    k.shift = b.nk - b.nq;
    k.open = max(k.shift + row0 / p.G + 1, 0);
    k.parent = nullptr; k.nodes = 0;
}

// Workgroups that the blocks of any lengths fit: every sequence has at most one block that is not full.
inline unsigned prompt_grid(const PromptParams &p, int rows)
{
    const long full = (long)p.n_q * p.G / rows, part = p.n_seq > kPromptCounted || p.n_seq < p.n_q ? p.n_seq : p.n_q;
    return (unsigned)((full + part) * p.Hkv);
}

}  // namespace reform
