// Packed prompts of few rows behind many keys: the key tiles shared out over the whole chip (see reform_prompt_attend in reform.h).
//
// As tree_list.h, with a batch's own lists: an item is a block of R rows of one KV head of one sequence, its places are the sequence's
// key tiles and kTreeStart more, and the items of up to 64 sequences, one to a lane, form the list that is cut into shares.  The rows
// of a sequence that see fewer keys than its last ones are masked, so an item has all of the sequence's tiles.
#pragma once
#include "prompt_blocks.h"
#include "tree_list.h"

namespace reform {

template <int R, int TK>
struct PromptShares {
    PromptSeq seq;                       // sequence `lane`
    int tiles, incl;                     // its key tiles; places up to its last
    int total, shares, each, more;       // as in TreeList

    __device__ __forceinline__ explicit PromptShares(const PromptParams &p)
    {
        const int l = threadIdx.x & 63;
        seq = {0, 0, 0, 0, 0};
        if (l < p.n_seq) seq = prompt_seq<R>(p, l);
        tiles = (seq.nk + TK - 1) / TK;
        incl = wave_incl_scan(own(p));
        total = __builtin_amdgcn_readlane(incl, 63);
        const int items = __builtin_amdgcn_readlane(wave_incl_scan(seq.blocks), 63) * p.Hkv;
        const int most = (int)((unsigned)total / (unsigned)p.least);                 // as in TreeList
        shares = max(1, min(p.shares, max(items, max(min(most, p.units), most >> 1))));
        each = (int)((unsigned)total / (unsigned)shares);
        more = total - each * shares;
    }
    __device__ __forceinline__ int places() const { return tiles + kTreeStart; }
    __device__ __forceinline__ int own(const PromptParams &p) const { return seq.blocks * p.Hkv * places(); }
    __device__ __forceinline__ int begin(int share) const { return share * each + min(share, more); }
    __device__ __forceinline__ int share_of(int x) const
    {
        const int y = x - more * (each + 1);
        return y < 0 ? (int)((unsigned)x / (unsigned)(each + 1)) : more + (int)((unsigned)y / (unsigned)each);
    }
    // The sequence that place x (< total) lies in, which of its items, and that one's first place.
    __device__ __forceinline__ int find(const PromptParams &p, int x, int &item, int &pos) const
    {
        const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(x < incl));
        const int first = __builtin_amdgcn_readlane(incl - own(p), l), each_item = __builtin_amdgcn_readlane(places(), l);
        item = (x - first) / each_item;
        pos = first + item * each_item;
        return l;
    }
    // Item `item` of sequence l: KV head item % Hkv, block item / Hkv.
    __device__ __forceinline__ PromptBlock block(const PromptParams &p, int l, int item) const
    {
        return {item / p.Hkv, __builtin_amdgcn_readlane(seq.q0, l), __builtin_amdgcn_readlane(seq.nq, l), __builtin_amdgcn_readlane(seq.k0, l),
                __builtin_amdgcn_readlane(seq.nk, l), __builtin_amdgcn_readlane(tiles, l)};
    }
};

// A share's piece of an item that it does not cover alone.
__device__ __forceinline__ long prompt_slot(int share, int t0) { return 2l * share + (t0 > 0 ? 0 : 1); }

// The items of one workgroup, as tree_walk.
template <class T, int R, int TK, class F>
__device__ __forceinline__ void prompt_walk(const PromptParams &p, F f)
{
    const PromptShares<R, TK> list(p);
    if (list.total == 0 || (int)blockIdx.x >= list.shares) return;
    int which, item, pos;
    const int share = tree_share(blockIdx.x, list.shares, 1, which), begin = list.begin(share), end = list.begin(share + 1);
    int l = list.find(p, begin, item, pos);
    bool again = false;
    while (pos < end) {
        const PromptBlock blk = list.block(p, l, item);
        const int t0 = max(begin - pos - kTreeStart, 0), t1 = min(end - pos - kTreeStart, blk.tiles);
        const bool keyless = blk.tiles == 0 && begin <= pos;             // rows without keys are written by the share that their item begins in
        if (t0 < t1 || keyless) {
            if (again) __syncthreads();                  // the sums of the item before are still read
            again = true;
            const int kvh = item - blk.rb * p.Hkv;
            SeqRows r;
            SeqKeys k;
            prompt_block_operands<T>(p, blk, kvh, blk.rb * R, r, k);
            f(r, k, t0, keyless ? 0 : t1, keyless || (t0 == 0 && t1 == blk.tiles) ? -1l : prompt_slot(share, t0));
        }
        pos += blk.tiles + kTreeStart;
        if (++item == p.Hkv * ((blk.nq * p.G + R - 1) / R)) {
            item = 0;
            do {
                if (++l >= p.n_seq) return;
            } while (__builtin_amdgcn_readlane(list.seq.blocks, l) == 0);
        }
    }
}

// The pieces of the items that the shares' ends cut, `rows` rows to a workgroup.
template <int D, int R, int TK, bool BF16>
__global__ __launch_bounds__(256) void prompt_merge(PromptParams p, int rows)
{
    const PromptShares<R, TK> list(p);
    const int chunks = (p.part_rows + rows - 1) / rows;
    if (list.total == 0 || (int)blockIdx.x >= list.shares * chunks) return;
    int chunk, item, pos;
    const int own = tree_share(blockIdx.x, list.shares, chunks, chunk);
    const int l_seq = list.find(p, list.begin(own + 1) - 1, item, pos);
    const PromptBlock blk = list.block(p, l_seq, item);
    pos += kTreeStart;
    if (blk.tiles == 0 || list.share_of(pos) != own) return;
    const int n = list.share_of(pos + blk.tiles - 1) - own + 1, r0 = chunk * rows, here = min(rows, min(R, blk.nq * p.G - blk.rb * R) - r0);
    if (n <= 1 || here <= 0) return;
    int r, c4;
    f32x4 y;
    float m, l;
    if (!merge_pieces<D>(p.part_o, p.part_ml, p.part_rows, n, r0, here, rows, [&](int x) { return prompt_slot(own + x, x); }, r, c4, y, m, l)) return;
    const int row = blk.rb * R + r0 + r, at = blk.q0 + row / p.G, head = (item - blk.rb * p.Hkv) * p.G + row % p.G;
    const size_t dst = (size_t)head * p.o_hs + (size_t)at * p.o_rs + c4;
    y *= l == 0.f ? 0.f : 1.0f / l;
    if (c4 < p.D) {
        if (BF16) *(v2u *)((u16 *)p.out + dst) = (v2u){pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        else *(f32x4 *)((float *)p.out + dst) = y;
    }
    if (c4 == 0 && p.lse) p.lse[(size_t)head * p.n_q + at] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D, int R, int TK, bool BF16>
inline void prompt_merge_launch(const PromptParams &p, hipStream_t st)
{
    int rows = 1;
    while (2 * rows <= 1024 / D && rows < p.part_rows && p.shares * ((p.part_rows + rows - 1) / rows) > 3 * p.units) rows *= 2;   // as tree_merge_launch
    hipLaunchKernelGGL((prompt_merge<D, R, TK, BF16>), dim3(p.shares * ((p.part_rows + rows - 1) / rows)), dim3(256), 0, st, p, rows);
}

}  // namespace reform
