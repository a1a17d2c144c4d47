// How drafted tokens' attention is dealt to workgroups (see reform_tree_attend in reform.h).
//
// Every (sequence, KV head, row block) is an item with as many places as the sequence has key tiles, and
// kTreeStart more in front for the time it takes to begin one.  The items of all sequences form one list, and
// `shares` workgroups take equal parts of it, whatever items these cut through: a batch of caches of any lengths
// fills the chip evenly, and the host need not know the lengths.  An item that one share covers alone is
// finished there; the others' pieces are added up by tree_merge.
#pragma once
#include "attend_seq.h"

namespace reform {

constexpr int kTreeStart = 4;

struct TreeSeq {
    int len, nodes, blocks, tiles;       // cached rows, drafted nodes, row blocks, key tiles
};

template <int R, int TK>
__device__ __forceinline__ TreeSeq tree_seq(const TreeParams &p, int b)
{
    TreeSeq s;
    s.len = min(max(p.cache_len[b], 0), p.max_len);
    s.nodes = p.node_count ? min(max(p.node_count[b], 0), p.T) : p.T;
    s.blocks = (s.nodes * p.G + R - 1) / R;
    s.tiles = (s.len + s.nodes + TK - 1) / TK;
    return s;
}

// Places of one of a sequence's items, and of all of them.
__device__ __forceinline__ int tree_places(const TreeSeq &s) { return s.tiles + kTreeStart; }
__device__ __forceinline__ int tree_all_places(const TreeParams &p, const TreeSeq &s) { return p.Hkv * s.blocks * tree_places(s); }

// The list as all lanes of a wave see it.
template <int R, int TK>
struct TreeList {
    int total, shares;                   // places, shares that are not empty

    __device__ __forceinline__ explicit TreeList(const TreeParams &p)
    {
        int items = 0;
        total = 0;
        for (int b0 = 0; b0 < p.n_seq; b0 += 64) {
            int mine = 0, count = 0;
            const int b = b0 + (threadIdx.x & 63);
            if (b < p.n_seq) {
                const TreeSeq s = tree_seq<R, TK>(p, b);
                mine = tree_all_places(p, s);
                count = p.Hkv * s.blocks;
            }
            total += __builtin_amdgcn_readlane(wave_incl_scan(mine), 63);
            items += __builtin_amdgcn_readlane(wave_incl_scan(count), 63);
        }
        shares = max(1, min(p.shares, max(items, total / p.least)));
    }
    __device__ __forceinline__ int begin(int share) const { return (int)((long)total * share / shares); }
    // the share that place x lies in: begin(w) <= x  <=>  w total / shares < x + 1
    __device__ __forceinline__ int share_of(int x) const { return (int)((((long)x + 1) * shares - 1) / total); }
    // places in front of sequence b
    __device__ __forceinline__ int before(const TreeParams &p, int b) const
    {
        int sum = 0;
        for (int b0 = 0; b0 < b; b0 += 64) {
            const int x = b0 + (threadIdx.x & 63);
            const int mine = x < b ? tree_all_places(p, tree_seq<R, TK>(p, x)) : 0;
            sum += __builtin_amdgcn_readlane(wave_incl_scan(mine), 63);
        }
        return sum;
    }
    // the sequence that place x (< total) lies in, and its first place
    __device__ __forceinline__ int find(const TreeParams &p, int x, int &first) const
    {
        int sum = 0;
        for (int b0 = 0;; b0 += 64) {
            const int b = b0 + (threadIdx.x & 63);
            const int mine = b < p.n_seq ? tree_all_places(p, tree_seq<R, TK>(p, b)) : 0;
            const int incl = wave_incl_scan(mine), all = __builtin_amdgcn_readlane(incl, 63);
            if (x < sum + all) {
                const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(x < sum + incl));
                first = sum + __builtin_amdgcn_readlane(incl - mine, l);
                return b0 + l;
            }
            sum += all;
        }
    }
};

// Where a share's piece of an item that it does not cover alone goes.
__device__ __forceinline__ long tree_slot(int share, int t0) { return 2l * share + (t0 > 0 ? 0 : 1); }

// The items of one workgroup, in the list's order: f(rows, keys, first tile, last tile + 1, slot of a piece or -1).
template <class T, int R, int TK, class F>
__device__ __forceinline__ void tree_walk(const TreeParams &p, F f)
{
    auto segment = [&](int b, const TreeSeq &seq, int item, int t0, int t1, long slot) {
        const int kvh = item / seq.blocks, rb = item - kvh * seq.blocks;
        SeqRows r;
        r.q = (const T *)p.q + (size_t)b * p.q_ss + (size_t)kvh * p.G * p.q_hs;
        r.out = (T *)p.out + (size_t)b * p.o_ss + (size_t)kvh * p.G * p.o_hs;
        r.lse = p.lse ? p.lse + ((size_t)b * p.Hq + (size_t)kvh * p.G) * p.T : nullptr;
        r.q_hs = p.q_hs; r.q_rs = p.q_rs; r.o_hs = p.o_hs; r.o_rs = p.o_rs; r.lse_hs = p.T;
        r.G = p.G; r.row0 = rb * R; r.rows = seq.nodes * p.G;
        SeqKeys k;
        k.k = (const T *)p.k + (size_t)b * p.kv_ss + (size_t)kvh * p.kv_hs;
        k.v = (const T *)p.v + (size_t)b * p.kv_ss + (size_t)kvh * p.kv_hs;
        k.k_rs = k.v_rs = p.D;
        k.n = seq.len + seq.nodes; k.open = seq.len; k.shift = 0;
        k.parent = p.parent ? p.parent + (size_t)b * p.T : nullptr;
        k.nodes = seq.nodes;
        f(r, k, t0, t1, slot);
    };
    const bool whole = p.shares == 0;                    // one item to a workgroup
    int b, item, pos = 0, begin = 0, end;
    TreeSeq seq;
    if (whole) {
        const int items = p.Hkv * p.row_blocks;
        b = blockIdx.x / items;
        item = blockIdx.x - b * items;
        seq = tree_seq<R, TK>(p, b);
        if (item >= p.Hkv * seq.blocks) return;
        end = tree_places(seq);
    } else {
        const TreeList<R, TK> list(p);
        const int share = blockIdx.x;
        if (share >= list.shares || list.total == 0) return;
        begin = list.begin(share);
        end = list.begin(share + 1);
        if (begin >= end) return;
        int first;
        b = list.find(p, begin, first);
        seq = tree_seq<R, TK>(p, b);
        item = (begin - first) / tree_places(seq);
        pos = first + item * tree_places(seq);
    }
    bool again = false;
    while (pos < end) {
        const int t0 = max(begin - pos - kTreeStart, 0), t1 = min(end - pos - kTreeStart, seq.tiles);
        if (t0 < t1) {
            if (again) __syncthreads();                  // the sums of the item before are still read
            again = true;
            segment(b, seq, item, t0, t1, t0 > 0 || t1 < seq.tiles ? tree_slot(blockIdx.x, t0) : -1);
        }
        pos += tree_places(seq);
        if (whole) return;
        if (++item == p.Hkv * seq.blocks) {
            item = 0;
            do {
                if (++b >= p.n_seq) return;
                seq = tree_seq<R, TK>(p, b);
            } while (seq.blocks == 0);
        }
    }
}

// The pieces of the items that several shares covered, in the order of the shares.  A thread has four columns
// of a row and every fourth piece; four threads' sums meet in LDS.
template <int D, int R, int TK, bool BF16>
__global__ __launch_bounds__(256) void tree_merge(TreeParams p, int rows_each)
{
    constexpr int C4 = D / 4, ROWS = 64 / C4 < 1 ? 1 : 64 / C4;         // quads of a row, rows of a pass
    __shared__ f32x4 so[4][64];
    __shared__ float sl[4][64];
    const TreeList<R, TK> list(p);
    if (list.total == 0) return;
    const int per_seq = p.Hkv * p.row_blocks, chunks = (p.part_rows + rows_each - 1) / rows_each;
    const int chunk = blockIdx.x % chunks, at = blockIdx.x / chunks;
    const int b = at / per_seq, item = at - b * per_seq;
    const TreeSeq seq = tree_seq<R, TK>(p, b);
    if (item >= p.Hkv * seq.blocks) return;
    const int kvh = item / seq.blocks, rb = item - kvh * seq.blocks;
    const int pos = list.before(p, b) + item * tree_places(seq) + kTreeStart;
    const int w0 = list.share_of(pos), w1 = list.share_of(pos + seq.tiles - 1);
    if (w0 == w1) return;
    const int rows = min(R, seq.nodes * p.G - rb * R);
    const int g = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int r0 = chunk * rows_each; r0 < min((chunk + 1) * rows_each, rows); r0 += ROWS) {
        const int row = r0 + lane / C4, c4 = lane % C4 * 4;
        const bool live = row < rows && lane < ROWS * C4;
        float m = -INFINITY;
        if (live) {
            for (int w = w0; w <= w1; ++w) m = fmaxf(m, p.part_ml[(size_t)tree_slot(w, w - w0) * p.part_rows + row].x);
        }
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
        if (live) {
            for (int w = w0 + g; w <= w1; w += 4) {
                const size_t slot = (size_t)tree_slot(w, w - w0) * p.part_rows + row;
                const float2 ml = p.part_ml[slot];
                const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
                l += ml.y * f;
                y += *(const f32x4 *)(p.part_o + slot * D + c4) * f;
            }
        }
        so[g][lane] = y;
        sl[g][lane] = l;
        __syncthreads();
        if (g == 0 && live) {
#pragma unroll
            for (int i = 1; i < 4; ++i) {
                y += so[i][lane];
                l += sl[i][lane];
            }
            const int node = (rb * R + row) / p.G, head = kvh * p.G + (rb * R + row) % p.G;
            const float inv = l == 0.f ? 0.f : 1.0f / l;
            const size_t dst = (size_t)b * p.o_ss + (size_t)head * p.o_hs + (size_t)node * p.o_rs + c4;
            y *= inv;
            if (c4 < p.D) {
                if (BF16) *(v2u *)((u16 *)p.out + dst) = (v2u){pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
                else *(f32x4 *)((float *)p.out + dst) = y;
            }
            if (c4 == 0 && p.lse) p.lse[((size_t)b * p.Hq + head) * p.T + node] = (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
        }
        __syncthreads();
    }
}

template <int D, int R, int TK, bool BF16>
inline void tree_merge_launch(const TreeParams &p, hipStream_t st)
{
    const int rows_each = p.part_rows < 4 ? p.part_rows : 4;
    const unsigned chunks = (p.part_rows + rows_each - 1) / rows_each;
    hipLaunchKernelGGL((tree_merge<D, R, TK, BF16>), dim3((unsigned)p.n_seq * p.Hkv * p.row_blocks * chunks), dim3(256), 0, st, p,
                       rows_each);
}

// Row blocks, shares and the rows of a piece for blocks of R rows and tiles of TK keys.  No shares where every
// item is short (`least` tiles: what keeps the waves of one workgroup busy): then one workgroup takes an item whole,
// and there is nothing to merge.
inline void tree_plan(TreeParams &p, int R, int TK, int least, int workgroups)
{
    const int rows = p.T * p.G;
    p.row_blocks = (rows + R - 1) / R;
    p.part_rows = rows < R ? rows : R;
    p.least = least;
    const int tiles = (p.max_len + p.T + TK - 1) / TK;
    if (tiles <= least) return;
    const double items = (double)p.n_seq * p.Hkv * p.row_blocks, most = items * (tiles + kTreeStart) / least;
    const double want = items > most ? items : most;
    p.shares = want < workgroups ? (int)want : workgroups;
}

}  // namespace reform
