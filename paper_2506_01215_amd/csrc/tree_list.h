// How drafted tokens' attention is dealt to workgroups (see reform_tree_attend in reform.h).
//
// Every (sequence, KV head) is an item with as many places as the sequence has key tiles, and kTreeStart more in front
// for the time it takes to begin one.  The items of all sequences form one list, which is cut into `shares` equal
// parts, whatever items these cut through: a batch of caches of any lengths fills the chip evenly, and the host
// need not know the lengths.  The rows of an item (nodes times heads of the group) may be several blocks: then as
// many workgroups go through a share side by side, on one XCD, so that K and V come from memory once and for the other
// blocks from its L2.  An item that one share covers alone is finished there; the others' pieces are added up by
// tree_merge.
#pragma once
#include "attend_seq.h"

#include <cmath>

namespace reform {

constexpr int kTreeStart = 8;

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
__device__ __forceinline__ int tree_items(const TreeParams &p, const TreeSeq &s) { return s.blocks ? p.Hkv : 0; }
__device__ __forceinline__ int tree_all_places(const TreeParams &p, const TreeSeq &s) { return tree_items(p, s) * tree_places(s); }

// The list as all lanes of a wave see it.  The first 64 sequences stay in the lanes' registers: with no more
// than these the lengths are read once.
template <int R, int TK>
struct TreeList {
    int total, shares;                   // places, shares that are not empty
    int each, more;                      // places of a share; the first `more` shares have one place more
    TreeSeq lane;                        // sequence `lane`
    int lane_places;                     // and its places

    __device__ __forceinline__ int load(const TreeParams &p, int b, TreeSeq &s) const
    {
        s = {0, 0, 0, 0};
        if (b >= p.n_seq) return 0;
        s = tree_seq<R, TK>(p, b);
        return tree_all_places(p, s);
    }
    __device__ __forceinline__ void read(const TreeParams &p)
    {
        const int l = threadIdx.x & 63;
        lane_places = load(p, l, lane);
        int places = lane_places, items = tree_items(p, lane);
#pragma unroll 4
        for (int b = 64 + l; b < p.n_seq; b += 64) {
            TreeSeq s;
            places += load(p, b, s);
            items += tree_items(p, s);
        }
        total = __builtin_amdgcn_readlane(wave_incl_scan(places), 63);
        items = __builtin_amdgcn_readlane(wave_incl_scan(items), 63);
        // up to a share for every compute unit short ones, beyond that (two workgroups to a unit) of twice as many places at least
        const int most = (int)((unsigned)total / (unsigned)max(p.least, 1));
        shares = max(1, min(p.shares, max(items, max(min(most, p.units), most >> 1))));
        each = (int)((unsigned)total / (unsigned)shares);
        more = total - each * shares;
    }
    __device__ __forceinline__ int begin(int share) const { return share * each + min(share, more); }
    __device__ __forceinline__ int share_of(int x) const           // the share that place x lies in
    {
        const int y = x - more * (each + 1);
        return y < 0 ? (int)((unsigned)x / (unsigned)(each + 1)) : more + (int)((unsigned)y / (unsigned)each);
    }
    // sequence b (the same in all lanes)
    __device__ __forceinline__ TreeSeq seq(const TreeParams &p, int b) const
    {
        if (b >= 64) return tree_seq<R, TK>(p, b);
        return {__builtin_amdgcn_readlane(lane.len, b), __builtin_amdgcn_readlane(lane.nodes, b),
                __builtin_amdgcn_readlane(lane.blocks, b), __builtin_amdgcn_readlane(lane.tiles, b)};
    }
    // places in front of sequence b
    __device__ __forceinline__ int before(const TreeParams &p, int b) const
    {
        const int l = threadIdx.x & 63;
        int places = l < b ? lane_places : 0;
#pragma unroll 4
        for (int x = 64 + l; x < b; x += 64) {
            TreeSeq s;
            places += load(p, x, s);
        }
        return __builtin_amdgcn_readlane(wave_incl_scan(places), 63);
    }
    // the sequence that place x (< total) lies in, and its first place
    __device__ __forceinline__ int find(const TreeParams &p, int x, int &first) const
    {
        const int l = threadIdx.x & 63;
        int sum = 0, mine[4] = {lane_places, 0, 0, 0};
        for (int b0 = 0, n = 1;; b0 += 64 * n, n = 4) {  // n sequences to a lane
            if (b0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    TreeSeq s;
                    mine[i] = load(p, b0 + 4 * l + i, s);
                }
            }
            const int own = mine[0] + mine[1] + mine[2] + mine[3], incl = wave_incl_scan(own), all = __builtin_amdgcn_readlane(incl, 63);
            if (x < sum + all) {
                const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(x < sum + incl));
                first = sum + __builtin_amdgcn_readlane(incl - own, at);
                int b = b0 + n * at;
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    const int places = __builtin_amdgcn_readlane(mine[i], at);
                    if (x < first + places) return b;
                    first += places;
                    ++b;
                }
                return b;
            }
            sum += all;
        }
    }
};

// Share of a workgroup, and which one of the share's `side` workgroups it is.  Workgroups go to the eight XCDs in turn, so those of
// one share are eight apart.
__device__ __forceinline__ int tree_share(int block, int shares, int side, int &which)
{
    const int each = shares >> 3, even = 8 * each * side;                // shares of an XCD
    const int j = block < even ? block >> 3 : block - even;
    const int s = j / side;
    which = j - s * side;
    return block < even ? (block & 7) * each + s : 8 * each + s;
}

// Where a share's piece of an item that it does not cover alone goes.
__device__ __forceinline__ long tree_slot(const TreeParams &p, int share, int t0, int rb)
{
    return (2l * share + (t0 > 0 ? 0 : 1)) * p.row_blocks + rb;
}

// The items of one workgroup, in the list's order: f(rows, keys, first tile, last tile + 1, slot of a piece or -1).
template <class T, int R, int TK, class F>
__device__ __forceinline__ void tree_walk(const TreeParams &p, F f)
{
    int rb;
    auto segment = [&](int b, const TreeSeq &seq, int kvh, int t0, int t1, long slot) {
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
    TreeList<R, TK> list;
    int b, kvh, pos = 0, begin = 0, end, share = 0;
    TreeSeq seq;
    if (whole) {
        const int item = blockIdx.x / p.row_blocks;
        rb = blockIdx.x - item * p.row_blocks;
        b = item / p.Hkv;
        kvh = item - b * p.Hkv;
        seq = tree_seq<R, TK>(p, b);
        if (rb >= seq.blocks) return;
        end = tree_places(seq);
    } else {
        list.read(p);
        if ((int)blockIdx.x >= list.shares * p.row_blocks || list.total == 0) return;
        share = tree_share(blockIdx.x, list.shares, p.row_blocks, rb);
        begin = list.begin(share);
        end = list.begin(share + 1);
        int first;
        b = list.find(p, begin, first);
        seq = list.seq(p, b);
        kvh = (begin - first) / tree_places(seq);
        pos = first + kvh * tree_places(seq);
    }
    bool again = false;
    while (pos < end) {
        const int t0 = max(begin - pos - kTreeStart, 0), t1 = min(end - pos - kTreeStart, seq.tiles);
        if (t0 < t1 && rb < seq.blocks) {
            if (again) __syncthreads();                  // the sums of the item before are still read
            again = true;
            segment(b, seq, kvh, t0, t1, t0 > 0 || t1 < seq.tiles ? tree_slot(p, share, t0, rb) : -1);
        }
        pos += tree_places(seq);
        if (whole) return;
        if (++kvh == p.Hkv) {
            kvh = 0;
            do {
                if (++b >= p.n_seq) return;
                seq = list.seq(p, b);
            } while (seq.blocks == 0);
        }
    }
}

// Two for each of this chip's 256 compute units: the most that any form keeps there at once.
constexpr int kTreeMaxShares = 512;

// Row r0 + r of an item's n pieces, piece x in slot slot(x), put together by a workgroup of 256 threads that has `rows` rows (a power of
// two), of which `here` exist.  A thread has four columns of one of them and every n-th piece, which it adds up against the largest
// reference of its own, references, sums and columns all loaded at once; then the n threads' sums meet in LDS.  The order is that
// of the shares, whoever is done first.  True for the threads that then have the result of row r, columns c4 on.
template <int D, class SLOT>
__device__ __forceinline__ bool merge_pieces(const float *part_o, const float2 *part_ml, int part_rows, int n, int r0, int here, int rows,
                                             SLOT slot, int &r, int &c4, f32x4 &y, float &m, float &l)
{
    constexpr int C4 = D / 4, BATCH = 4;                 // quads of a row, pieces of a trip
    __shared__ f32x4 so[256];
    __shared__ float2 sml[256];
    const int group = rows * C4, groups = 256 / group;   // threads that have different quads
    const int g = threadIdx.x / group, q = threadIdx.x - g * group;
    r = q / C4;
    c4 = q % C4 * 4;
    y = (f32x4){0.f, 0.f, 0.f, 0.f};
    m = -INFINITY;
    l = 0.f;
    if (g < groups && r < here) {
        for (int w = g; w < n; w += BATCH * groups) {
            float2 ml[BATCH];
            f32x4 o[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {            // pieces past the last repeat it, without weight
                const int x = min(w + i * groups, n - 1);
                const size_t at = (size_t)slot(x) * part_rows + r0 + r;
                ml[i] = part_ml[at];
                o[i] = *(const f32x4 *)(part_o + at * D + c4);
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (w + i * groups >= n) ml[i] = make_float2(-INFINITY, 0.f);
                top = fmaxf(top, ml[i].x);
            }
            const float ref = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f(m - ref);
            y *= old;
            l *= old;
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (w + i * groups >= n) continue;
                const float f = __builtin_amdgcn_exp2f(ml[i].x - ref);           // 0 where no key was seen
                l += ml[i].y * f;
                y += o[i] * f;
            }
            m = top;
        }
    }
    so[threadIdx.x] = y;
    sml[threadIdx.x] = make_float2(m, l);
    __syncthreads();
    if (g != 0 || r >= here) return false;
    for (int i = 1; i < groups; ++i) m = fmaxf(m, sml[i * group + q].x);
    const float ref = m == -INFINITY ? 0.f : m;
    y = (f32x4){0.f, 0.f, 0.f, 0.f};
    l = 0.f;
    for (int i = 0; i < groups; ++i) {
        const float2 ml = sml[i * group + q];
        const float f = __builtin_amdgcn_exp2f(ml.x - ref);
        l += ml.y * f;
        y += so[i * group + q] * f;
    }
    return true;
}

// The pieces of the items that several shares covered.  A workgroup has `rows` rows of the item that the end of its share cuts (by_share), or
// of an item whether it is cut or not.
template <int D, int R, int TK, bool BF16>
__global__ __launch_bounds__(256) void tree_merge(TreeParams p, int rows, int by_share)
{
    TreeList<R, TK> list;
    list.read(p);
    if (list.total == 0) return;
    const int chunks = (p.part_rows + rows - 1) / rows * p.row_blocks;
    int b, kvh, pos, rb, w0, own = -1;
    TreeSeq seq;
    if (by_share) {                                      // the item that the share's end cuts
        if ((int)blockIdx.x >= list.shares * chunks) return;
        own = tree_share(blockIdx.x, list.shares, chunks, rb);
        const int x = list.begin(own + 1) - 1;
        b = list.find(p, x, pos);
        seq = list.seq(p, b);
        kvh = (x - pos) / tree_places(seq);
    } else {
        // an item's workgroups on the XCD that most of its shares ran on (tree_share): its L2 holds the pieces
        const int item = tree_share(blockIdx.x, p.n_seq * p.Hkv, chunks, rb);
        b = item / p.Hkv;
        kvh = item - b * p.Hkv;
        seq = list.seq(p, b);
        pos = list.before(p, b);
    }
    const int chunk = rb / p.row_blocks;
    rb -= chunk * p.row_blocks;
    if (rb >= seq.blocks) return;
    pos += kvh * tree_places(seq) + kTreeStart;
    w0 = list.share_of(pos);
    if (by_share && w0 != own) return;
    const int n = list.share_of(pos + seq.tiles - 1) - w0 + 1;
    const int r0 = chunk * rows, here = min(rows, seq.nodes * p.G - rb * R - r0);
    if (n == 1 || here <= 0) return;
    int r, c4;
    f32x4 y;
    float m, l;
    if (!merge_pieces<D>(p.part_o, p.part_ml, p.part_rows, n, r0, here, rows, [&](int x) { return tree_slot(p, w0 + x, x, rb); }, r, c4, y, m, l))
        return;
    const int row = rb * R + r0 + r, node = row / p.G, head = kvh * p.G + row % p.G;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const size_t dst = (size_t)b * p.o_ss + (size_t)head * p.o_hs + (size_t)node * p.o_rs + c4;
    y *= inv;
    if (c4 < p.D) {
        if (BF16) *(v2u *)((u16 *)p.out + dst) = (v2u){pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        else *(f32x4 *)((float *)p.out + dst) = y;
    }
    if (c4 == 0 && p.lse) p.lse[((size_t)b * p.Hq + head) * p.T + node] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// With more items than shares most are finished by one workgroup, so the shares' ends are gone through, else the items (32/8 heads of
// 128, 30 nodes, caches of up to 2000 rows, us, by share / by item: 512 caches 556 / 690, 16 caches 44 / 36; 8 nodes,
// 8/2 heads, 8192 caches of 1000 rows 1715 / 3225).
// One row to a workgroup where that makes no more than three workgroups a compute unit, else two, four or more (16 ragged caches, 17 nodes, 24/8 heads
// of 64, whole call, two inputs in turn: up to eight 28.1 us, three 25.7, one 25.6, on another machine 28.4 and 25.3; one cache, 48 nodes, 32/8 of
// 128: 32.7, 32.4, 35.3.  With more inputs in turn, whose caches come from memory, the first takes 28.9).
template <int D, int R, int TK, bool BF16>
inline void tree_merge_launch(const TreeParams &p, hipStream_t st)
{
    const bool by_share = (long)p.n_seq * p.Hkv > p.shares;
    const long blocks = (by_share ? p.shares : (long)p.n_seq * p.Hkv) * p.row_blocks;
    int rows = 1;
    while (2 * rows <= 1024 / D && rows < p.part_rows && blocks * ((p.part_rows + rows - 1) / rows) > 3l * p.units) rows *= 2;
    const unsigned chunks = (p.part_rows + rows - 1) / rows;
    hipLaunchKernelGGL((tree_merge<D, R, TK, BF16>), dim3((unsigned)blocks * chunks), dim3(256), 0, st, p, rows, (int)by_share);
}

// Row blocks, shares and the rows of a piece for blocks of R rows and tiles of TK keys.  `least`: tiles that a share has at least (TreeList).
// No shares where every item is short: then one workgroup takes an item whole, and there is nothing to merge.  Short is up to
// `whole` keys where one item is alone on the chip, and up to 2.5 times as many where there are as many items as compute
// units, since sharing these out gains only what their lengths differ by.
inline void tree_plan(TreeParams &p, int R, int TK, int whole, int least, int compute_units, int workgroups)
{
    const int rows = p.T * p.G;
    p.block = R;
    p.row_blocks = (rows + R - 1) / R;
    p.part_rows = rows < R ? rows : R;
    p.least = least;
    p.units = compute_units;
    const double items = (double)p.n_seq * p.Hkv, taken = items * p.row_blocks < compute_units ? items * p.row_blocks / compute_units : 1.0;
    const double keys = (double)p.max_len + p.T;
    if (keys * (1.0 - 0.6 * taken) <= whole) return;
    const double most = items * (std::ceil(keys / TK) + kTreeStart) / least;
    const double want = items > most ? items : most;
    int room = workgroups / p.row_blocks;
    room = room < 1 ? 1 : room > kTreeMaxShares ? kTreeMaxShares : room;
    p.shares = want < room ? (int)want : room;
}

}  // namespace reform
