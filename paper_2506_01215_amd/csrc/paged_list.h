// How single tokens' attention over caches in pages is dealt to workgroups (see reform_paged_attend in reform.h).
//
// The list of tree_list.h: every (sequence, KV head) is an item with a place for each key tile that it goes through, and the list is
// cut into equal shares.  With a window these tiles are two runs, those of the first keys and those of the window, which are
// counted through (PagedSpan): "virtual" tiles and keys are the ones counted so.
//
// With a score the logits q.k of all virtual keys are kept, [sequence][head][virtual key], since a key's probability needs the sum
// over all keys: 4 bytes a key and head that are read once more, against d elements of K.  An item that one workgroup takes whole is
// scored by it at once; the others in a second launch, which puts the pieces together as well (paged_join).
#pragma once
#include "tree_list.h"

namespace reform {

// The key tiles that a sequence of n keys goes through.
template <int TK>
struct PagedSpan {
    int n, lo, sinks;        // keys; j >= lo or j < sinks is seen
    int front, skip, tiles;  // tiles of the first keys; tiles between them and the window's; all that are gone through
    __device__ __forceinline__ PagedSpan(const PagedParams &p, int len)
    {
        n = len;
        lo = p.window ? max(n - p.window, 0) : 0;
        sinks = min(p.n_sink, lo);
        front = (sinks + TK - 1) / TK;
        skip = max(lo / TK - front, 0);
        tiles = max((n + TK - 1) / TK - skip, 1);        // one where there is no key: the result has to be written
    }
    __device__ __forceinline__ int tile(int u) const { return u < front ? u : u + skip; }
    __device__ __forceinline__ bool seen(int j) const { return j < n && (j >= lo || j < sinks); }
};

template <int R, int TK>
__device__ __forceinline__ TreeSeq tree_seq(const PagedParams &p, int b)
{
    TreeSeq s;
    s.len = min(max(p.cache_len[b], 0), p.max_len);
    s.nodes = 1;
    s.blocks = p.row_blocks;
    s.tiles = PagedSpan<TK>(p, s.len).tiles;
    return s;
}

// What the score wants of a row: its reference (log2 units), 0 where it saw no key so that -inf stays a weight of 0, and 1 / sum.
__device__ __forceinline__ float2 score_row(float m, float l)
{
    return make_float2(m == -INFINITY ? 0.f : m, l == 0.f ? 0.f : 1.0f / l);
}

// A row's reference (log2 units) and sum with another piece's.
__device__ __forceinline__ void add_piece(float &m, float &l, float m1, float l1)
{
    const float top = fmaxf(m, m1), ref = top == -INFINITY ? 0.f : top;
    l = l * __builtin_amdgcn_exp2f(m - ref) + l1 * __builtin_amdgcn_exp2f(m1 - ref);
    m = top;
}

constexpr int kScoreChunk = 256;             // virtual keys that a wave scores at once, four to a lane

// The score of an item's virtual tiles [t0, t1) and of its part of the keys between the two runs, by waves that share out the
// chunks: this one takes those whose number, counted on from `counter` (which goes up by the item's chunks), is `mine` modulo `waves`.
// rows(r0): score_row of the group's row r0 + lane, asked for where the wave has a chunk.
template <int TK, class ROWS>
__device__ __forceinline__ void paged_score(const PagedParams &p, int b, int kvh, int len, int t0, int t1, int &counter, int mine, int waves, ROWS rows)
{
    const PagedSpan<TK> s(p, len);
    const int lane = threadIdx.x & 63, chunks = ((t1 - t0) * TK + kScoreChunk - 1) / kScoreChunk;
    int at = mine - counter % waves;
    if (at < 0) at += waves;
    counter += chunks;
    if (at >= chunks) return;
    const float c = p.scale * kLog2e;
    float *score = p.score + (size_t)b * p.score_ss + (size_t)kvh * p.score_hs;
    const float *logits = p.logits + ((size_t)b * p.Hq + (size_t)kvh * p.G) * p.logit_keys;
    float2 y = rows(0);
    for (; at < chunks; at += waves) {
        const int v0 = t0 * TK + at * kScoreChunk, v = min(v0 + 4 * lane, t1 * TK - 4);          // four keys lie in one tile
        const int j = v < s.front * TK ? v : v + s.skip * TK, here = v0 + 4 * lane < t1 * TK ? min(4, len - j) : 0;
        f32x4 before = {0.f, 0.f, 0.f, 0.f}, sum = {0.f, 0.f, 0.f, 0.f};
        if (p.accumulate && here > 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) before[e] = score[min(j + e, len - 1)];
        }
        for (int r0 = 0; r0 < p.G; r0 += 64) {
            if (p.G > 64) y = rows(r0);
            const float *x = logits + (size_t)r0 * p.logit_keys + v;
            const int n = min(64, p.G - r0);
            // four rows' logits on their way at once; behind the last row it is taken again, against its own reference (another row's
            // may lie further below than a float reaches), with a weight of 0
            for (int r = 0; r < n; r += 4) {
                f32x4 l[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) l[i] = *(const f32x4 *)(x + (size_t)min(r + i, n - 1) * p.logit_keys);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = min(r + i, n - 1);
                    const float ref = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(y.x), row));
                    const float inv = r + i < n ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(y.y), row)) : 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] += __builtin_amdgcn_exp2f(fmaf(l[i][e], c, -ref)) * inv;
                }
            }
        }
        // Beside a row whose sum is no number the weight of a key that is not seen has to stay 0: its logits are -inf in every row.
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!((sum[0] + sum[1]) + (sum[2] + sum[3]) < INFINITY)) != 0ull, 0)) {
            f32x4 most = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
            for (int r = 0; r < p.G; ++r) {
                const f32x4 l = *(const f32x4 *)(logits + (size_t)r * p.logit_keys + v);
#pragma unroll
                for (int e = 0; e < 4; ++e) most[e] = l[e] == -INFINITY ? most[e] : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = most[e] == 0.f ? sum[e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < here) score[j + e] = (j + e == len - 1 ? 0.f : before[e]) + sum[e];          // the new token has no score yet
        if (p.accumulate || s.skip == 0) continue;
        const long gap = (long)s.skip * TK;              // between the runs: as large a part as of the item's chunks
        const int a = v0 / TK, z = min(a + kScoreChunk / TK, t1);
        const int g0 = s.front * TK + (int)(gap * a / s.tiles), g1 = s.front * TK + (int)(gap * z / s.tiles);
        for (int g = g0 + lane; g < g1; g += 64) score[g] = 0.f;
    }
}

// The second launch: its first `merges` workgroups put pieces together as tree_merge does, the others score the keys of a share (or of an
// item), `parts` of them each.
template <int D, int R, int TK, bool BF16>
__global__ __launch_bounds__(256) void paged_join(PagedParams p, int merges, int rows, int by_share, int parts)
{
    using List = TreeList<R, TK, PagedParams>;
    if ((int)blockIdx.x >= merges) {
        const int block = ((int)blockIdx.x - merges) / parts, part = ((int)blockIdx.x - merges) % parts;
        const int lane = threadIdx.x & 63, mine = 4 * part + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        int counter = 0;
        auto item = [&](int b, int len, int kvh, int t0, int t1, int w0, int n) {      // n pieces from share w0 on, or 0: finished already
            paged_score<TK>(p, b, kvh, len, t0, t1, counter, mine, 4 * parts, [&](int r0) {
                // the lanes divide the rows' pieces (one lane to a row: 7 heads, 32 pieces 28.9 us the call, so 24.0; 64 pieces in fp32 81.6, 75.2)
                int width = 1;
                while (width < min(64, p.G - r0)) width *= 2;
                const int row = min(r0 + (lane & (width - 1)), p.G - 1), rb = row / R, mine0 = lane / width, step = 64 / width;
                if (n == 0) {
                    const float2 y = p.row_ml[(size_t)b * p.Hq + (size_t)kvh * p.G + row];
                    return score_row(y.x, y.y);
                }
                float m = -INFINITY, l = 0.f;
                for (int x = mine0; x < n; x += 4 * step) {                      // pieces past the last repeat it, without weight
                    float2 y[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int piece = min(x + i * step, n - 1);
                        y[i] = p.part_ml[tree_slot(p, w0 + piece, piece, rb) * p.part_rows + row - rb * R];
                        if (x + i * step >= n) y[i] = make_float2(-INFINITY, 0.f);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) add_piece(m, l, y[i].x, y[i].y);
                }
                for (int o = width; o < 64; o *= 2) add_piece(m, l, __shfl_xor(m, o), __shfl_xor(l, o));
                return score_row(m, l);
            });
        };
        if (p.shares == 0) {
            const int b = block / p.Hkv, kvh = block - b * p.Hkv;
            const TreeSeq seq = tree_seq<R, TK>(p, b);
            item(b, seq.len, kvh, 0, seq.tiles, 0, 0);
            return;
        }
        List list;
        list.read(p);
        if (block >= list.shares) return;
        int which, first;
        const int share = tree_share(block, list.shares, 1, which), begin = list.begin(share), end = list.begin(share + 1);
        int b = list.find(p, begin, first);
        TreeSeq seq = list.seq(p, b);
        int kvh = (begin - first) / tree_places(seq);
        int pos = first + kvh * tree_places(seq);
        while (pos < end) {
            const int t0 = max(begin - pos - kTreeStart, 0), t1 = min(end - pos - kTreeStart, seq.tiles);
            if (t0 < t1) {
                const int w0 = list.share_of(pos + kTreeStart), n = list.share_of(pos + kTreeStart + seq.tiles - 1) - w0 + 1;
                item(b, seq.len, kvh, t0, t1, w0, n == 1 ? 0 : n);
            }
            pos += tree_places(seq);
            if (++kvh == p.Hkv) {
                kvh = 0;
                if (++b >= p.n_seq) return;
                seq = list.seq(p, b);
            }
        }
        return;
    }
    List list;
    list.read(p);
    const int chunks = (p.part_rows + rows - 1) / rows * p.row_blocks;
    int b, kvh, pos, rb, own = -1;
    TreeSeq seq;
    if (by_share) {                                      // the item that the share's end cuts
        if ((int)blockIdx.x >= list.shares * chunks) return;
        own = tree_share(blockIdx.x, list.shares, chunks, rb);
        const int x = list.begin(own + 1) - 1;
        b = list.find(p, x, pos);
        seq = list.seq(p, b);
        kvh = (x - pos) / tree_places(seq);
    } else {                                             // an item's workgroups on the XCD that most of its shares ran on
        const int item = tree_share(blockIdx.x, p.n_seq * p.Hkv, chunks, rb);
        b = item / p.Hkv;
        kvh = item - b * p.Hkv;
        seq = list.seq(p, b);
        pos = list.before(p, b);
    }
    const int chunk = rb / p.row_blocks;
    rb -= chunk * p.row_blocks;
    pos += kvh * tree_places(seq) + kTreeStart;
    const int w0 = list.share_of(pos);
    if (by_share && w0 != own) return;
    const int n = list.share_of(pos + seq.tiles - 1) - w0 + 1;
    const int r0 = chunk * rows, here = min(rows, p.G - rb * R - r0);
    if (n == 1 || here <= 0) return;
    int r, c4;
    f32x4 y;
    float m, l;
    if (!merge_pieces<D>(p.part_o, p.part_ml, p.part_rows, n, r0, here, rows, [&](int x) { return tree_slot(p, w0 + x, x, rb); }, r, c4, y, m, l))
        return;
    const int head = kvh * p.G + rb * R + r0 + r;
    const size_t dst = (size_t)b * p.o_ss + (size_t)head * p.o_hs + c4;
    y *= l == 0.f ? 0.f : 1.0f / l;
    if (c4 < p.D) {
        if (BF16) *(v2u *)((u16 *)p.out + dst) = (v2u){pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
        else *(f32x4 *)((float *)p.out + dst) = y;
    }
    if (c4 == 0 && p.lse) p.lse[(size_t)b * p.Hq + head] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Whether an item's workgroup scores it by itself: it has all of the item's keys and rows.
__device__ __forceinline__ bool paged_scores_alone(const PagedParams &p) { return p.logits && p.shares == 0 && p.row_blocks == 1; }

template <int D, int R, int TK, bool BF16>
inline void paged_join_launch(const PagedParams &p, hipStream_t st)
{
    const bool by_share = (long)p.n_seq * p.Hkv > p.shares;
    const long blocks = (by_share ? p.shares : (long)p.n_seq * p.Hkv) * p.row_blocks;
    int rows = 1;                                        // as in tree_merge_launch
    while (2 * rows <= 1024 / D && rows < p.part_rows && blocks * ((p.part_rows + rows - 1) / rows) > 3l * p.units) rows *= 2;
    const long merges = p.shares ? blocks * ((p.part_rows + rows - 1) / rows) : 0;
    // One workgroup to a share of few logits, three to others: finding its place takes a workgroup as long as thousands of logits.  us with 1, 2, 3
    // of them: 16 caches of up to 13711 keys, 24/8 heads of 64 (10 thousand logits a share at most) 66.0, 67.7, 67.8; 4 of up to 5028, 32/8 of 128
    // (3) 22.6, 23.7, 23.8; 32 of up to 8192 (33) 135.9, 135.2, 134.3; 16 of up to 26333 (53) 250.0, 247.6, 247.4 (four: 247.7); 32 of up to 3679,
    // 64/1 (118) 43.2, 35.4, 35.3
    const long scored = p.shares ? p.shares : (long)p.n_seq * p.Hkv;
    const int parts = (double)p.n_seq * p.Hq * p.logit_keys < 24576.0 * (double)scored ? 1 : 3;
    const long scores = !p.logits || (p.shares == 0 && p.row_blocks == 1) ? 0 : parts * scored;
    if (merges + scores)
        hipLaunchKernelGGL((paged_join<D, R, TK, BF16>), dim3((unsigned)(merges + scores)), dim3(256), 0, st, p, (int)merges, rows, (int)by_share, parts);
}

// Keys that the longest sequence may go through, in whole tiles of 32, and the list for blocks of R rows and tiles of TK keys (list_plan).
inline void paged_plan(PagedParams &p, int R, int TK, int whole, int least, int workgroups)
{
    auto up = [](long x) { return (x + 31) / 32 * 32; };
    long keys = up(p.max_len);
    // a window of w keys lies in up to w / 32 + 2 tiles
    if (p.window && up(p.n_sink) + up(p.window) + 32 < keys) keys = up(p.n_sink) + up(p.window) + 32;
    if (keys < 32) keys = 32;
    p.logit_keys = (int)keys;
    list_plan(p, p.G, (double)keys, R, TK, whole, least, p.units, workgroups);
    // K and V that are read once, and too large to be there still when they are read next, as far as the host can tell: by the longest that the caches
    // may be, so short ones in a wide table take the hint as well, and the times of the small sizes.  8 sequences, pages of 16, us with / without
    // the hint, a program that goes round 3 such caches | 24 of them: 31 MB 15.6 / 13.0 | 15.8 / 17.4, 63 MB 19.8 / 19.9 | 20.3 /
    // 22.1, 127 MB 28.9 / 31.5 | 29.6 / 32.9, 399 MB 68.1 / 77.7; several row blocks (64/1 heads, 67 MB) 32.3 / 26.5 | 32.9 / 31.2
    // fp32: from twice as many bytes on (8 caches, 98 MB 33.0 / 34.0, 65 MB 31.8 / 31.6)
    p.stream = p.row_blocks == 1 && (double)p.n_seq * p.Hkv * (double)keys * p.D * 4.0 >= 64e6;
}

}  // namespace reform
