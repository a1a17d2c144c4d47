// Caches in pages go back to their budget (see reform_paged_evict in reform.h).
//
//   paged_select   a workgroup has one sequence's KV head: finds the budget-th score between the first and the last keys
//                  that are always kept, and lists the kept keys; others set rows aside for the moves (stage_segments)
//   paged_move     row r becomes row kept[r]: a workgroup has one head's rows, of K or of V and of those a slice of
//                  128 bytes each, and goes through them in ascending order
//
// In place without flags: rank r comes from row kept[r] >= r, so what a chunk of ranks [r0, r1) overwrites is read by
// ranks below r1 only.  A workgroup that has loaded all of a chunk may store it, and the next chunk's rows can be on their way
// meanwhile.  Slices do not touch each other's bytes.  Few items of many rows are cut into segments of ranks that move at once; the rows
// that a segment may need of the next one's are set aside first, while the keys are selected.
//
// Bound: reading and writing the rows that move.  Cold caches, all rows moving: 112 heads from 4352 to 4096 rows of 128 elements bf16
// 440 MB in 102 us, 4.3 TB/s (a large copy: 4.9), and 8 for the selection; 8 heads from 33024 to 32768 266 MB in 63 us, 18 for the selection, which
// has one compute unit for each head, and the setting aside on the others.  Rows pass the caches' usual order of replacement (114 -> 103 us).  Chunks of 1024 threads x 4 x 16 bytes
// against 512 x 8: 95 against 103; twice as deep 150; with the next chunk's loads before this one's stores 109; 64 bytes of a row to a
// workgroup 142, 256 more than twice as slow for few items.
#include "common.h"

#include <climits>

namespace reform {

namespace {

constexpr int kSelBins = 2048, kSelGroup = 4;
constexpr int kLeastSegment = 128, kSmallSegment = 256;
constexpr int kMoveLanes = 8, kMoveDeep = 4;             // a chunk: 512 rows of 128 bytes with 1024 threads, 64 bytes a thread

__device__ __forceinline__ int clamped_len(const PagedEvictParams &p, int b) { return min(max(p.cache_len[b], 0), p.max_len); }

// Lanes below this one that are in the mask.
__device__ __forceinline__ int lanes_below(unsigned long long mask)
{
    return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
}

// ordered_key in fewer instructions (-0 + 0 is 0), and 1 at least.
__device__ __forceinline__ uint32_t candidate_key(float f)
{
    const int u = __float_as_int(f + 0.f);
    return max((uint32_t)u ^ ((uint32_t)(u >> 31) | 0x80000000u), 1u);
}

// What the waves before this one counted: one read and a scan, where a loop would wait for each of up to 15 reads.
__device__ __forceinline__ int waves_before(const int *counts, int lane, int wave)
{
    return __builtin_amdgcn_readlane(row_incl_scan(lane < wave ? counts[lane] : 0), 15);
}

// Ranks of a segment of an item that loses `gone` keys.
__host__ __device__ __forceinline__ int segment_rows(const PagedEvictParams &p, int gone)
{
    const int fit = (int)((unsigned)p.budget / (unsigned)gone), quarter = fit / 4, half = fit / 2 < p.enough ? fit / 2 : p.enough;
    int count = quarter > half ? quarter : half;
    count = count < 1 ? 1 : count < p.segs ? count : p.segs;
    return (p.budget + count - 1) / count;
}

// The segments that an item of n keys is moved in: the fewer the more keys go, since the rows that are set aside for each are that many.
// (count - 1) * gone is no more than half the budget and (p.segs - 1) * (most keys that go): paged_evict_plan's room.
struct Segments {
    int count, rows, gone;   // ranks of a segment; keys that go, rows that are set aside behind its end
    __device__ __forceinline__ Segments(const PagedEvictParams &p, int n)
    {
        gone = n - p.budget;
        rows = segment_rows(p, gone);
        count = (p.budget - 1) / rows + 1;
    }
};

__device__ __forceinline__ char *stage_of(const PagedEvictParams &p, int item, int what)
{
    return p.stage + ((size_t)item * 2 + what) * p.stage_rows * p.row_bytes;
}

// Before segments move at once: the rows that a segment's last ranks may need and the next segment overwrites, 16 bytes a thread.  These are
// the first ones behind the segment's end, whichever of them stay, so this need not wait for the selection.
template <int NT>
__device__ __forceinline__ void stage_segments(const PagedEvictParams &p, int block, int groups)
{
    const int item = block / (2 * groups), rest = block - item * 2 * groups, what = rest / groups, group = rest - what * groups;
    const int b = item / p.Hkv, g = item - b * p.Hkv, n = clamped_len(p, b);
    if (n <= p.budget) return;
    const Segments s(p, n);
    const int pieces = p.row_bytes / 16, i = group * NT + threadIdx.x;
    const int row = i / pieces, c = (i - row * pieces) * 16, seg = row / s.gone;
    if (seg >= s.count - 1) return;
    const long off = pool_row(p.pool, p.pool.table + (size_t)b * p.pool.table_stride, (seg + 1) * s.rows + row - seg * s.gone);
    const char *base = (const char *)(what ? p.v : p.k) + (size_t)g * p.pool.head_stride * p.elt;
    if (off >= 0) *(v4u *)(stage_of(p, item, what) + (size_t)row * p.row_bytes + c) = __builtin_nontemporal_load((const v4u *)(base + off * p.elt + c));
}

// The scores are compared as ordered integers (ordered_key).  Each pass counts the candidates inside [lo, hi] in 2048 bins of equal
// width and goes on with the bin that holds the need-th largest, so three passes decide 32 bits, two where the scores spread
// over less than 22.
//
// A wave has a run of candidates.  Up to K times 64 of them stay in its lanes' registers, so that a pass is its additions to LDS and the
// workgroup's barriers; of longer rows every pass reads them again, the next eight loads on their way meanwhile.
//
// What bounds it is the instructions of 16 waves on one compute unit, scalar ones as much as vector ones, so each step over 64 keys
// has few of both and no branch of its own: 8 heads of 33024 keys 28 -> 19 us in a trace, 128 of up to 4352 10.8 -> 8.4, 8 heads of
// 131328 148 -> 83 (groups of kSelGroup keys: 1 21.0, 9.2; 2 19.4, 8.6; 4 18.9, 8.4; 8 18.9, 9.5).  The rest are the first reads, 4 us, and
// barriers.
template <int NT, int K>
__global__ __launch_bounds__(NT) void paged_select(PagedEvictParams p, int groups)
{
    if ((int)blockIdx.x >= p.n_seq * p.Hkv) {
        stage_segments<NT>(p, (int)blockIdx.x - p.n_seq * p.Hkv, groups);
        return;
    }
    constexpr int NW = NT / 64, PER = kSelBins / NT;     // waves; bins of a thread
    __shared__ int bins[kSelBins];
    __shared__ int sh_a[NW], sh_b[NW];
    __shared__ uint32_t sh_lo[NW], sh_hi[NW], sh_from, sh_to;
    __shared__ int sh_need, sh_all;
    const int item = blockIdx.x, b = item / p.Hkv, g = item - b * p.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = clamped_len(p, b);
    if (p.new_len && g == 0 && tid == 0) p.new_len[b] = min(n, p.budget);
    int32_t *kept = p.kept ? p.kept + (size_t)item * p.budget : nullptr;      // null only where no sequence can outgrow its budget
    if (n <= p.budget) {
        for (int r = tid; kept && r < n; r += NT) kept[r] = r;
        return;
    }
    const float *score = p.score + (size_t)b * p.score_ss + (size_t)g * p.score_hs + p.n_sink;
    const int m = n - p.n_sink - p.n_recent, want = p.budget - p.n_sink - p.n_recent;      // candidates, and how many stay
    const int each = ((m + NW - 1) / NW + 63) / 64 * 64, i0 = min(wave * each, m), i1 = min(i0 + each, m);
    const bool kept_here = each <= 64 * K;
    // a key is 1 at least, 0 where there is no candidate: outside every [lo, hi] and above none
    auto key = [&](int i, float s) { return i + lane < i1 ? candidate_key(s) : 0u; };
    uint32_t mine[K];
    if (kept_here) {
        float s[K];                                      // all on their way before the first is looked at
#pragma unroll
        for (int x = 0; x < K; ++x) s[x] = score[min(i0 + 64 * x + lane, m - 1)];
#pragma unroll
        for (int x = 0; x < K; ++x) mine[x] = key(i0 + 64 * x, s[x]);
    }
    // f(first candidate of 64, the lane's key): the wave's candidates in order
    auto keys = [&](auto f) {
        if (kept_here) {
#pragma unroll
            for (int x = 0; x < K; x += kSelGroup)
                if (i0 + 64 * x < i1) {
#pragma unroll
                    for (int y = 0; y < kSelGroup; ++y) f(i0 + 64 * (x + y), mine[x + y]);
                }
        } else {
            float next[8];
            auto load = [&](int i) {
                if (i + 512 <= m) {
#pragma unroll
                    for (int x = 0; x < 8; ++x) next[x] = (score + i)[64 * x + lane];
                } else {
#pragma unroll
                    for (int x = 0; x < 8; ++x) next[x] = score[min(i + 64 * x + lane, m - 1)];
                }
            };
            load(i0);
            for (int i = i0; i < i1; i += 512) {
                float s[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) s[x] = next[x];
                load(i + 512);
                if (i + 512 <= i1) {
#pragma unroll
                    for (int x = 0; x < 8; ++x) f(i + 64 * x, candidate_key(s[x]));
                } else {
#pragma unroll
                    for (int x = 0; x < 8; ++x) f(i + 64 * x, key(i + 64 * x, s[x]));
                }
            }
        }
    };
    uint32_t lo = ~0u, hi = 0u;
    keys([&](int, uint32_t u) {
        lo = min(lo, u - 1u);                            // 0, no candidate, is the largest then
        hi = max(hi, u);
    });
    lo += 1u;
    if (lo == 0u) lo = ~0u;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, o));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
    }
    if (lane == 0) { sh_lo[wave] = lo; sh_hi[wave] = hi; }
    for (int i = tid; i < kSelBins; i += NT) bins[i] = 0;
    __syncthreads();
    for (int w = 0; w < NW; ++w) {
        lo = min(lo, sh_lo[w]);
        hi = max(hi, sh_hi[w]);
    }
    int need = want;                                     // of the candidates inside [lo, hi]; all above hi stay
    bool all = false;                                    // all inside [lo, hi] stay
    while (want > 0 && !all && lo < hi) {                // the bins are 0
        const uint32_t range = hi - lo;
        const int shift = max(21 - __clz((int)range), 0);                    // range >> shift < 2048
        // keys that many share would queue for one bin: the smallest (of scores: 0) is the likeliest, and is counted in a register
        int least = 0;
        keys([&](int, uint32_t u) {
            const uint32_t x = u - lo;
            least += (int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(x == 0u));
            if (x - 1u < range) atomicAdd(&bins[x >> shift], 1);
        });
        if (lane == 0 && least > 0) atomicAdd(&bins[0], least);
        __syncthreads();
        // bins from the largest down, PER to a thread
        int count[PER], own = 0;
#pragma unroll
        for (int x = 0; x < PER; ++x) {
            count[x] = bins[kSelBins - 1 - (PER * tid + x)];
            bins[kSelBins - 1 - (PER * tid + x)] = 0;
            own += count[x];
        }
        const int incl = wave_incl_scan(own);
        if (lane == 63) sh_a[wave] = incl;
        __syncthreads();
        int above = incl - own + waves_before(sh_a, lane, wave);
        if (above < need && need <= above + own) {
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                if (above < need && need <= above + count[x]) {
                    const uint32_t from = lo + ((uint32_t)(kSelBins - 1 - (PER * tid + x)) << shift), wide = (1u << shift) - 1u;
                    sh_from = from;
                    sh_to = hi - from > wide ? from + wide : hi;
                    sh_need = need - above;
                    sh_all = need - above == count[x];
                }
                above += count[x];
            }
        }
        __syncthreads();
        lo = sh_from;
        hi = sh_to;
        need = sh_need;
        all = sh_all != 0;
    }
    // stay: above hi; inside [lo, hi] (one value, or all of them stay) the first `need`
    if (want == 0) { lo = 1u; hi = ~0u; need = 0; }
    const uint32_t range = hi - lo;
    int stay = 0, tie = 0;
    keys([&](int, uint32_t u) {
        stay += u > hi;
        tie += u - lo <= range;
    });
    stay = __builtin_amdgcn_readlane(wave_incl_scan(stay), 63);
    tie = __builtin_amdgcn_readlane(wave_incl_scan(tie), 63);
    __syncthreads();                                     // sh_a has been read
    if (lane == 0) { sh_a[wave] = stay; sh_b[wave] = tie; }
    __syncthreads();
    const int stay0 = waves_before(sh_a, lane, wave), tie0 = waves_before(sh_b, lane, wave), rank = stay0 + min(tie0, need);
    int32_t *const to = kept + p.n_sink + rank;
    unsigned at = 0u;                                    // kept keys of the wave so far
    auto keep = [&](int i, unsigned long long stays) {
        if (__builtin_amdgcn_inverse_ballot_w64(stays))
            *(int32_t *)((char *)to + 4u * (at + (unsigned)lanes_below(stays))) = p.n_sink + i + lane;
        at += (unsigned)__builtin_popcountll(stays);
    };
    const bool first_goes = rank == i0 && stay0 + stay + min(tie0 + tie, need) < i1;         // no key of the waves before goes
    int first = INT_MAX;                                 // key that goes, with first_goes
    auto goes = [&](int i, unsigned long long stays) {
        if (first == INT_MAX && ~stays != 0ull) first = i + __builtin_ctzll(~stays);
    };
    if (tie0 >= need || tie0 + tie <= need) {            // the wave's ties all go, or all stay
        const uint32_t over = tie0 < need ? lo - 1u : hi;
        keys([&](int i, uint32_t u) { keep(i, __builtin_amdgcn_ballot_w64(u > over)); });
        if (first_goes) keys([&](int i, uint32_t u) { goes(i, __builtin_amdgcn_ballot_w64(u > over)); });
    } else {
        int left = need - tie0;
        keys([&](int i, uint32_t u) {
            unsigned long long stays = __builtin_amdgcn_ballot_w64(u > hi);
            const unsigned long long tied = __builtin_amdgcn_ballot_w64(u - lo <= range);
            stays |= tied & __builtin_amdgcn_ballot_w64(lanes_below(tied) < left);
            left -= (int)__builtin_popcountll(tied);
            keep(i, stays);
            goes(i, stays);
        });
    }
    if (first_goes && lane == 0) p.first[item] = p.n_sink + first;
    for (int r = tid; r < p.n_sink; r += NT) kept[r] = r;
    for (int r = tid; r < p.n_recent; r += NT) kept[p.budget - p.n_recent + r] = n - p.n_recent + r;
}

// Ranks [r0, r1) of one segment's rows, LANES threads of 16 bytes to a row.  Three things of a row follow from each other: which key it
// comes from, where that key's row is, and what is in it.  They are fetched two chunks, one chunk and no chunk ahead.  Rows from
// key `bound` on are the next segment's to overwrite: they come from `stage`, where key bound + x is row x.
template <int NT>
__device__ __forceinline__ void move_rows(const PagedEvictParams &p, const int32_t *kept, int r0, int r1, int bound, char *base, const char *stage,
                                          const int32_t *table, int col)
{
    constexpr int ROWS = NT / kMoveLanes, CHUNK = kMoveDeep * ROWS;
    const int tr = threadIdx.x / kMoveLanes, tc = threadIdx.x % kMoveLanes;
    char *const at = base + col + tc * 16;
    const char *const staged = stage + col + tc * 16;
    const int end = col + tc * 16 < p.row_bytes ? r1 : 0;                // lanes behind a row's last bytes move nothing
    int key[kMoveDeep];
    const char *from[kMoveDeep];
    char *to[kMoveDeep];
    v4u data[kMoveDeep];
    auto place = [&](int j) {
        const long off = pool_row(p.pool, table, j);
        return off >= 0 ? at + off * p.elt : nullptr;
    };
    auto keys = [&](int r) {
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i) key[i] = r + i * ROWS + tr < end ? kept[r + i * ROWS + tr] : -1;
    };
    auto places = [&](int r) {
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i) {
            from[i] = nullptr;
            if (key[i] >= bound) from[i] = pool_row(p.pool, table, key[i]) >= 0 ? staged + (size_t)(key[i] - bound) * p.row_bytes : nullptr;
            else if (key[i] >= 0) from[i] = place(key[i]);
        }
    };
    auto fetch = [&](int r) {
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i) {
            to[i] = from[i] ? place(r + i * ROWS + tr) : nullptr;
            if (from[i]) data[i] = __builtin_nontemporal_load((const v4u *)from[i]);
        }
    };
    keys(r0);
    places(r0);
    keys(r0 + CHUNK);
    fetch(r0);
    places(r0 + CHUNK);
    keys(r0 + 2 * CHUNK);
    for (; r0 < r1; r0 += CHUNK) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // what this wave moves has left its place ...
        __syncthreads();                                 // ... and what the others move
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i)
            if (to[i]) __builtin_nontemporal_store(data[i], (v4u *)to[i]);
        fetch(r0 + CHUNK);                               // none of its rows lies where this chunk goes
        places(r0 + 2 * CHUNK);
        keys(r0 + 3 * CHUNK);
    }
}

// The same for four bytes a row in one piece of memory (score, pos).
template <int NT>
__device__ __forceinline__ void move_words(const PagedEvictParams &p, const int32_t *kept, int first, int n, uint32_t *base)
{
    uint32_t data[kMoveDeep];
    for (int r0 = first; r0 < p.budget; r0 += kMoveDeep * NT) {
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i) {
            const int r = r0 + i * NT + threadIdx.x;
            if (r < p.budget) data[i] = base[min(kept[r], n - 1)];
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i) {
            const int r = r0 + i * NT + threadIdx.x;
            if (r < p.budget) base[r] = data[i];
        }
    }
}

// XCDs take workgroups in turn: those of one item are eight apart, so that a row's slices meet in one L2.
__device__ __forceinline__ int item_of(int block, int items, int parts, int &part)
{
    const int each = items >> 3, even = 8 * each * parts;                // items of an XCD
    const int j = block < even ? block >> 3 : block - even, i = j / parts;
    part = j - i * parts;
    return block < even ? (block & 7) * each + i : 8 * each + i;
}

template <int NT>
__global__ __launch_bounds__(NT) void paged_move(PagedEvictParams p, int slices, int parts)
{
    int part;
    const int item = item_of(blockIdx.x, p.n_seq * p.Hkv, parts, part);
    const int b = item / p.Hkv, g = item - b * p.Hkv, n = clamped_len(p, b);
    if (n <= p.budget) return;
    const int first = p.first[item];
    const int32_t *kept = p.kept + (size_t)item * p.budget;
    if (part >= 2 * slices * p.segs) {
        const size_t at = (size_t)b * p.score_ss + (size_t)g * p.score_hs;
        move_words<NT>(p, kept, first, n, part == 2 * slices * p.segs ? (uint32_t *)p.score + at : (uint32_t *)p.pos + at);
        return;
    }
    const Segments s(p, n);
    const int seg = part / (2 * slices), rest = part - seg * 2 * slices, what = rest / slices;
    const bool last = seg == s.count - 1;
    const int r0 = max(first, seg * s.rows), r1 = last ? p.budget : (seg + 1) * s.rows;
    if (seg >= s.count || r0 >= r1) return;
    move_rows<NT>(p, kept, r0, r1, last ? INT_MAX : r1, (char *)(what ? p.v : p.k) + (size_t)g * p.pool.head_stride * p.elt,
                  last ? nullptr : stage_of(p, item, what) + (size_t)seg * s.gone * p.row_bytes, p.pool.table + (size_t)b * p.pool.table_stride,
                  rest % slices * kMoveLanes * 16);
}

}  // namespace

// How many segments an item's rows are moved in, at most: as makes 1.75 workgroups for each compute unit.  A segment's chunks follow each other, some
// 4 us each whatever else runs, so few workgroups leave the chip idle.  The call, us, cold caches of heads 128 wide, all rows moving, at 1, 1.25, 1.5,
// 1.75, 2 and 3 workgroups: 8 heads of 32768 rows 96, 106, 97, 93, 100, 98 (whole 350); 16 of them 195, 172, 156, 149, 158, 158; 64 of 8192 (rounded
// to two segments from 1.5 on) 179, 178, 134, 134, 135, 152; over 74 batches 12, 9, 2.4, 0.8, 1.1 and 4.6 % above the best of them.  112 heads of 4096,
// which move in one: 102, in two 106.
//
// Segments of 128 rows at least (of 1024, 512, 256, 128: 8 heads of 1827 rows 27.5, 19.3, 18.6, 18.2; 4 of 444 14.2, 14.0, 13.8, 12.2), and of four times the
// rows that are set aside for one, or twice if that leaves compute units idle (twice / four times: 8 heads of 64 in fp32 that lose 671 of 7517 rows 35.8 / 49.2,
// 8 of 128 that lose 441 of 4891 32.5 / 39.2; with a workgroup to each compute unit at four times, 8 heads that lose 512
// of 16896 63 / 55, 8 of 64 in fp32 that lose 256 of 8448 38 / 32).
// Short segments in workgroups of 512 threads, since their chunks would be half empty (152 heads back to 114 rows 18.6 -> 15.8; 12 back to 372 13.7 -> 14.8).
void paged_evict_plan(PagedEvictParams &p)
{
    const double items = (double)p.n_seq * p.Hkv;
    const int slices = (p.row_bytes + kMoveLanes * 16 - 1) / (kMoveLanes * 16), most_gone = p.max_len - p.budget;
    p.segs = 1;
    p.move_threads = p.budget <= kSmallSegment ? 512 : 1024;
    p.stage_rows = 0;
    if (most_gone <= 0) return;
    const double one = p.units / (items * 2.0 * slices), want = 1.75 * one + 0.5;            // segments for a workgroup to each compute unit
    int segs = want < 32.0 ? (int)want : 32;
    p.enough = (int)one;
    if (segs > p.budget / kLeastSegment) segs = p.budget / kLeastSegment;
    if (segs <= 1 || items * p.budget * p.row_bytes / 16.0 >= 2147483648.0) return;        // threads of stage_segments
    p.segs = segs;
    // workgroups of segments that there are not would cost some us, unless it is not known how few keys may go
    const int fit = p.budget / most_gone, rows = segment_rows(p, most_gone);
    if (fit >= 4) p.segs = (p.budget - 1) / rows + 1;
    if (rows <= kSmallSegment) p.move_threads = 512;
    const int64_t all = (int64_t)(p.segs - 1) * most_gone;
    p.stage_rows = all < p.budget / 2 ? (int)all : p.budget / 2;
}

size_t paged_evict_stage_bytes(const PagedEvictParams &p) { return (size_t)p.n_seq * p.Hkv * 2 * p.stage_rows * p.row_bytes; }

hipError_t paged_evict_launch(const PagedEvictParams &p, hipStream_t st)
{
    const int items = p.n_seq * p.Hkv, most = p.max_len - p.n_sink - p.n_recent;
    auto select = [&](auto kernel, int threads) {
        const int groups = (p.stage_rows * (p.row_bytes / 16) + threads - 1) / threads;
        hipLaunchKernelGGL(kernel, dim3((unsigned)items * (1 + 2 * groups)), dim3(threads), 0, st, p, groups);
    };
    if (most <= 2048) select(paged_select<256, 8>, 256);
    else if (most <= 8192) select(paged_select<1024, 8>, 1024);
    else select(paged_select<1024, 32>, 1024);
    if (p.max_len <= p.budget) return hipGetLastError();
    const int slices = (p.row_bytes + kMoveLanes * 16 - 1) / (kMoveLanes * 16), parts = 2 * slices * p.segs + (p.pos ? 2 : 1);
    if (p.move_threads == 512) hipLaunchKernelGGL(paged_move<512>, dim3((unsigned)items * parts), dim3(512), 0, st, p, slices, parts);
    else hipLaunchKernelGGL(paged_move<1024>, dim3((unsigned)items * parts), dim3(1024), 0, st, p, slices, parts);
    return hipGetLastError();
}

}  // namespace reform
