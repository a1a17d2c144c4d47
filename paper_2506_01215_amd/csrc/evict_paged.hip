// Caches in pages go back to their budget (see reform_paged_evict in reform.h), in two launches.
//
//   paged_select   a workgroup has one sequence's KV head: finds the budget-th score between the first and the last keys
//                  that are always kept, and lists the kept keys and the pool rows that hold them
//   paged_move     row r becomes row kept[r]: a workgroup has one head's rows, of K or of V and of those a slice of
//                  64 bytes each, and goes through them in ascending order
//
// In place without flags: rank r comes from row kept[r] >= r, so what a chunk of ranks [r0, r1) overwrites is read by
// ranks below r1 only.  A workgroup that has loaded all of a chunk may store it, and the next chunk's rows can be on their way
// meanwhile.  Slices do not touch each other's bytes.
#include "common.h"

#include <climits>

namespace reform {

namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64, kSelBins = 2048;
constexpr int kSelCached = 36864;            // candidates that stay in LDS (144 of the 160 KB)
constexpr int kMoveThreads = 512, kMoveSlice = 64, kMoveDeep = 8;

__device__ __forceinline__ int clamped_len(const PagedEvictParams &p, int b) { return min(max(p.cache_len[b], 0), p.max_len); }

// The keys are compared as ordered integers (ordered_key).  Each pass counts the candidates inside [lo, hi] in 2048 bins of
// equal width and goes on with the bin that holds the need-th largest, so three passes decide 32 bits, two where the
// scores spread over less than 22.
__global__ __launch_bounds__(kSelThreads) void paged_select(PagedEvictParams p, int cached)
{
    extern __shared__ uint32_t row[];        // [cached] candidates as ordered keys
    __shared__ int bins[kSelBins];
    __shared__ int wave_sum_[kSelWaves], wave_tie[kSelWaves], wave_out[kSelWaves];
    __shared__ uint32_t sh_lo, sh_hi;
    __shared__ int sh_need, sh_all;
    const int item = blockIdx.x, b = item / p.Hkv, g = item - b * p.Hkv;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = clamped_len(p, b);
    if (p.new_len && g == 0 && tid == 0) p.new_len[b] = min(n, p.budget);
    int32_t *kept = p.kept ? p.kept + (size_t)item * p.budget : nullptr;
    if (n <= p.budget) {
        for (int r = tid; kept && r < n; r += kSelThreads) kept[r] = r;
        return;
    }
    int32_t *src = p.src + (size_t)item * p.budget;
    const int32_t *table = p.pool.table + (size_t)b * p.pool.table_stride;
    auto list = [&](int r, int j) {          // rank r is key j
        const unsigned page = pool_page(p.pool, (unsigned)j), id = (unsigned)table[page];
        if (kept) kept[r] = j;
        src[r] = id < p.pool.n_pages ? (int)(id * p.pool.page_len + ((unsigned)j - page * p.pool.page_len)) : -1;
    };
    const float *score = p.score + (size_t)b * p.score_ss + (size_t)g * p.score_hs + p.n_sink;
    const int m = n - p.n_sink - p.n_recent, want = p.budget - p.n_sink - p.n_recent;      // candidates, and how many stay
    const bool in_lds = m <= cached;
    auto key = [&](int i) { return in_lds ? row[i] : ordered_key(score[i]); };
    if (tid == 0) { sh_lo = ~0u; sh_hi = 0u; sh_need = want; sh_all = 0; }
    __syncthreads();
    uint32_t lo = ~0u, hi = 0u;
    for (int i = tid; i < m; i += kSelThreads) {
        const uint32_t u = ordered_key(score[i]);
        if (in_lds) row[i] = u;
        lo = min(lo, u);
        hi = max(hi, u);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, o));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
    }
    if (lane == 0) { atomicMin(&sh_lo, lo); atomicMax(&sh_hi, hi); }
    __syncthreads();
    lo = sh_lo;
    hi = sh_hi;
    int need = want;                         // of the candidates inside [lo, hi]; all above hi stay
    bool all = false;                        // all inside [lo, hi] stay
    while (want > 0 && !all && lo < hi) {
        const uint32_t range = hi - lo;
        const int shift = max(21 - __clz((int)range), 0);                    // range >> shift < 2048
        for (int i = tid; i < kSelBins; i += kSelThreads) bins[i] = 0;
        __syncthreads();
        for (int i = tid; i < m; i += kSelThreads) {
            const uint32_t u = key(i) - lo;
            if (u <= range) atomicAdd(&bins[u >> shift], 1);
        }
        __syncthreads();
        // bins from the largest down, two to a thread
        const int hi_bin = bins[kSelBins - 1 - 2 * tid], lo_bin = bins[kSelBins - 2 - 2 * tid], own = hi_bin + lo_bin;
        const int incl = wave_incl_scan(own);
        if (lane == 63) wave_sum_[wave] = incl;
        __syncthreads();
        int above = incl - own;
        for (int w = 0; w < wave; ++w) above += wave_sum_[w];
        if (above < need && need <= above + own) {
            const bool first = need <= above + hi_bin;
            const uint32_t bin = kSelBins - (first ? 1 : 2) - 2 * tid;
            const int over = first ? above : above + hi_bin;
            const uint32_t from = lo + (bin << shift), wide = (1u << shift) - 1u;
            sh_lo = from;
            sh_hi = hi - from > wide ? from + wide : hi;
            sh_need = need - over;
            sh_all = need - over == (first ? hi_bin : lo_bin);
        }
        __syncthreads();
        lo = sh_lo;
        hi = sh_hi;
        need = sh_need;
        all = sh_all != 0;
    }
    // stay: above hi; inside [lo, hi] (one value, or all of them stay) the first `need`
    if (want == 0) { lo = 1u; hi = ~0u; need = 0; }
    const int each = ((m + kSelWaves - 1) / kSelWaves + 63) / 64 * 64, i0 = min(wave * each, m), i1 = min(i0 + each, m);
    int stay = 0, tie = 0;
    for (int i = i0 + lane; i < i1; i += 64) {
        const uint32_t u = key(i);
        stay += u > hi;
        tie += u >= lo && u <= hi;
    }
    stay = __builtin_amdgcn_readlane(wave_incl_scan(stay), 63);
    tie = __builtin_amdgcn_readlane(wave_incl_scan(tie), 63);
    if (lane == 0) { wave_sum_[wave] = stay; wave_tie[wave] = tie; }
    __syncthreads();
    int rank = p.n_sink, ties = 0;
    for (int w = 0; w < wave; ++w) {
        rank += wave_sum_[w];
        ties += wave_tie[w];
    }
    rank += min(ties, need);
    int first = INT_MAX;                     // first key that goes
    for (int i = i0; i < i1; i += 64) {
        const bool is = i + lane < i1;
        const uint32_t u = is ? key(i + lane) : 0u;
        const bool over = is && u > hi, same = is && u >= lo && u <= hi;
        const unsigned long long below = (1ull << lane) - 1ull, tied = __builtin_amdgcn_ballot_w64(same);
        const bool stays = over || (same && ties + __builtin_popcountll(tied & below) < need);
        const unsigned long long mask = __builtin_amdgcn_ballot_w64(stays), gone = __builtin_amdgcn_ballot_w64(is && !stays);
        if (stays) list(rank + __builtin_popcountll(mask & below), p.n_sink + i + lane);
        if (gone && first == INT_MAX) first = p.n_sink + i + __builtin_ctzll(gone);
        rank += __builtin_popcountll(mask);
        ties += __builtin_popcountll(tied);
    }
    for (int r = tid; r < p.n_sink; r += kSelThreads) list(r, r);
    for (int r = tid; r < p.n_recent; r += kSelThreads) list(p.budget - p.n_recent + r, n - p.n_recent + r);
    if (lane == 0) wave_out[wave] = first;
    __syncthreads();
    if (tid == 0) {
        for (int w = 0; w < kSelWaves; ++w) first = min(first, wave_out[w]);
        p.first[item] = first;
    }
}

// Rows [first, budget) of one head, LANES threads of 16 bytes to a row.
template <int LANES>
__device__ __forceinline__ void move_rows(const PagedEvictParams &p, int item, int first, char *base, const int32_t *table, int col)
{
    constexpr int ROWS = kMoveThreads / LANES;
    const int tr = threadIdx.x / LANES, tc = threadIdx.x % LANES;
    const int32_t *src = p.src + (size_t)item * p.budget;
    const bool in = col + tc * 16 < p.row_bytes;
    char *const at = base + col + tc * 16;
    auto address = [&](unsigned x) {         // of a pool row
        const unsigned page = pool_page(p.pool, x);
        return at + ((long)page * p.pool.page_stride + (long)(x - page * p.pool.page_len) * p.pool.row_stride) * p.elt;
    };
    int from[kMoveDeep];
    v4u data[kMoveDeep];
    auto look = [&](int r0) {
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i) {
            const int r = r0 + i * ROWS + tr;
            from[i] = in && r < p.budget ? src[r] : -1;
        }
    };
    auto load = [&] {
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i)
            if (from[i] >= 0) data[i] = *(const v4u *)address((unsigned)from[i]);
    };
    look(first);
    for (int r0 = first; r0 < p.budget; r0 += kMoveDeep * ROWS) {
        load();
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // what this wave moves has left its place ...
        __syncthreads();                                 // ... and what the others move
        char *to[kMoveDeep];
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i) {
            const int r = r0 + i * ROWS + tr;
            const long off = from[i] >= 0 ? pool_row(p.pool, table, r) : -1l;
            to[i] = off >= 0 ? at + off * p.elt : nullptr;
        }
        look(r0 + kMoveDeep * ROWS);
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i)
            if (to[i]) *(v4u *)to[i] = data[i];
    }
}

// The same for four bytes a row in one piece of memory (score, pos).
__device__ __forceinline__ void move_words(const PagedEvictParams &p, int item, int first, uint32_t *base)
{
    const int b = item / p.Hkv, n = clamped_len(p, b);
    const int32_t *kept = p.kept + (size_t)item * p.budget;
    uint32_t data[kMoveDeep];
    for (int r0 = first; r0 < p.budget; r0 += kMoveDeep * kMoveThreads) {
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i) {
            const int r = r0 + i * kMoveThreads + threadIdx.x;
            if (r < p.budget) data[i] = base[min(kept[r], n - 1)];
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMoveDeep; ++i) {
            const int r = r0 + i * kMoveThreads + threadIdx.x;
            if (r < p.budget) base[r] = data[i];
        }
    }
}

template <int LANES>
__global__ __launch_bounds__(kMoveThreads) void paged_move(PagedEvictParams p, int slices, int parts)
{
    const int item = blockIdx.x / parts, part = blockIdx.x - item * parts;
    const int b = item / p.Hkv, g = item - b * p.Hkv;
    if (clamped_len(p, b) <= p.budget) return;
    const int first = p.first[item];
    if (part < 2 * slices) {
        char *base = (char *)(part < slices ? p.k : p.v) + (size_t)g * p.pool.head_stride * p.elt;
        move_rows<LANES>(p, item, first, base, p.pool.table + (size_t)b * p.pool.table_stride, part % slices * LANES * 16);
    } else {
        const size_t at = (size_t)b * p.score_ss + (size_t)g * p.score_hs;
        move_words(p, item, first, part == 2 * slices ? (uint32_t *)p.score + at : (uint32_t *)p.pos + at);
    }
}

}  // namespace

hipError_t paged_evict_launch(const PagedEvictParams &p, hipStream_t st)
{
    const int items = p.n_seq * p.Hkv;
    const int most = p.max_len - p.n_sink - p.n_recent, cached = most < kSelCached ? (most > 0 ? most : 0) : kSelCached;
    const hipError_t e = raise_lds<paged_select>(4 * kSelCached);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_select, dim3(items), dim3(kSelThreads), 4 * (size_t)cached, st, p, cached);
    if (p.max_len <= p.budget) return hipGetLastError();
    constexpr int LANES = kMoveSlice / 16;
    const int slices = (p.row_bytes + kMoveSlice - 1) / kMoveSlice, parts = 2 * slices + (p.pos ? 2 : 1);
    hipLaunchKernelGGL((paged_move<LANES>), dim3((unsigned)items * parts), dim3(kMoveThreads), 0, st, p, slices, parts);
    return hipGetLastError();
}

}  // namespace reform
