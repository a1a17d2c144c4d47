// One new token of each sequence over caches in pages (see reform_paged_attend in reform.h).
#include "attend_simple.h"

namespace reform {

// A wave has a sequence's KV head.
template <class T>
__global__ __launch_bounds__(64) void paged_attend_simple(PagedParams p)
{
    const int b = blockIdx.x / p.Hkv, g = blockIdx.x % p.Hkv;
    const int n = min(max(p.cache_len[b], 0), p.max_len), lo = p.window ? max(n - p.window, 0) : 0;
    const int32_t *table = p.pool.table + (size_t)b * p.pool.table_stride;
    const T *k = (const T *)p.k + (size_t)g * p.pool.head_stride, *v = (const T *)p.v + (size_t)g * p.pool.head_stride;
    float *score = p.score ? p.score + (size_t)b * p.score_ss + (size_t)g * p.score_hs : nullptr;
    for (int j = threadIdx.x; score && j < n; j += 64)
        if (!p.accumulate || j == n - 1) score[j] = 0.f;
    __syncthreads();
    for (int i = 0; i < p.G; ++i) {
        const int head = g * p.G + i;
        SimpleRow<T> r;
        r.begin((const T *)p.q + (size_t)b * p.q_ss + (size_t)head * p.q_hs, p.D);
        for (int j = 0; j < n; ++j) {
            if (j < lo && j >= p.n_sink) continue;
            const long at = pool_row(p.pool, table, j);
            if (at >= 0) r.key(r.logit(k + at, p.D, p.scale), v + at, p.D);
        }
        r.end((T *)p.out + (size_t)b * p.o_ss + (size_t)head * p.o_hs, p.lse ? p.lse + (size_t)b * p.Hq + head : nullptr, p.D);
        for (int j = 0; score && j < n; ++j) {
            if (j < lo && j >= p.n_sink) continue;
            const long at = pool_row(p.pool, table, j);
            if (at < 0) continue;
            const float x = r.logit(k + at, p.D, p.scale);
            if (threadIdx.x == 0) score[j] += __expf(x - r.m) / r.l;
        }
    }
}

hipError_t paged_attend_launch(const PagedParams &p, bool bf16, hipStream_t st)
{
    if (bf16) hipLaunchKernelGGL((paged_attend_simple<u16>), dim3(p.n_seq * p.Hkv), dim3(64), 0, st, p);
    else hipLaunchKernelGGL((paged_attend_simple<float>), dim3(p.n_seq * p.Hkv), dim3(64), 0, st, p);
    return hipGetLastError();
}

}  // namespace reform
