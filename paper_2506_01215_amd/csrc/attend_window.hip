// Attention over packed prompts whose rows see a sliding window and a few first keys (see reform_window_attend in reform.h).
#include "attend_simple.h"

namespace reform {

template <class T>
__global__ __launch_bounds__(64) void window_attend_simple(WindowParams p)
{
    const int row = blockIdx.x, head = blockIdx.y, g = head / p.G;
    const int32_t *cu_k = p.cu_k ? p.cu_k : p.cu_q;
    int q0 = 0, nq = 0, k0 = 0, nk = 0;
    for (int s = 0; s < p.n_seq; ++s) {
        const int a = min(max(p.cu_q[s], 0), p.n_q), b = min(max(p.cu_q[s + 1], 0), p.n_q);
        if (row < a || row >= b) continue;
        q0 = a;
        nq = b - a;
        k0 = min(max(cu_k[s], 0), p.n_k);
        nk = max(min(max(cu_k[s + 1], 0), p.n_k) - k0, 0);
        break;
    }
    if (nq == 0) return;
    const int t = nk - nq + row - q0;                    // the row's own key
    const int lo = max(t - p.window + 1, 0), sinks = min(p.n_sink, min(lo, t + 1));
    SimpleRow<T> r;
    r.begin((const T *)p.q + (size_t)head * p.q_hs + (size_t)row * p.q_rs, p.D);
    const T *k = (const T *)p.k + (size_t)g * p.k_hs + (size_t)k0 * p.k_rs, *v = (const T *)p.v + (size_t)g * p.v_hs + (size_t)k0 * p.v_rs;
    for (int j = 0; j < sinks; ++j) r.key(r.logit(k + (size_t)j * p.k_rs, p.D, p.scale), v + (size_t)j * p.v_rs, p.D);
    for (int j = lo; j <= t; ++j) r.key(r.logit(k + (size_t)j * p.k_rs, p.D, p.scale), v + (size_t)j * p.v_rs, p.D);
    r.end((T *)p.out + (size_t)head * p.o_hs + (size_t)row * p.o_rs, p.lse ? p.lse + (size_t)head * p.n_q + row : nullptr, p.D);
}

hipError_t window_attend_launch(const WindowParams &p, bool bf16, hipStream_t st)
{
    if (bf16) hipLaunchKernelGGL((window_attend_simple<u16>), dim3(p.n_q, p.Hq), dim3(64), 0, st, p);
    else hipLaunchKernelGGL((window_attend_simple<float>), dim3(p.n_q, p.Hq), dim3(64), 0, st, p);
    return hipGetLastError();
}

}  // namespace reform
