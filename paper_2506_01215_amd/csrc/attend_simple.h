// One query row by one wave, a key at a time: softmax in one pass with a running maximum and sum.
#pragma once
#include "attend_tile.h"

namespace reform {

__device__ __forceinline__ float simple_load(const float *p) { return *p; }
__device__ __forceinline__ float simple_load(const u16 *p) { return bf16_bits_to_f32(*p); }
__device__ __forceinline__ void simple_store(float *p, float x) { *p = x; }
__device__ __forceinline__ void simple_store(u16 *p, float x) { *p = f32_to_bf16_bits(x); }

template <class T>
struct SimpleRow {
    float q[4], o[4], m, l;                              // elements lane + 64 i

    __device__ __forceinline__ void begin(const T *from, int D)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (int)threadIdx.x + 64 * i;
            q[i] = c < D ? simple_load(from + c) : 0.f;
            o[i] = 0.f;
        }
        m = -INFINITY;
        l = 0.f;
    }
    __device__ __forceinline__ float logit(const T *k, int D, float scale) const
    {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (int)threadIdx.x + 64 * i;
            if (c < D) x = fmaf(q[i], simple_load(k + c), x);
        }
        return wave_sum(x) * scale;
    }
    __device__ __forceinline__ void key(float x, const T *v, int D)
    {
        const float top = fmaxf(m, x), f = __expf(m - top), p = __expf(x - top);
        m = top;
        l = l * f + p;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (int)threadIdx.x + 64 * i;
            if (c < D) o[i] = fmaf(p, simple_load(v + c), o[i] * f);
        }
    }
    __device__ __forceinline__ void end(T *out, float *lse, int D) const
    {
        const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (int)threadIdx.x + 64 * i;
            if (c < D) simple_store(out + c, o[i] * inv);
        }
        if (lse && threadIdx.x == 0) *lse = m + logf(l);
    }
};

}  // namespace reform
