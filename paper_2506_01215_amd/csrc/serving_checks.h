// What the serving calls' descriptors are checked for alike (host code).
#pragma once
#include "../../include/reform.h"
#include "common.h"
#include "overlap.h"

#include <cmath>

namespace reform {

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
inline int64_t elt_size(int dtype) { return dtype == REFORM_BF16 ? 2 : 4; }
inline bool known_dtype(int dtype) { return dtype == REFORM_F32 || dtype == REFORM_BF16; }

// Strides of something that is written: its pieces of `extent` elements, at every combination of the walks' steps, must not
// overlap.  Sorted by their steps, each walk's step has to pass over all that the ones before it cover.
inline bool bad_out_strides(int64_t extent, std::initializer_list<Walk> walks)
{
    Walk w[4];
    int n = 0;
    for (const Walk &x : walks) {
        if (x.step < 0) return true;
        if (x.n > 1) w[n++] = x;
    }
    std::sort(w, w + n, [](const Walk &x, const Walk &y) { return x.step < y.step; });
    double covered = (double)extent;
    for (int i = 0; i < n; ++i) {
        if ((double)w[i].step < covered) return true;
        covered += (double)(w[i].n - 1) * (double)w[i].step;
    }
    return false;
}

// Whether an output has a byte in common with another output or an input.
inline bool mixed(std::initializer_list<Area> outs, std::initializer_list<Area> ins)
{
    for (const Area *x = outs.begin(); x != outs.end(); ++x) {
        for (const Area *y = x + 1; y != outs.end(); ++y)
            if (areas_meet(*x, *y)) return true;
        for (const Area &y : ins)
            if (areas_meet(*x, y)) return true;
    }
    return false;
}

// What the attention calls support of types and heads.
inline reform_status check_heads(int32_t dtype, int32_t n_q, int32_t n_kv, int32_t dim, float scale)
{
    if (!known_dtype(dtype) || n_q <= 0 || n_kv <= 0 || n_q % n_kv || dim <= 0) return REFORM_ERR_INVALID_ARG;
    if (!(scale > 0.f) || !std::isfinite(scale)) return REFORM_ERR_INVALID_ARG;
    if (dtype == REFORM_BF16 ? dim != 64 && dim != 128 : dim % 4 || dim > 256) return REFORM_ERR_UNSUPPORTED;
    return REFORM_OK;
}

constexpr double kMaxGroups = 8388607.0;                 // workgroups of 512 threads in a grid
constexpr int64_t kMaxRowStride = 1 << 24;               // offsets inside a tile of 64 rows stay within 32 bits

inline int compute_units()
{
    const int n = device_compute_units();
    return n > 0 ? n : 256;
}

}  // namespace reform
