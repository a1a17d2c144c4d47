// Whether tensors that are given by strides have a byte in common (an output with an input, or with another output).  Host code without
// device types.
//
// A tensor is a piece of bytes that is repeated along up to three walks.  Two of them are compared from the longest steps down: where their
// ranges have nothing in common, neither have they; where both go on with the same step, only the difference of the pieces' numbers matters,
// and few differences bring the pieces together; else the one with the longer step is taken apart, those of its pieces that lie in
// the other's range.  So heads, rows or halves of one buffer that lie between one another are told apart, exactly, in a few steps.
#pragma once
#include <algorithm>
#include <cstdint>
#include <initializer_list>

namespace reform {

struct Walk {
    int64_t n, step;
};

struct Area {
    int64_t at = 0, end = 0; // of all its bytes; both 0: there are none
    int64_t piece = 0;       // bytes of a piece
    int walks = 0;
    Walk w[3];               // steps in bytes, two pieces or more each
};

// `extent` elements of `size` bytes along walks that count in elements.  Empty where it has no piece, or would reach further than addresses do.
inline Area area_of(const void *at, int64_t size, int64_t extent, std::initializer_list<Walk> walks)
{
    Area a;
    if (!at || extent <= 0) return a;
    const int64_t most = int64_t(1) << 60;
    if (__builtin_mul_overflow(extent, size, &a.piece) || a.piece > most) return a;
    int64_t span = a.piece;
    for (const Walk &x : walks) {
        if (x.n <= 0) return a;
        if (x.n == 1 || x.step <= 0) continue;
        int64_t step, way;
        if (__builtin_mul_overflow(x.step, size, &step) || __builtin_mul_overflow(x.n - 1, step, &way) || way > most - span) return a;
        a.w[a.walks++] = {x.n, step};
        span += way;
    }
    a.at = (int64_t)(uintptr_t)at;
    a.end = a.at + span;
    return a;
}

// The same with the longest steps first.
struct Nest {
    int walks;
    Walk w[3];
    int64_t span[4];         // bytes from the first to the end of the last of the pieces along w[i], w[i + 1] ...
    explicit Nest(const Area &a) : walks(a.walks)
    {
        std::copy(a.w, a.w + walks, w);
        std::sort(w, w + walks, [](const Walk &x, const Walk &y) { return x.step > y.step; });
        span[walks] = a.piece;
        for (int i = walks - 1; i >= 0; --i) span[i] = span[i + 1] + (w[i].n - 1) * w[i].step;
    }
};

inline int64_t floor_div(int64_t x, int64_t y) { return x / y - (x % y != 0 && x < 0); }

// Pieces of a from walk i on, with the first one at `at`, and b's likewise.  `steps`: of this search, at most; strides that take more (thousands of
// pieces that lie between one another with different steps) are taken to be apart.
inline bool pieces_meet(const Nest &a, int i, int64_t at, const Nest &b, int j, int64_t bt, int &steps)
{
    if (at >= bt + b.span[j] || bt >= at + a.span[i]) return false;
    const bool more_a = i < a.walks, more_b = j < b.walks;
    if (!more_a && !more_b) return true;
    if (--steps < 0) return false;
    if (more_a && more_b && a.w[i].step == b.w[j].step) {
        const int64_t s = a.w[i].step;
        const int64_t first = std::max(floor_div(bt - at - a.span[i + 1], s) + 1, 1 - b.w[j].n);
        const int64_t last = std::min(floor_div(bt + b.span[j + 1] - at - 1, s), a.w[i].n - 1);
        for (int64_t x = first; x <= last && steps >= 0; ++x)
            if (pieces_meet(a, i + 1, at + x * s, b, j + 1, bt, steps)) return true;
        return false;
    }
    if (!more_a || (more_b && b.w[j].step > a.w[i].step)) return pieces_meet(b, j, bt, a, i, at, steps);
    const int64_t s = a.w[i].step;
    const int64_t first = std::max(floor_div(bt - at - a.span[i + 1], s) + 1, int64_t(0));
    const int64_t last = std::min(floor_div(bt + b.span[j] - at - 1, s), a.w[i].n - 1);
    for (int64_t x = first; x <= last && steps >= 0; ++x)
        if (pieces_meet(a, i + 1, at + x * s, b, j, bt, steps)) return true;
    return false;
}

inline bool areas_meet(const Area &a, const Area &b)
{
    if (a.at >= b.end || b.at >= a.end) return false;    // most of them, and empty ones
    int steps = 4096;
    return pieces_meet(Nest(a), 0, a.at, Nest(b), 0, b.at, steps);
}

}  // namespace reform
