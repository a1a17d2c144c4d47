// Which form of the packed prompts' attention a batch with a sliding window takes (attend_window.hip).  Host code without device types.
//
// The forms are prompt_plan.h's (without 256 rows at head_dim 64, which no batch of those below took less time in), and the time of one is estimated as there, with as many tiles as a block goes through: those up to its last
// row's key, but no more than the window, the block's own rows and the first keys take.  The costs are of their own: with few tiles
// to a block more of them are masked, and more of the time is a block's beginning and end.
//
// Fitted to 160 batches (30 to 17000 rows, 1 to 32 sequences, windows of 1 to 6000 keys, up to 256 first ones, with and without keys in front),
// each in all forms, when a tile of the first keys held no key of the window.  Of 280 other batches, with tiles as they are, the form that is
// chosen takes 0.9 % more time in the mean than the best, at worst 36 % (222 rows of four, window 2, 16/2 heads of 128: blocks of 128 9.1 us, of
// 16 6.6); costs fitted to 170 of them anew, and without the tile that first keys add, chose no better.  Measured, us,
// blocks of 128 / 32 / 16 at head_dim 64: 525 rows of two, window 2, 14/2 heads 7.2 / 6.2 / 8.7; blocks of 128 / 128 with two
// groups / 32 / 16 at 128: 157 rows of four, window 305, 24/8 8.5 / 10.1 / 8.3 / 6.7; 1072 rows, window 146, 8/1 11.3 / 12.4 / 9.8 / 15.1.
#pragma once
#include "prompt_plan.h"

namespace reform {

inline int window_form_count(int head_dim) { return head_dim == 64 ? 3 : 4; }

inline const PromptForm *window_forms(int head_dim)
{
    static const PromptForm wide64[3] = {{128, 1, 64, 0.77, 0.89, 5.8, 3.3}, {32, 4, 32, 0.41, 0.64, 5.3, 1.6}, {16, 8, 32, 0.75, 1.98, 2.8, 3.2}};
    static const PromptForm wide128[4] = {{128, 1, 64, 1.09, 1.63, 6.1, 5.3}, {128, 2, 64, 2.52, 2.59, 6.6, 6.9},
                                          {32, 4, 32, 0.91, 1.33, 6.4, 2.9}, {16, 8, 32, 1.74, 3.32, 2.7, 3.6}};
    return head_dim == 64 ? wide64 : wide128;
}

inline double window_estimate(const PromptForm &f, int G, int Hkv, int n_seq, double n_q, double n_k, double window, double n_sink, int units)
{
    const double mean = n_q / n_seq, before = std::max(0.0, (n_k - n_q) / n_seq);
    const double part[3] = {0.25, 0.75, 2.0};
    double steps = 0.0, blocks = 0.0, longest = 0.0;
    for (int i = 0; i < 3; ++i) {
        const double len = std::max(1.0, n_seq == 1 ? mean : mean * part[i]), nb = std::ceil(len * G / f.rows), own = len / nb;
        const double most = window + own + std::min(n_sink, before + len) + (n_sink > 0.0 ? f.keys : 0.5 * f.keys);
        // keys of the blocks, the last one's `most` at most: a block that ends at row x has before + x of them
        const double first = before + own, last = before + len, all = 0.5 * (first + last);
        const double keys = most >= last ? all : most <= first ? most : all - 0.5 * (last - most) * (last - most) / (last - first);
        const double tiles = keys / f.keys + 0.5, each = std::max(1.0, tiles / f.groups + (f.groups > 1 ? 0.5 : 0.0));
        steps += n_seq / 3.0 * nb * each;
        blocks += n_seq / 3.0 * nb;
        longest = std::max(longest, std::ceil(std::ceil(std::min(last, most) / f.keys) / f.groups));
    }
    const double full = (steps * f.rate + blocks * f.block) * Hkv / units, alone = longest * f.alone;
    return f.start + std::cbrt(full * full * full + alone * alone * alone);
}

// Index of the form in window_forms(head_dim).
inline int window_choose(int head_dim, int G, int Hkv, int n_seq, int n_q, int n_k, int window, int n_sink, int units)
{
    const PromptForm *forms = window_forms(head_dim);
    int best = 0;
    double least = 0.0;
    for (int i = 0; i < window_form_count(head_dim); ++i) {
        const double t = window_estimate(forms[i], G, Hkv, n_seq, n_q, n_k, window, n_sink, units);
        if (i == 0 || t < least) { best = i; least = t; }
    }
    return best;
}

}  // namespace reform
