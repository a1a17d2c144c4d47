// Which form of the packed prompts' attention a batch with a sliding window takes (attend_window.hip).  Host code without device types.
//
// The forms and their costs are prompt_plan.h's; what differs is how many tiles a block goes through: those up to its last
// row's key, but no more than the window, the block's own rows and the first keys take.
#pragma once
#include "prompt_plan.h"

namespace reform {

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

// Index of the form in prompt_forms(head_dim).
inline int window_choose(int head_dim, int G, int Hkv, int n_seq, int n_q, int n_k, int window, int n_sink, int units)
{
    const PromptForm *forms = prompt_forms(head_dim);
    int best = 0;
    double least = 0.0;
    for (int i = 0; i < kPromptForms; ++i) {
        const double t = window_estimate(forms[i], G, Hkv, n_seq, n_q, n_k, window, n_sink, units);
        if (i == 0 || t < least) { best = i; least = t; }
    }
    return best;
}

}  // namespace reform
