// Which form of the packed prompts' attention a batch takes (attend_prompt.hip).  Host code without device types.
//
// The lengths are on the device; the host knows the rows of the whole batch and the number of sequences.  It takes a
// quarter, three quarters and twice the mean length for a third of the sequences each, and estimates every form's
// time in microseconds: what all blocks' steps take at the rate of the whole chip, and what the longest block takes by
// itself.  A step is one key tile of each of the form's groups of waves.
//
// The constants were fitted to measurements of 136 batches (60 to 12000 rows, 1 to 24 sequences, 1 to 8 heads a group, with
// and without keys in front) in every form: mean error 5 to 9 %, and the form that is chosen takes 1 to 2 % more time in
// the mean than the best, at worst 24 %.  Examples, us, blocks of 256 / 128 / 128 with two groups / 64 with two groups / 32
// with eight: head_dim 64, one prompt of 700, 24/8 heads 18 / 15 / 14 / 12 / 19, of 700, 4/4 heads 18 / 14 / 13 / 11 / 9, 24 of
// together 11988, 24/8 68 / 66 / 102 / 89 / 246; head_dim 128, one of 1500, 32/8 46 / 39 / 35 / 50 / 74, of 3200, 8/8 82 / 64 / 52 /
// 44 / 59, six of together 11996, 32/8 371 / 365 / 427 / 675 / 886.
#pragma once
#include <algorithm>
#include <cmath>

namespace reform {

// Blocks of `rows` rows, by `groups` groups of waves that divide the key tiles of `keys` keys.
struct PromptForm {
    int rows, groups, keys;
    double rate;             // us for a step of every compute unit's share of the blocks, chip full
    double alone;            // us for a step of a block by itself
    double start, block;     // us a call, and for a block of every compute unit
};

constexpr int kPromptForms = 4;

inline const PromptForm *prompt_forms(int head_dim)
{
    static const PromptForm wide64[kPromptForms] = {{256, 1, 64, 1.07, 1.05, 7.5, 4.2}, {128, 1, 64, 0.551, 0.726, 6.6, 2.02},
                                                    {64, 2, 64, 0.634, 0.782, 6.66, 1.97}, {32, 8, 32, 0.852, 0.780, 6.0, 4.2}};
    static const PromptForm wide128[kPromptForms] = {{256, 1, 64, 1.67, 1.50, 8.0, 6.6}, {128, 1, 64, 0.860, 1.138, 7.1, 3.3},
                                                     {128, 2, 64, 1.908, 1.650, 8.1, 5.8}, {64, 2, 64, 1.476, 1.371, 6.3, 5.1}};
    return head_dim == 64 ? wide64 : wide128;
}

inline double prompt_estimate(const PromptForm &f, int G, int Hkv, int n_seq, double n_q, double n_k, int units)
{
    const double mean = n_q / n_seq, before = std::max(0.0, (n_k - n_q) / n_seq);
    const double part[3] = {0.25, 0.75, 2.0};
    double steps = 0.0, blocks = 0.0, longest = 0.0;
    for (int i = 0; i < 3; ++i) {
        const double len = std::max(1.0, n_seq == 1 ? mean : mean * part[i]), nb = std::ceil(len * G / f.rows);
        const double tiles = (before + len * (nb + 1.0) / (2.0 * nb)) / f.keys + 0.5;        // of the mean block
        const double each = std::max(1.0, tiles / f.groups + (f.groups > 1 ? 0.5 : 0.0));
        steps += n_seq / 3.0 * nb * each;
        blocks += n_seq / 3.0 * nb;
        longest = std::max(longest, std::ceil(std::ceil((before + len) / f.keys) / f.groups));
    }
    const double full = (steps * f.rate + blocks * f.block) * Hkv / units, alone = longest * f.alone;
    return f.start + std::cbrt(full * full * full + alone * alone * alone);
}

// Index of the form in prompt_forms(head_dim).
inline int prompt_choose(int head_dim, int G, int Hkv, int n_seq, int n_q, int n_k, int units)
{
    const PromptForm *forms = prompt_forms(head_dim);
    int best = 0;
    double least = 0.0;
    for (int i = 0; i < kPromptForms; ++i) {
        const double t = prompt_estimate(forms[i], G, Hkv, n_seq, n_q, n_k, units);
        if (i == 0 || t < least) { best = i; least = t; }
    }
    return best;
}

}  // namespace reform
