// Which form of the packed prompts' attention a batch takes (attend_prompt.hip).  Host code without device types.
//
// The lengths are on the device; the host knows the rows of the whole batch and the number of sequences.  It takes a
// quarter, three quarters and twice the mean length for a third of the sequences each, and estimates every form's
// time in microseconds: what all blocks' steps take at the rate of the whole chip, and what the longest block takes by
// itself.  A step is one key tile of each of the form's groups of waves.
//
// The constants were fitted to measurements of 370 batches (1 to 32000 rows, 1 to 50 sequences, 1 to 8 heads a group, with
// and without keys in front) in eight forms: error 6 to 15 % (root mean square), and the one of these four that is chosen takes 2 % more time in
// the mean than the best of the eight, at worst 47 %.  300 other batches, of up to 18000 rows, against the best of the four: 2.7 % in the mean, at worst
// 90 % (50 sequences of together 511 rows behind 3000 keys each, 28/4 heads of 128: 118 us, in blocks of 128 62).  (256 rows at head_dim 128, 64 by two groups, 32 by eight and 16 by four add nothing; without the last two forms
// it is 4 % at head_dim 64 and 16 % at 128.)  Measured, us, blocks of 256 / 128 / 128 with two groups (head_dim 128) / 32 / 16:
//   head_dim 64: 32 prompts of together 14586 behind 500 keys each, 8/4 heads 60 / 46 / - / 71 / -, four of 2445, 3/1 17.5 / 14.3 / - / 9.3 / 11.5, one
//   row behind 3000 keys, 2/1 39 / 40 / - / 16 / 11.5, one of 32768, 32/8 4658 / 4799
//   head_dim 128: 50 of together 2859, 56/8 44 / 37 / 59 / 85 / -, one of 6673, 8/1 171 / 135 / 102 / 146 / 270, one of 2674, 4/4 69 / 53 / 43 / 27 / 34,
//   eight of together 75 behind 3000 keys each, 8/8 54 / 56 / - / 28 / 24, one of 16384, 32/8 1877 / 1884, of 32768 7769 / 7427
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
    static const PromptForm wide64[kPromptForms] = {{256, 1, 64, 1.13, 0.790, 6.30, 8.50}, {128, 1, 64, 0.592, 0.790, 5.20, 2.62},
                                                    {32, 4, 32, 0.382, 0.522, 5.54, 1.57}, {16, 8, 32, 0.812, 0.788, 3.30, 3.40}};
    static const PromptForm wide128[kPromptForms] = {{128, 1, 64, 0.900, 1.117, 6.43, 4.30}, {128, 2, 64, 2.030, 1.671, 7.17, 6.81},
                                                     {32, 4, 32, 0.748, 0.872, 6.78, 3.08}, {16, 8, 32, 1.465, 1.620, 3.66, 4.23}};
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

// Rows of a block where the keys of `items` items of `rows` rows (rows of a sequence times heads of a group) are shared out over the chip: the smallest
// of up to 64 that does not make a compute unit go through more than so many keys, with 400 for the time it takes to begin a block; else
// 128.  Blocks that take all rows read K and V least often, and are right where the chip is busy; where it is not, smaller ones are done
// sooner, being more.  (Fitted on drafted trees, tree.hip.)
inline int shared_rows(int head_dim, double rows, double keys, double items, int units)
{
    const double each = (keys + 400.0) * items / units;
    const bool narrow = head_dim == 64;
    auto few = [&](int R, double limit) { return rows <= R || std::ceil(rows / R) * each <= limit; };
    return few(16, narrow ? 1600.0 : 1300.0) ? 16 : few(32, narrow ? 1800.0 : 600.0) ? 32 : few(64, narrow ? 2000.0 : 1000.0) ? 64 : 128;
}

// Blocks whose keys are shared out (prompt_share.h): no block takes longer than its share, but all go through all of their sequence's
// tiles, and there is a second launch.
struct PromptShared {
    PromptForm form;
    int least;               // keys that a share has at least
    int workgroups;          // shares of a compute unit
};

// Rows of such a block where sharing out is faster than the best form, else 0; `shared`: how.
// Measured: 150 batches of 2 to 9000 rows, 1 to 50 sequences behind 500 to 16000 keys each, 0.89 of the whole forms' time in the mean, at worst 1.07 times
// it; the best of whole and all blocks 0.84, since the rule keeps some whole that blocks of 128 rows would finish sooner (16 sequences of together 435
// rows behind 16000 keys each, 8/1 heads of 128: 113 us, 67).  Three rows behind 16000 keys, 4/1 heads of 128 80.9 -> 18.5 us, four sequences of 16 rows behind 8000, 32/8 heads 52 -> 35; but eight of together 364 rows behind
// 16000, 56/8 heads 261 whole, 734 in blocks of 16 shared out: the rates here are 1.2 to 2.8 times those of the whole forms.
inline int prompt_share_rows(int head_dim, int G, int Hkv, int n_seq, int n_q, int n_k, int units, PromptShared &shared)
{
    static const PromptShared forms64[4] = {{{16, 4, 32, 0.53, 0.0, 12.0, 1.66}, 256, 2}, {{32, 4, 32, 0.84, 0.0, 12.0, 3.45}, 128, 2},
                                            {{64, 2, 64, 1.30, 0.0, 12.0, 5.2}, 128, 1}, {{128, 1, 64, 1.30, 0.0, 12.0, 5.7}, 128, 2}};
    static const PromptShared forms128[4] = {{{16, 8, 32, 1.76, 0.0, 12.0, 5.1}, 128, 1}, {{32, 8, 32, 4.1, 0.0, 12.0, 12.7}, 128, 1},
                                             {{64, 2, 64, 3.2, 0.0, 12.0, 11.2}, 128, 1}, {{128, 1, 64, 2.5, 0.0, 12.0, 12.0}, 128, 2}};
    const double keys = (double)n_k / n_seq, rows = std::ceil((n_seq > 1 ? 1.3 : 1.0) * n_q / n_seq) * G, items = (double)n_seq * Hkv;
    if (keys * (head_dim == 64 ? 0.788 : 1.62) < 256.0 * 2.5) return 0;              // a block's chain takes less than the second launch
    // sequences one to a lane, places counted in 32 bits, also where broken boundaries give all rows to every one of them
    if (n_seq > 64 || ((double)n_q * G / 16.0 + n_seq) * Hkv * ((double)n_k / 32.0 + 16.0) >= 33554432.0) return 0;
    const int R = shared_rows(head_dim, rows, keys, items, units);
    shared = (head_dim == 64 ? forms64 : forms128)[R == 16 ? 0 : R == 32 ? 1 : R == 64 ? 2 : 3];
    const PromptForm &f = shared.form;
    const double t = f.start + items * std::ceil(rows / R) / units * (keys / (f.keys * f.groups) * f.rate + f.block);
    const PromptForm *whole = prompt_forms(head_dim);
    for (int i = 0; i < kPromptForms; ++i)
        if (prompt_estimate(whole[i], G, Hkv, n_seq, n_q, n_k, units) <= t) return 0;
    return R;
}

}  // namespace reform
