// Whether a batch of packed prompts has its keys shared out, and in blocks of how many rows (prompt_plan.h), compiled for the host.
#include "prompt_plan.h"

using namespace reform;

// Rows of a block, 0: not shared out.  keys, groups: a tile's, and the groups of waves; least, workgroups: of PromptShared.
extern "C" int plan_share(int head_dim, int G, int Hkv, int n_seq, int n_q, int n_k, int units, int *keys, int *groups, int *least,
                          int *workgroups)
{
    PromptShared f = {{0, 0, 0, 0.0, 0.0, 0.0, 0.0}, 0, 0};
    const int rows = prompt_share_rows(head_dim, G, Hkv, n_seq, n_q, n_k, units, f);
    *keys = f.form.keys;
    *groups = f.form.groups;
    *least = f.least;
    *workgroups = f.workgroups;
    return rows;
}
