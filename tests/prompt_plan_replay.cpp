// The choice of the packed prompts' form (prompt_plan.h), compiled for the host.
#include "prompt_plan.h"

using namespace reform;

extern "C" int plan_form(int head_dim, int G, int Hkv, int n_seq, int n_q, int n_k, int units, int *rows, int *groups)
{
    const int i = prompt_choose(head_dim, G, Hkv, n_seq, n_q, n_k, units);
    const PromptForm &f = prompt_forms(head_dim)[i];
    *rows = f.rows;
    *groups = f.groups;
    return i;
}

extern "C" double plan_estimate(int form, int head_dim, int G, int Hkv, int n_seq, int n_q, int n_k, int units)
{
    return prompt_estimate(prompt_forms(head_dim)[form], G, Hkv, n_seq, n_q, n_k, units);
}
