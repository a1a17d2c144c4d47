// The choice of the form that window prompts take (window_plan.h), compiled for the host.
#include "window_plan.h"

using namespace reform;

extern "C" int plan_form(int head_dim, int G, int Hkv, int n_seq, int n_q, int n_k, int window, int n_sink, int units, int *rows, int *groups)
{
    const int i = window_choose(head_dim, G, Hkv, n_seq, n_q, n_k, window, n_sink, units);
    const PromptForm &f = window_forms(head_dim)[i];
    *rows = f.rows;
    *groups = f.groups;
    return i;
}

extern "C" double plan_estimate(int form, int head_dim, int G, int Hkv, int n_seq, int n_q, int n_k, int window, int n_sink, int units)
{
    return window_estimate(window_forms(head_dim)[form], G, Hkv, n_seq, n_q, n_k, window, n_sink, units);
}
