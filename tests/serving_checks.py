"""The checks of serving_reference.py with every number required to be one.  A comparison with NaN is false, so "no output is
further off than its bound" holds for outputs that are NaN, and for any output where the reference or its bound is."""
import math

import torch

import serving_reference as ref

_check_attention, _check_rotary = ref.check_attention, ref.check_rotary


def finite(t, what):
    wrong = ~torch.isfinite(t)
    assert not bool(wrong.any()), f"{what}: {int(wrong.sum())} of {t.numel()} not finite"


def check_attention(out, lse, want_out, want_lse, a, err, keys, dtype, what=""):
    for t, name in ((want_out, "reference"), (a, "bound"), (err, "bound"), (out, "outputs")):
        finite(t, f"{what} {name}")
    lse64 = lse.double().cpu()
    assert not bool(torch.isnan(want_lse).any()), f"{what}: reference lse"
    finite(lse64[want_lse != -math.inf], f"{what} lse of rows that see keys")
    _check_attention(out, lse, want_out, want_lse, a, err, keys, dtype, what)


def check_rotary(got, want, size, dtype, magnitude=1.0, what=""):
    for t, name in ((want, "reference"), (size, "bound"), (got, "outputs")):
        finite(t, f"{what} {name}")
    _check_rotary(got, want, size, dtype, magnitude, what)
