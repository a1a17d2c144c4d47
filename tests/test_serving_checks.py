"""The strict checks of the serving calls reject what is not a number, wherever it stands, and accept what is right."""
import math

import pytest
import torch

import serving_checks as checks
import serving_reference as ref

BAD = [math.nan, math.inf, -math.inf]


def attention(dtype):
    g = torch.Generator().manual_seed(1)
    q, k, v = (ref.randn(g, 2, n, 16, dtype=dtype) for n in (5, 4, 4))        # the first row sees no key
    want = ref.prompt_attend(q, k, v, [5], [4], 0.25)
    return want[0].to(dtype), want[1].float(), *want


def rotary(dtype):
    g = torch.Generator().manual_seed(2)
    x, pos = ref.randn(g, 2, 5, 16, dtype=dtype), torch.arange(5)
    want, size = ref.rotary(x, pos, 8, ref.frequencies(8, 1e4))
    return want.to(dtype), want, size


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_right_results_pass(dtype):
    checks.check_attention(*attention(dtype), 4, dtype)
    checks.check_rotary(*rotary(dtype), dtype)


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("everywhere", [True, False])
@pytest.mark.parametrize("which", ["out", "lse"])
def test_attention_that_is_no_number_is_rejected(which, everywhere, bad):
    out, lse, *want = attention(torch.float32)
    held = out if which == "out" else lse
    if everywhere:
        held.fill_(bad)
    else:
        held[1, 3] = bad
    with pytest.raises(AssertionError):
        checks.check_attention(out, lse, *want, 4, torch.float32)


def test_rows_that_see_nothing_have_minus_infinity_and_nothing_else():
    for bad in (math.nan, math.inf, 0.0):
        out, lse, *want = attention(torch.float32)
        assert bool((lse[:, 0] == -math.inf).all())
        lse[0, 0] = bad
        with pytest.raises(AssertionError):
            checks.check_attention(out, lse, *want, 4, torch.float32)


@pytest.mark.parametrize("at", range(4))
def test_a_reference_that_is_no_number_is_rejected(at):
    """Rows that the reference left out (it marks them by NaN) would be compared with nothing."""
    out, lse, *want = attention(torch.float32)
    want[at][1, 3] = math.nan
    with pytest.raises(AssertionError):
        checks.check_attention(out, lse, *want, 4, torch.float32)


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("everywhere", [True, False])
def test_rotations_that_are_no_numbers_are_rejected(everywhere, bad):
    for at in range(3):
        held = list(rotary(torch.float32))
        if everywhere:
            held[at].fill_(bad)
        else:
            held[at][1, 2, 15 if at < 2 else 3] = bad                          # element 15 is copied, not rotated
        with pytest.raises(AssertionError):
            checks.check_rotary(*held, torch.float32)
