"""Checks of the 8-bit product that fail on whatever is not a number: a comparison with NaN is false, so what is asked is that every
element IS within its bound, not that none is outside."""
import torch

import i8_reference as ref


def within(out, want):
    """Every element of `out` within the product's bound of fp64 `want`: the sums are exact; the conversion of the sum and two products
    round once each (3 u), and bf16 once more."""
    rel = 3.01 * ref.U if out.dtype == torch.float32 else 2.0 ** -8 * (1 + 2.0 ** -12)
    good = (out.double() - want).abs() <= rel * want.abs()
    assert good.all(), (int((~good).sum()), int((~torch.isfinite(out)).sum()))


def product(out, x, sx, w, sw):
    within(out, ref.linear(x, sx, w, sw))
