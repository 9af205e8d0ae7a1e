"""The logit that min-p cuts at, against the definition in 60 digits: exp((x - top) / T), rounded to whole units of 2^-44, >= min_p.  On the CPU; the kernel runs the
same code."""
import math
import random
from decimal import Decimal, getcontext
from fractions import Fraction

import numpy as np
import pytest

getcontext().prec = 60
F32 = np.float32
LOWEST, TINY, BELOW_1 = float(np.finfo(F32).min), float(F32(1e-45)), float(F32(1) - F32(2.0 ** -24))


@pytest.fixture(scope="module")
def least():
    from paper_2605_11186_b200 import binding
    return binding.sample_least


def _check(least, top, t, m):
    """The result is the largest logit, or within what fp64 rounds of the threshold, and the fp32 number below it is not above."""
    top, t, m = float(F32(top)), float(F32(t)), float(F32(m))
    x = least(top, t, m)
    assert x <= top and x == float(F32(x)), (top, t, m, x)
    if m > 1:
        assert x == top
        return
    reach = (Decimal(math.ceil(Fraction(m) * 2 ** 44)) - Decimal(0.5)) / 2 ** 44
    at = Decimal(top) + Decimal(t) * reach.ln()
    # fp64: the logarithm and log2 e / T are rounded once or twice each, the difference and the product once
    off = 6 * Decimal(2) ** -53 * abs(Decimal(t) * reach.ln())
    if at - off <= Decimal(LOWEST):
        assert x == LOWEST or Decimal(x) - at <= off
        return
    assert Decimal(x) >= at - off, (top, t, m, x)
    below = float(np.nextafter(F32(x if x != 0 else 0.0), F32(-np.inf)))
    assert below == -np.inf or Decimal(below) <= at + off, (top, t, m, x)


TEMPERATURES = [TINY, 1e-40, 5e-39, 1e-30, 1e-3, 0.7, 1.0, 1.5, 1e4, 1e30, 3e38]
MIN_PS = [TINY, 1e-30, 1e-3, 0.05, 0.5, 0.9, 0.9999999, BELOW_1, 1.0, 7.0]


@pytest.mark.parametrize("top", [0.0, -0.0, TINY, -TINY, 3e-44, 1e-38, -1e-38, 1e-20, -1e-20, 2.0, -2.0, 17.25, -3e5, 3e38, -3e38, LOWEST])
def test_every_end_of_the_ranges(least, top):
    for t in TEMPERATURES:
        for m in MIN_PS:
            _check(least, top, t, m)


def test_thresholds_next_to_zero(least):
    """top + T ln min_p cancels: rows whose threshold is the nearest to 0 that fp32 has, and logits beside it."""
    rng = random.Random(1)
    for _ in range(400):
        t, m = float(F32(10 ** rng.uniform(-3, 3))), float(F32(10 ** rng.uniform(-4, -0.001)))
        top = F32(-t * np.log(m))
        for step in range(-2, 3):
            x = top
            for _ in range(abs(step)):
                x = np.nextafter(x, F32(np.sign(step) * np.inf))
            _check(least, x, t, m)


def test_a_sum_that_cancels_in_fp64(least):
    """A threshold nearer to 0 than fp64 tells from 0: the logits that it cannot tell apart are half of all there are."""
    best = None
    for k in range(1, 4000):            # min_p = 2^-k has an exact logarithm: top = k T ln 2
        t = F32(1) + F32(k) * F32(2.0 ** -23)
        exact = Decimal(float(t)) * Decimal(2).ln()
        top = F32(float(exact))
        d = abs(Decimal(float(top)) - exact)
        if best is None or d < best[0]:
            best = (d, float(top), float(t))
    assert best[0] < Decimal(2) ** -34
    _check(least, best[1], best[2], 0.5)


def test_any_row(least):
    rng = random.Random(2)
    for _ in range(3000):
        _check(least, rng.choice([-1, 1]) * 10 ** rng.uniform(-44, 38), 10 ** rng.uniform(-44, 38), 10 ** rng.uniform(-44, 0))


def test_no_min_p(least):
    for m in (0.0, -0.0, -1.0):
        assert least(3.0, 1.0, m) == -float("inf")
    inf = float("inf")
    assert least(3.0, inf, 0.3) == LOWEST and least(3.0, inf, 1.0) == LOWEST and least(3.0, inf, 1.5) == 3.0
