"""Shares of a sum of weights, to the last digit: top_p of it rounded up, the random number times it rounded down.  On the CPU; the kernel runs the same code."""
import ctypes as C
import random
from fractions import Fraction

import numpy as np
import pytest


@pytest.fixture(scope="module")
def part():
    from paper_2605_11186_b200 import binding
    f = binding.lib.cats_debug_sample_part
    f.restype, f.argtypes = C.c_int64, [C.c_float, C.c_int64, C.c_int]
    return f


def _check(part, x, n):
    x = float(np.float32(x))
    exact = Fraction(x) * n
    assert part(x, n, 0) == exact.__floor__() and part(x, n, 1) == exact.__ceil__(), (x, n)


def test_every_digit(part):
    rng = random.Random(1)
    ends = [0.0, float(np.float32(1e-45)), 1e-40, 2.0 ** -126, 2.0 ** -64, 2.0 ** -24, 0.25, 0.5, 0.9, 1 - 2.0 ** -24]
    sums = [0, 1, 2, 3, 2 ** 24 + 1, 2 ** 44, 2 ** 53 + 1, 2 ** 54 + 1, 2 ** 62 - 1, 2 ** 62 - 2 ** 44 + 5]
    for x in ends + [rng.random() for _ in range(300)] + [2.0 ** rng.uniform(-149, 0) * 0.999 for _ in range(300)]:
        for n in sums + [rng.getrandbits(rng.randint(1, 62)) for _ in range(20)]:
            _check(part, x, n)


def test_a_sum_that_fp64_does_not_hold(part):
    """Half of 2^54 + 1: fp64 loses the one."""
    assert part(0.5, 2 ** 54 + 1, 1) == 2 ** 53 + 1 and part(0.5, 2 ** 54 + 1, 0) == 2 ** 53
