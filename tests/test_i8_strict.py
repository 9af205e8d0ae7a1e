"""The checks themselves, on the CPU: a planted mistake is found."""
import pytest
import torch

import i8_strict


@pytest.fixture()
def problem():
    g = torch.Generator().manual_seed(1)
    x, w = torch.randint(-127, 128, (6, 40), generator=g, dtype=torch.int8), torch.randint(-127, 128, (9, 40), generator=g, dtype=torch.int8)
    sx, sw = torch.rand(6, generator=g) + 0.1, torch.rand(9, generator=g) + 0.1
    out = (x.double() @ w.double().t()).float() * sx[:, None] * sw
    return out, x, sx, w, sw


def test_a_right_product_passes(problem):
    i8_strict.product(*problem)
    out, x, sx, w, sw = problem
    i8_strict.product(out.bfloat16(), x, sx, w, sw)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), 0.0])
def test_one_wrong_element_is_found(problem, value):
    out, *rest = problem
    out[3, 4] = value
    with pytest.raises(AssertionError):
        i8_strict.product(out, *rest)


def test_nothing_but_nan_is_found(problem):
    out, *rest = problem
    with pytest.raises(AssertionError):
        i8_strict.product(out * float("nan"), *rest)


def test_one_step_too_many_is_found(problem):
    out, *rest = problem
    with pytest.raises(AssertionError):
        i8_strict.product(out * (1 + 2.0 ** -21), *rest)
