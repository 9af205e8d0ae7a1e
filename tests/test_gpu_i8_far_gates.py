"""cats_swiglu_i8 where the gate's sigmoid is below the smallest normal number but the product with the up value is not."""
import pytest
import torch

import i8_reference as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _error(gate):
    """Relative error of the kernel's fp32 y.  e^g as the square of 2^(g log2(e) / 2): the constant and its product are off by u each,
    so the exponent by 2 u of |g| / 2 in units of e, twice; two 2^x off by 2^-22 = 4 u each, and three products: (2 |g| + 11) u.
    Gates near zero, with one 2^x and a reciprocal, are below the same bound."""
    return (2 * gate.double().abs().max().item() + 11) * U


def _check(cats, gate, up):
    x = torch.cat([gate, up], 1)
    q, scale = cats.new_i8(*gate.shape)
    cats.cats_swiglu_i8(x, q, scale)
    y = ref.swiglu(x)
    ref.check_held(q, scale, y, _error(gate))
    return q, y


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [64, 1000, 4096, 5001, 11008, 20000])
def test_rows_of_far_gates(cats, cols, kind):
    """One gate per row, from where the sigmoid is still a normal number to where the largest up value gives 2^-54."""
    g = torch.Generator(device="cuda").manual_seed(1)
    gate = torch.tensor([-70.0, -79.5, -80.5, -87.0, -88.0, -89.5, -95.0, -103.0, -110.0, -126.0], device="cuda")[:, None].expand(-1, cols)
    up = (torch.rand(10, cols, generator=g, device="cuda") * 2 - 1) * 3e38
    q, y = _check(cats, gate.to(kind), up.to(kind))
    assert (q.abs().amax(1) == 127).all()


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [64, 1000, 4096, 5001])
def test_far_gates_among_others(cats, cols, kind):
    """Ordinary gates and up values; single far gates whose large up values bring them among the row's largest results."""
    g = torch.Generator(device="cuda").manual_seed(2)
    gate, up = torch.randn(30, cols, generator=g, device="cuda"), torch.randn(30, cols, generator=g, device="cuda")
    for r in range(30):
        c = r * 37 % cols
        gate[r, c], up[r, c] = -88.0 - r * 0.1, 3e38 * (-1) ** r
    q, y = _check(cats, gate.to(kind), up.to(kind))
    want = ref.held(y)[1]
    assert all(abs(want[r, r * 37 % cols].item()) > 1 and q[r, r * 37 % cols] != 0 for r in range(30))


def test_gates_beyond_any_up_value(cats):
    """silu(g) u with g down to the lowest finite value is zero for every finite u; an infinite gate or up value is not a number."""
    low = torch.finfo(torch.float32).min
    gate = torch.tensor([-400.0, -1e4, -1e30, low, -float("inf"), -90.0], device="cuda")[:, None].repeat(1, 96)
    up = torch.full((6, 96), 3e38, device="cuda")
    up[5, 3] = float("inf")
    q, scale = cats.new_i8(6, 96)
    cats.cats_swiglu_i8(torch.cat([gate, up], 1), q, scale)
    assert (q == 0).all()
    assert (scale[:4].double() == torch.tensor(2.0 ** -100 / 127).float().item()).all() and torch.isnan(scale[4:]).all()
