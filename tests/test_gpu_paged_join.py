"""Parts of a head group that many blocks have, added in two steps: every head size and number of heads, half-filled warps among them."""
import pytest
import torch

from test_gpu_paged_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


@pytest.mark.parametrize("heads", [1, 3, 7, 8, 9, 13, 16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_parts_of_every_block(cats, kind, dim, heads):
    """One key head, so that every block has a part of it; the sums of the first step lie where their first parts lay.  The same bits each time."""
    p = Problem(cats, [70001], heads, 1, dim, 64, kind, seed=heads)
    first = p.run().clone()
    p.check()
    outs = [torch.empty_like(first) for _ in range(10)]
    for out in outs:
        p.run(out=out)
    assert all(torch.equal(out, first) for out in outs)


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_parts_of_several_groups(cats, kind):
    """Groups that share their first and last blocks with others."""
    p = Problem(cats, [30000, 50, 41000, 1], 14, 2, 64, 16, kind, seed=2)
    p.run()
    p.check()
