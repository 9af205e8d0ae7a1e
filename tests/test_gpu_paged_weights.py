"""The bits that a row's weight keeps over an int8 cache.

Queries of zeros make every score 0 and every probability the same power of two, so that the output is the mean of scale_v times the bytes: what is off is
the weights' rounding (two fp16 parts: 2^-22 each at most, 2^-21 of the mean of |v| here), the sums (as in paged_reference.attention_off), and
the last quotient and products.  The output is then rounded to bf16, which is monotone: it lies between what the two ends of that interval round to."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged_attention import HEADS, Problem, _rand
from test_gpu_paged_scales import _written

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


@pytest.mark.parametrize("heads,kv", HEADS + [(2, 1), (3, 1), (12, 3), (20, 5)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("spread", [1.0, 2.0 ** 10])
def test_means_to_the_last_bit_but_few(cats, spread, dim, heads, kv):
    p = Problem(cats, [1, 2, 7, 100, 1000, 5000], heads, kv, dim, 16, "i8", seed=heads)
    p.q.zero_()
    _written(p.cache.vs, 0.01 * spread ** torch.rand(p.cache.vs.shape, generator=_rand(1), device="cuda") * (1 + torch.rand(p.cache.vs.shape, generator=_rand(2), device="cuda")))
    p.run()
    assert int(p.st.item()) == 0
    for i, n in enumerate(p.lens):
        at = torch.arange(n, device="cuda")
        at = ref.places(p.table, 16, torch.full_like(at, i), at)
        v = p.cache.rows("v", *at)
        off = (2.0 ** -21 + ((n / 64 + 64) * 2 * 2 + 8) * ref.U) * v.abs().mean(0)
        lo, hi = ((v.mean(0) + d).float().bfloat16().repeat_interleave(heads // kv, 0).float() for d in (-off, off))
        got = p.out[i].float()
        assert ((got >= lo) & (got <= hi)).all(), (n, int(((got < lo) | (got > hi)).sum()), got.numel())


def test_a_head_s_result_does_not_depend_on_its_group(cats):
    """The same query, alone and among up to sixteen heads of a group: the two ways of the two parts give the same to the sums' rounding."""
    outs = []
    for heads in (1, 2, 4, 5, 8, 9, 16):
        p = Problem(cats, [3000, 60], heads, 1, 128, 16, "i8", seed=3)
        p.q[:] = torch.randn(2, 1, 128, generator=_rand(7), device="cuda").bfloat16()
        p.run()
        p.check()
        assert all(torch.equal(p.out[:, h], p.out[:, 0]) for h in range(heads))
        outs.append(p.out[:, 0].float())
    for o in outs[1:]:
        assert ((o - outs[0]).abs() <= 2.0 ** -7 * outs[0].abs() + 1e-6).all() and (o == outs[0]).float().mean() > 0.98
