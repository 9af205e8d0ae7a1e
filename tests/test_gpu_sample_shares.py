"""Cuts that one unit of 2^-44 of the largest weight decides."""
import math

import pytest
import torch

from test_gpu_sample import draw

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


@pytest.mark.parametrize("vocab", [3000, 60000, 200000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_unit_more_than_half(cats, vocab, dtype):
    """1024 equal tokens, and with them none or some that weigh one unit each: half of 2^54 + k units takes 512 tokens, and one more if k > 0."""
    unit = float(torch.tensor(-44 * math.log(2)).to(dtype))                  # rounds to one unit: 2^-44 to within a twentieth
    assert 0.6 < 2.0 ** 44 * math.exp(unit) < 1.4
    for extra in (0, 1, 2, 3, 100):
        x = torch.full((6, vocab), -INF)
        x[:, 5:5 + 1024] = 0.0
        x[:, 1500:1500 + extra] = unit
        want = 5 + 512 + (1 if extra else 0) - 1
        k = [0, 2 ** 30, 1024 + extra, 0, 0, 2000]
        token, prob = draw(cats, x.to(dtype).cuda(), [1.0] * 6, k=k, p=[0.5] * 6)
        assert token == [want] * 6 and all(abs(v * (want - 4) - 1) < 1e-6 for v in prob), (extra, token)


def test_the_random_number_times_an_odd_sum(cats):
    """u = 1/2 of 2^54 + k units: the sum up to the 512th token is 2^53, which exceeds it for no k."""
    for extra in (0, 1, 2, 100):
        x = torch.full((1, 5000), -INF)
        x[:, :1024] = 0.0
        x[:, 2000:2000 + extra] = -44 * math.log(2)
        token, _ = draw(cats, x.cuda(), [0.5])
        assert token == [512]
        x = x.flip(1)                                                        # the small ones in front: they count towards the half
        token, _ = draw(cats, x.cuda(), [0.5])
        assert token == [5000 - 1024 + (511 if extra else 512)], extra
