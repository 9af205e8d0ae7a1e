"""min-p at the ends of its range: thresholds next to 0 and next to the largest logit, rows whose largest is 0, any temperature."""
import numpy as np
import pytest
import torch

from test_gpu_sample import INF, check, draw, logits, uniform

pytestmark = pytest.mark.gpu

TEMPERATURES = [1e-45, 5e-39, 1e-30, 1e-3, 0.1, 1.0, 10.0, 1e4, 1e30, 3e38, INF]
MIN_PS = [0.05, 0.9, 1 - 2.0 ** -24]


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


@pytest.mark.parametrize("zero", [0.0, -0.0])
@pytest.mark.parametrize("vocab", [700, 40000, 140000])
def test_rows_whose_largest_is_zero(cats, vocab, zero):
    """Log-probabilities: nothing above 0, and 0 once, twice or at every tenth token."""
    n = len(TEMPERATURES)
    x = -logits(n, vocab, torch.float32, vocab).abs() - 0.01
    x[:, vocab // 3] = zero
    x[n // 3:, vocab // 2] = zero
    x[2 * n // 3:, ::10] = zero
    for m in MIN_PS:
        for k in (None, [50] * n, [5000] * n):
            check(cats, x, uniform(n, 1), t=TEMPERATURES, k=k, m=[m] * n)
        check(cats, x, uniform(n, 2), t=TEMPERATURES, p=[0.8] * n, m=[m] * n)


@pytest.mark.parametrize("vocab", [700, 70000])
def test_the_cut_is_where_the_host_finds_it(cats, vocab):
    """The last kept token of rows whose other logits are neighbours of the threshold, at or next to 0: logits from 8 steps above to 8 below it.
    The fp64 logarithms of host and device are each within one unit in the last place, 2^-52 relative, of the right one: log2 min_p, and with it the
    distance top - threshold = -T ln min_p, differs by at most 2^-51 of itself.  Logits that near the host's threshold may be cut or kept."""
    for t, m in [(1.0, 0.5), (0.7, 0.05), (1e-3, 0.9), (1e4, 0.3), (1e-40, 0.9999999), (1e-45, 0.9), (1e30, 0.2)]:
        t, m = float(np.float32(t)), float(np.float32(m))
        for top in (float(np.float32(-t * np.log(m))), 0.0, 3.0, -3.0 * min(t, 1e6)):
            top = float(np.float32(top))
            at = np.float32(cats.sample_least(top, t, m))
            near = [at]
            for _ in range(8):
                near.append(np.nextafter(near[-1], np.float32(-np.inf)))
            for _ in range(8):
                near.insert(0, min(np.nextafter(near[0], np.float32(np.inf)), np.float32(top)))
            row = torch.full((vocab,), -INF)
            places = torch.arange(len(near)) * (vocab // 20) + 2
            row[places] = torch.from_numpy(np.array(near, dtype=np.float32))
            row[0] = top
            x = row.cuda()[None].repeat(3, 1)
            off = -t * np.log(m) * 2.0 ** -51
            first, last = (max(int(i) for i, v in zip([0] + places.tolist(), [top] + near) if float(v) - float(at) >= d) for d in (min(off, top - float(at)), -off))
            for k in (None, [30] * 3):
                token, _ = draw(cats, x, [1.0, 0.0, 7.0], t=[t] * 3, k=k, m=[m] * 3)
                assert first <= token[0] <= last and token == [token[0], 0, token[0]], (t, m, top)


@pytest.mark.parametrize("vocab", [40, 50000])
def test_equal_weights_reach_a_min_p_of_one(cats, vocab):
    """At temperature inf, or one so large that all weights round to 1, min-p 1 keeps every token."""
    x = logits(6, vocab, torch.float32, 3)
    x[:, ::3] = -INF
    for k in (None, [20] * 6, [vocab] * 6):
        check(cats, x, uniform(6, 4), t=[INF, 1e30, 3e38, INF, 1e20, 1e25], k=k, m=[1.0] * 6)
        check(cats, x, uniform(6, 5), t=[INF, 1e30, 3e38, INF, 1e20, 1e25], k=k, p=[0.7] * 6, m=[1.0] * 6)


@pytest.mark.parametrize("vocab", [40, 50000, 200000])
def test_a_min_p_that_no_weight_reaches(cats, vocab):
    """The first of the order is left, also where others equal it."""
    x = logits(5, vocab, torch.bfloat16, 4)
    x[2] = 1.0
    x[3, ::7] = 30.0
    first = [int((r == r.max()).nonzero()[0]) for r in x]
    for t in (1.0, 0.0, INF, 1e-30):
        for m in (1 + 2.0 ** -23, 2.0, INF):
            for k in (None, [9] * 5):
                token, prob = draw(cats, x, [0.99, 1.0, 0.5, 1.0, 0.0], t=[t] * 5, k=k, p=[1.0, 0.9, 0.9, 1.0, 0.1], m=[m] * 5)
                assert token == first and prob == [1.0] * 5, (t, m)
