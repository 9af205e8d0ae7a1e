"""int8 caches whose rows of V differ in size by many powers of two: what a row weighs does not depend on how large it is."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged_attention import Problem, _rand
from test_gpu_paged_scales import _written

pytestmark = pytest.mark.gpu

ZEROS = 2.0 ** -100 / 127           # the scale that append gives a row of zeros


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def test_a_few_large_rows(cats):
    """One row in a hundred is large: it is most of the sum, and the rest does not become NaN."""
    p = Problem(cats, [5000], 8, 2, 128, 16, "i8")
    g = _rand(1)
    _written(p.cache.vs, torch.where(torch.rand(p.cache.vs.shape, generator=g, device="cuda") < 0.01, 1e36, 0.01))
    p.cache.v[:, :, :, ::7] = 0
    p.run()
    assert torch.isfinite(p.out).all() and (p.out[..., ::7] == 0).all()
    p.check()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("heads", [1, 12])
@pytest.mark.parametrize("ahead", [17, 20, 30])
@pytest.mark.parametrize("where", ["first", "last", "middle"])
@pytest.mark.parametrize("n", [131071, 3000])
def test_a_row_ahead_of_a_long_run_of_zeros(cats, n, where, ahead, heads, page):
    """One row with values of V, `ahead` powers of two before all others, whose V is zero: they weigh (n - 1) 2^-ahead beside it, in every tile, warp and block."""
    p = Problem(cats, [n], heads, 1, 128, page, "i8")
    one = {"first": 0, "last": n - 1, "middle": n // 2}[where]
    at = p.table[0, one // page].long(), one % page
    p.cache.k.zero_()
    p.cache.v.zero_()
    _written(p.cache.vs, ZEROS)
    _written(p.cache.ks, 1.0)
    p.q.zero_()
    p.q[:, :, 0] = 1.0
    p.cache.k[at] = 1
    p.cache.v[at] = 100
    p.cache.vs[at] = 1.0
    p.run(ahead * 0.6931471805599453)
    share = 1 / (1 + (n - 1) * 2.0 ** -ahead)
    assert ((p.out.double() / (100 * share) - 1).abs() <= 2.0 ** -8 + 2.0 ** -10).all(), (p.out.double() / (100 * share)).min().item()
    p.check()


@pytest.mark.parametrize("value", [1e-25, 1e-5, 1e30])
def test_rows_of_zeros_beside_rows_of_any_size(cats, value):
    """Half of the rows are zeros (as append holds them): they take half of the weight."""
    p = Problem(cats, [4000, 70], 6, 2, 64, 16, "i8")
    g = _rand(4)
    none = torch.rand(p.cache.vs.shape, generator=g, device="cuda") < 0.5
    p.cache.v[none] = 0
    _written(p.cache.vs, torch.where(none, ZEROS, value))
    p.run()
    p.check()


@pytest.mark.parametrize("score", [1.0, 1e6, 3e9, -3e9, 1e30])
def test_equal_scores_of_any_size(cats, score):
    """The mean of rows whose scales of V lie apart, however large the one score that all of them have."""
    n = 700
    p = Problem(cats, [n], 2, 1, 64, 16, "i8")
    p.cache.k.zero_()
    p.cache.k[..., 0] = 1
    _written(p.cache.ks, 1.0)
    _written(p.cache.vs, 10.0 ** (torch.rand(p.cache.vs.shape, generator=_rand(5), device="cuda") * 6 - 3))
    p.q.zero_()
    p.q[:, :, 0] = 1.0
    p.run(score)
    at = torch.arange(n, device="cuda")
    at = ref.places(p.table, 16, torch.zeros_like(at), at)
    v = p.cache.rows("v", *at)[:, 0]
    off = (2.0 ** -11 + 2.0 ** -14) * v.abs().mean(0)             # the weights' rounding to fp16, the sums
    ref.check_bf16(p.out[0], v.mean(0).expand(2, -1), off.expand(2, -1))
    assert int(p.st.item()) == 0


@pytest.mark.parametrize("heads,kv,dim", [(3, 1, 128), (20, 1, 64)])
@pytest.mark.parametrize("scores", [60.0, -60.0, 3000.0])
@pytest.mark.parametrize("sizes", [0, 20, -20, 100, -100, "steps"])
def test_scores_and_sizes_along_a_sequence(cats, sizes, scores, heads, kv, dim):
    """Scores that rise or fall from row to row while the scales of V rise, fall or jump: references and exponents move both ways in every tile."""
    n = 2500
    p = Problem(cats, [n], heads, kv, dim, 16, "i8")
    g = _rand(6)
    at = torch.arange(n, device="cuda")
    x = at.double() / n - 0.5
    at = ref.places(p.table, 16, torch.zeros_like(at), at)
    p.cache.k.zero_()
    p.cache.k[..., 0] = 1
    p.q.zero_()
    p.q[:, :, 0] = 1.0
    p.cache.ks[at] = (scores * x + torch.rand(n, generator=g, device="cuda")).float()[:, None].expand(-1, kv)
    tens = torch.randint(-12, 13, (n,), generator=g, device="cuda").double() if sizes == "steps" else sizes * x * 0.6
    p.cache.vs[at] = (10.0 ** tens).float().clamp(1e-32, 1e32)[:, None].expand(-1, kv)
    p.run(1.0)
    p.check()


@pytest.mark.parametrize("heads", [1, 4, 5, 16])
@pytest.mark.parametrize("behind", [4, 12, 20, 24, 27, 28])
@pytest.mark.parametrize("by", ["score", "scale"])
def test_a_channel_that_the_largest_row_leaves_to_others(cats, by, behind, heads):
    """Channels in which the row with the largest weight is 0 show a row 2^-behind of it, to half a step of fp16 and the output's rounding."""
    p = Problem(cats, [300], heads, 1, 64, 16, "i8")
    p.cache.k.zero_()
    p.cache.v.zero_()
    p.q.zero_()
    p.q[:, :, 0] = 1.0
    _written(p.cache.ks, 1.0)
    _written(p.cache.vs, ZEROS)
    a, b = (p.table[0, 3].long(), 2), (p.table[0, 17].long(), 9)
    for at, score in ((a, 100), (b, 100 - (behind if by == "score" else 0))):
        p.cache.k[at] = score
        p.cache.vs[at] = 1.0
    p.cache.vs[b] = 1.0 if by == "score" else 2.0 ** -behind
    p.cache.v[a][..., ::2] = 90
    p.cache.v[b][..., 1::2] = 77
    p.run(0.6931471805599453)                       # scores are powers of two; all other rows are 2^-100 behind
    share = 1 / (1 + 2.0 ** -behind) if by == "score" else 0.5
    want = torch.zeros(heads, 64, dtype=torch.float64, device="cuda")
    want[:, ::2], want[:, 1::2] = 90 * share, 77 * share * 2.0 ** -behind
    assert ((p.out[0].double() / want - 1).abs() <= 2.0 ** -8 + 2.0 ** -11 + 2.0 ** -16).all(), (p.out[0, 0, :2].tolist(), want[0, :2].tolist())
    assert int(p.st.item()) == 0


@pytest.mark.parametrize("heads,dim", [(1, 128), (4, 64), (8, 128), (16, 64)])
@pytest.mark.parametrize("step", [100.0, 3e4, 1e6, 1e20])
def test_scores_far_apart(cats, step, heads, dim):
    """Scores that lie `step` apart, in any order: the largest row alone is left, whatever the scales of V are.  (The others weigh n e^-step of it at most, and
    their values are up to 127e4, which shows in channels where the largest row is 0.)"""
    lens = [257 + i for i in range(60)]
    p = Problem(cats, lens, heads, 1, dim, 16, "i8", seed=heads)
    g = _rand(8)
    p.cache.k.zero_()
    p.cache.k[..., 0] = 1
    p.q.zero_()
    p.q[:, :, 0] = 1.0
    _written(p.cache.vs, 10.0 ** (torch.rand(p.cache.vs.shape, generator=g, device="cuda") * 8 - 4))
    want = []
    for i, n in enumerate(lens):
        at = torch.arange(n, device="cuda")
        at = ref.places(p.table, 16, torch.full_like(at, i), at)
        rank = torch.randperm(n, generator=g, device="cuda")
        p.cache.ks[at] = (rank - n // 2).float()[:, None]
        last = rank.argmax()
        want.append(p.cache.rows("v", at[0][last], at[1][last]).float()[0])
    p.run(step)
    want = torch.stack(want).double()[:, None].expand(-1, heads, -1)
    ref.check_bf16(p.out, want, 2.0 ** -20 * want.abs() + 320 * 2.718281828459045 ** -min(step, 700.0) * 127e4)
    assert int(p.st.item()) == 0
