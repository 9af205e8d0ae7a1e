"""Infinities in V of a bf16 cache: a weight times an infinity is that infinity, two of either sign are NaN, as in the plain form."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged_attention import Problem

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 64), (8, 2, 128), (32, 2, 128), (12, 1, 64)])
@pytest.mark.parametrize("n", [1, 2, 17, 300, 20000])
def test_infinite_values(cats, n, heads, kv, dim):
    p = Problem(cats, [n, 40], heads, kv, dim, 16, "bf16", seed=dim)
    rows = sorted({0, n // 3, n // 2, n - 1})
    for i, t in enumerate(rows):
        v = p.cache.v[p.table[0, t // 16].long(), t % 16]        # [kv][dim]
        v[0, 3 + 8 * i] = INF
        v[kv - 1, 4 + 8 * i] = -INF
        v[:, 50] = INF if i % 2 == 0 else -INF                   # one sign alone with one row, both with more
        v[0, 51] = NAN if i == 0 else INF
        v[:, 60] = 3.3e38 if i == 0 else -1.0                    # the largest numbers stay numbers
    p.run()
    assert int(p.st.item()) == 0
    p.check(only=[1])
    at = torch.arange(n, device="cuda")
    at = ref.places(p.table, 16, torch.zeros_like(at), at)
    k, v = p.cache.rows("k", *at), p.cache.rows("v", *at)
    want, _, _, _ = ref.attention(p.q[0], k, v, p.scale)
    got = p.out[0].double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isinf(got), torch.isinf(want)) and torch.equal(got[torch.isinf(want)], want[torch.isinf(want)])
    # finite channels: as without the others
    some = torch.isfinite(v).all(0)
    v = torch.where(some[None], v, 0.0)
    mask = some.repeat_interleave(heads // kv, 0)
    p.out[0][~mask] = 0
    ref.check_attention(p.out[0], p.q[0], k, v, p.scale, "bf16")


def test_every_row_infinite(cats):
    p = Problem(cats, [777], 8, 2, 64, 24, "bf16")
    p.cache.v[p.table[0, :33].long()] = -INF
    p.run()
    assert (p.out == -INF).all()
