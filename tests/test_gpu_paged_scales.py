"""int8 caches whose scales are at the ends of what append writes: values of V up to 3e38."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged_attention import Problem, _rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _written(t, value):
    """Scales of rows that hold something; the others stay NaN."""
    t.copy_(torch.where(torch.isnan(t), t, value))


@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 128), (16, 1, 64)])
@pytest.mark.parametrize("scale", [2.0 ** 112, 2.0 ** 113, 1e35, 1e36])
def test_large_values(cats, scale, heads, kv, dim):
    """All rows large; bytes of zero among them, and a whole row of zeros."""
    p = Problem(cats, [900, 33, 20000], heads, kv, dim, 16, "i8")
    p.q.mul_(0.25)
    _written(p.cache.vs, scale)
    p.cache.v[p.table[0, 2].long(), 5] = 0
    p.run()
    assert torch.isfinite(p.out).all()
    p.check()


def test_what_append_writes(cats):
    """Rows of 3e38 through append, then attended to: equal rows come back as they are."""
    cache = ref.Cache(cats, 3, 16, 2, 64, "i8", fill=0)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    n = 40
    k, v = torch.randn(n, 2, 64, generator=_rand(2), device="cuda"), torch.zeros(n, 2, 64, device="cuda")
    v[:, 0, ::2], v[:, 1, 1::2] = 3e38, -3e38
    seq, pos, st = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda"), cats.new_status()
    cats.cats_paged_append(cache.dev, table, seq, pos, None, k, v, 10000.0, None, st)
    q = torch.randn(1, 4, 64, generator=_rand(3), device="cuda").bfloat16()
    out = torch.empty_like(q)
    cats.cats_paged_attention(cache.dev, table, torch.tensor([n], dtype=torch.int32, device="cuda"), q, 0.1, out, cats.new_workspace_paged(1, 4, 2, 64), st)
    at = ref.places(table, 16, seq, pos)
    assert torch.isfinite(out).all() and int(st.item()) == 0
    ref.check_attention(out[0], q[0], cache.rows("k", *at), cache.rows("v", *at), 0.1, "i8")
