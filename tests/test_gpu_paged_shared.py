"""What calls of the paged attention share: a workspace between forms and captured graphs, pages between sequences, a table that is a part of another."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged_attention import Problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def test_one_workspace_for_every_form(cats):
    """Types, head sizes, groups of up to 8 and more heads, few and many sequences: eager, and as two captured graphs replayed in turn."""
    ps = [Problem(cats, lens, heads, kv, dim, 16, kind, seed=i) for i, (lens, heads, kv, dim, kind) in enumerate(
        [([30000], 8, 1, 128, "i8"), ([5000, 1, 300], 32, 2, 64, "bf16"), ([70] * 40, 16, 1, 128, "bf16"), ([9000, 9000], 8, 8, 64, "i8"), ([12000], 20, 1, 128, "i8")])]
    want = []
    for p in ps:
        want.append(p.run().clone())
        p.check()
    ws = max((p.ws for p in ps), key=lambda w: w.numel()).zero_()
    outs = [torch.empty_like(p.out) for p in ps]
    for p in ps:
        p.ws = ws
    for order in (range(5), range(4, -1, -1)):
        for i in order:
            ps[i].run(out=outs[i])
    assert all(torch.equal(o, w) for o, w in zip(outs, want))
    graphs = []
    for part in ((0, 1, 2), (3, 4)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            for i in part:
                ps[i].run(out=outs[i])
    for o in outs:
        o.fill_(5.0)
    for _ in range(10):
        for graph in graphs:
            graph.replay()
        ps[3].run()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want)) and torch.equal(ps[3].out, want[3])


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_sequences_that_share_pages(cats, kind):
    """A common beginning held once: three sequences with the same first pages, through a table that is the middle of a wider one."""
    p = Problem(cats, [1000], 16, 4, 128, 16, kind, seed=3)
    wide = torch.full((3, 100), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    table = wide[:, 20:20 + p.table.shape[1]]
    table.copy_(p.table.expand(3, -1))
    lens = [1000, 640, 17]
    q = torch.randn(3, 16, 128, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").bfloat16()
    out, st = torch.empty_like(q), cats.new_status()
    cats.cats_paged_attention(p.cache.dev, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), q, 0.1, out, cats.new_workspace_paged(3, 16, 4, 128), st)
    assert int(st.item()) == 0
    for i, n in enumerate(lens):
        at = torch.arange(n, device="cuda")
        at = ref.places(p.table, 16, torch.zeros_like(at), at)
        ref.check_attention(out[i], q[i], p.cache.rows("k", *at), p.cache.rows("v", *at), 0.1, kind)


def test_the_same_row_read_and_drawn_from_many_times(cats):
    """One cache row read into many output rows, one row of logits drawn from by many draws, on a stream that is not the current one's."""
    side = torch.cuda.Stream()
    p = Problem(cats, [50], 4, 4, 64, 16, "i8", seed=5)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        n = 300
        k, v = (torch.empty(n, 256, device="cuda") for _ in range(2))
        seq, pos, st = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.full((n,), 33, dtype=torch.int32, device="cuda"), cats.new_status()
        cats.cats_paged_read(p.cache.dev, p.table, seq, pos, k, v, st)
        x = torch.randn(2, 50001, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda")
        row, u = torch.ones(n, dtype=torch.int32, device="cuda"), torch.full((n,), 0.41, device="cuda")
        token, prob = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
        cats.cats_sample(x, row, None, None, torch.full((n,), 0.9, device="cuda"), None, u, token, prob, st)
    side.synchronize()
    assert int(st.item()) == 0
    for out in (k, v):
        assert torch.equal(out, out[:1].expand_as(out))
    at = ref.places(p.table, 16, torch.zeros(1, dtype=torch.long, device="cuda"), torch.tensor([33], device="cuda"))
    assert torch.equal(k[0].double(), p.cache.rows("k", *at).reshape(-1).float().double())
    want, share, near = ref.sample(x[1].double().cpu().numpy(), 1.0, 0, float(torch.tensor(0.9)), 0.0, float(torch.tensor(0.41)))
    assert near > 1e-9 and token.unique().tolist() == [want] and prob.unique().numel() == 1 and abs(float(prob[0]) - share) <= 3 * ref.U * share
