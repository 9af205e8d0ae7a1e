"""Attention of one new token over the paged cache against the plain form in 64 bits."""
import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _rand(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Problem:
    """Sequences of the given lengths; every row of the cache that belongs to none of them holds NaN (int8: a NaN scale)."""

    def __init__(self, cats, lens, heads, kv, dim, page, kind, order="heads", seed=0, spare=2, pad=0):
        self.cats, self.lens, self.heads, self.dim, self.page = cats, lens, heads, dim, page
        g = _rand(seed + sum(lens))
        n_pages = sum(-(-n // page) for n in lens) + spare
        self.cache = ref.Cache(cats, n_pages, page, kv, dim, kind, order, pad)
        self.table = ref.table_for(g, lens, page, n_pages)
        for i, n in enumerate(lens):
            at = torch.arange(n, device="cuda")
            self.cache.fill(g, *ref.places(self.table, page, torch.full_like(at, i), at))
        self.q = torch.randn(len(lens), heads, dim, generator=g, device="cuda").bfloat16()
        self.len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.out = torch.full_like(self.q, 9.0)
        self.ws = cats.new_workspace_paged(max(1, len(lens)), heads, kv, dim)
        self.st = cats.new_status()

    def run(self, scale=None, out=None):
        self.scale = self.dim ** -0.5 if scale is None else scale
        out = self.out if out is None else out
        self.cats.cats_paged_attention(self.cache.dev, self.table, self.len, self.q, self.scale, out, self.ws, self.st)
        return out

    def check(self, out=None, only=None):
        out = self.out if out is None else out
        assert int(self.st.item()) == 0
        for i, n in enumerate(self.lens):
            if only is not None and i not in only:
                continue
            at = torch.arange(n, device="cuda")
            at = ref.places(self.table, self.page, torch.full_like(at, i), at)
            ref.check_attention(out[i], self.q[i], self.cache.rows("k", *at), self.cache.rows("v", *at), self.scale, self.cache.kind)


HEADS = [(1, 1), (4, 4), (6, 3), (32, 8), (5, 1), (7, 1), (8, 1), (9, 1), (16, 1), (34, 2), (33, 1), (64, 1)]


@pytest.mark.parametrize("heads,kv", HEADS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_groups_of_heads(cats, kind, dim, heads, kv):
    p = Problem(cats, [1, 40, 0, 777, 17], heads, kv, dim, 16, kind)
    p.run()
    p.check()
    assert (p.out[2] == 0).all()


@pytest.mark.parametrize("page", [1, 3, 16, 24, 100, 1024])
@pytest.mark.parametrize("order", ["heads", "rows"])
@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_pages_and_orders(cats, kind, order, page):
    """Pages that end inside a tile, ends on and off a page's end, rows behind the heads of another."""
    p = Problem(cats, [99, 100, 101, 1, 2, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 2049], 8, 2, 128, page, kind, order, pad=16)
    p.run()
    p.check()


@pytest.mark.parametrize("lens", [[1], [2], [513], [131071], [40000, 1], [5] * 300, [0] * 7, [0, 0, 30000], list(range(1, 200))])
@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_lengths(cats, kind, lens):
    p = Problem(cats, lens, 16, 4, 128, 64, kind)
    p.run()
    p.check()


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_many_heads_of_their_own(cats, kind):
    p = Problem(cats, [700, 1500, 33], 40, 40, 128, 24, kind)
    p.run()
    p.check()


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_strides_and_neighbours(cats, kind):
    """q and out are parts of wider rows; nothing around out is touched; rows behind the last sequence stay."""
    p = Problem(cats, [70, 0, 5000], 12, 4, 64, 16, kind)
    wide = torch.full((5, 12 * 64 + 40), 9.0, dtype=torch.bfloat16, device="cuda")
    qw = torch.full((3, 12 * 64 + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    qw[:, 8:8 + 768] = p.q.view(3, 768)
    out = wide[:3, 2:2 + 768]
    cats.cats_paged_attention(p.cache.dev, p.table, p.len, qw[:, 8:8 + 768], 64 ** -0.5, out, p.ws, p.st)
    p.scale = 64 ** -0.5
    p.check(out.reshape(3, 12, 64))
    assert (wide[3:] == 9).all() and (wide[:, :2] == 9).all() and (wide[:, 770:] == 9).all()


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_scales_of_the_scores(cats, kind):
    """A large scale makes the softmax pick one row, zero the mean, a negative one the other end."""
    p = Problem(cats, [300, 4000, 1], 8, 2, 128, 16, kind)
    for scale in (0.0, -0.3, 2.0, 40.0):
        p.run(scale)
        p.check()


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_one_row_far_above_a_long_tail(cats, kind):
    """Half of the weight on one row, the rest spread over all others: the small ones must not be lost."""
    n = 60000
    p = Problem(cats, [n], 2, 1, 128, 64, kind)
    at = torch.arange(n, device="cuda")
    at = ref.places(p.table, 64, torch.zeros_like(at), at)
    if kind == "bf16":
        p.cache.k[at] = (p.cache.k[at].float() * 1e-3).bfloat16()
        p.cache.v[at] = (p.cache.v[at].float() * 0.01 + 1).bfloat16()
    else:
        p.cache.ks[at] = 1e-5
        p.cache.v[at] = torch.randint(100, 128, p.cache.v[at].shape, device="cuda", dtype=torch.int8)
    first = at[0][0], at[1][0]
    q = p.q[0, 0].float()
    key = (q / q.square().sum() * 11 * 128 ** 0.5).bfloat16()                       # a score of 11 = log(60000)
    if kind == "bf16":
        p.cache.k[first] = key
        p.cache.v[first] = -1
    else:
        step = key.float().abs().max() / 127
        p.cache.k[first], p.cache.ks[first] = (key.float() / step).round().to(torch.int8), step
        p.cache.v[first] = -100
    p.q[0, 1] = p.q[0, 0]
    p.run()
    p.check()


def test_scales_of_any_size(cats):
    """int8 rows whose scales lie far apart: tiny next to huge, zeros, and rows that weigh little but are large."""
    p = Problem(cats, [900, 64], 4, 2, 128, 16, "i8")
    g = _rand(3)
    p.cache.vs.copy_(torch.where(torch.isnan(p.cache.vs), p.cache.vs, 10.0 ** (torch.rand(p.cache.vs.shape, generator=g, device="cuda") * 40 - 30)))
    p.run()
    p.check()
    p.cache.vs.copy_(torch.where(torch.isnan(p.cache.vs), p.cache.vs, 2.0 ** -100 / 127))
    p.cache.ks.copy_(torch.where(torch.isnan(p.cache.ks), p.cache.ks, 0.0))
    p.run()
    p.check()


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_what_is_not_finite_stays_with_its_head(cats, kind):
    """A NaN or infinite row makes NaN of the heads that read it and touches no other."""
    p = Problem(cats, [200, 90], 8, 4, 64, 16, kind)
    at = p.table[0, 3].long(), 5                        # position 53 of sequence 0
    if kind == "i8":
        p.cache.ks[at[0], at[1], 1] = float("nan")
        p.cache.vs[at[0], at[1], 3] = float("nan")
    else:
        p.cache.k[at[0], at[1], 1, 7] = float("nan")
        p.cache.v[at[0], at[1], 3, :] = float("inf")
    p.run()
    assert torch.isnan(p.out[0, 2:4]).all() and torch.isfinite(p.out[0, [0, 1, 4, 5]]).all() and torch.isfinite(p.out[1]).all()
    assert (~torch.isfinite(p.out[0, 6:8])).all()
    p.check(only=[1])


def test_scores_of_minus_infinity(cats):
    """Rows whose score is -inf weigh nothing; if all are, the quotient 0 / 0 is NaN."""
    p = Problem(cats, [500, 40], 2, 1, 64, 16, "bf16")
    p.q[:] = p.q.abs()
    ninf = -float("inf")
    for i in range(2):
        for t in range(0, p.lens[i], 1 if i else 3):
            p.cache.k[p.table[i, t // 16].long(), t % 16] = ninf
    p.run()
    assert torch.isnan(p.out[1]).all()
    live = torch.tensor([t for t in range(500) if t % 3], device="cuda")
    at = ref.places(p.table, 16, torch.zeros_like(live), live)
    ref.check_attention(p.out[0], p.q[0], p.cache.rows("k", *at), p.cache.rows("v", *at), p.scale, "bf16")


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_bad_tables_are_reported(cats, kind):
    """Pages and lengths outside the tables: reported, nothing outside is read, the other sequences are right."""
    p = Problem(cats, [100, 300, 50], 4, 2, 64, 16, kind)
    for bad in (-1, p.cache.n_pages, 2 ** 31 - 1, -2 ** 31):
        good = p.table.clone()
        p.table[1, 7] = bad
        p.run()
        assert int(p.st.item()) == -1
        p.st.zero_()
        p.table.copy_(good)
        p.check(only=[0, 2])
    p.len[1] = 2 ** 31 - 1
    p.table[1] = p.table[1, 0]
    p.run()
    assert int(p.st.item()) == -1
    p.st.zero_()
    p.check(only=[0, 2])
    p.len[1] = -3
    p.run()
    assert int(p.st.item()) == 0 and (p.out[1] == 0).all()


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_offsets_past_32_bits(cats, kind):
    """A cache of more than 2^32 elements whose last pages are read."""
    n_pages = 2 ** 32 // (256 * 16 * 128) + 3
    cache = ref.Cache(cats, n_pages, 256, 16, 128, kind, fill=0)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, -1]], dtype=torch.int32, device="cuda")
    g, n = _rand(4), 700
    pos = torch.arange(n, device="cuda")
    at = ref.places(table, 256, torch.zeros_like(pos), pos)
    cache.fill(g, *at)
    q = torch.randn(1, 16, 128, generator=g, device="cuda").bfloat16()
    out, st = torch.empty_like(q), cats.new_status()
    cats.cats_paged_attention(cache.dev, table, torch.tensor([n], dtype=torch.int32, device="cuda"), q, 0.1, out,
                              cats.new_workspace_paged(1, 16, 16, 128), st)
    ref.check_attention(out[0], q[0], cache.rows("k", *at), cache.rows("v", *at), 0.1, kind)
    assert int(st.item()) == 0


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_same_bits_every_time(cats, kind):
    """Again and again on one workspace, between calls of other sizes, without a synchronisation."""
    p = Problem(cats, [3000, 1, 20000, 700, 0, 64], 16, 4, 128, 16, kind, seed=1)
    small = Problem(cats, [9, 2000], 16, 4, 128, 16, kind, seed=2)
    small.ws = p.ws
    first, first_small = p.run().clone(), small.run().clone()
    p.check()
    small.check()
    outs = [(torch.empty_like(first), torch.empty_like(first_small)) for _ in range(20)]
    for a, b in outs:
        p.run(out=a)
        small.run(out=b)
    torch.cuda.synchronize()
    assert all(torch.equal(a, first) and torch.equal(b, first_small) for a, b in outs)


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_captured_and_replayed(cats, kind):
    """Lengths, pages and queries are read when the graph runs: it is replayed while the sequences grow."""
    p = Problem(cats, [2000, 500, 64], 8, 2, 128, 16, kind)
    full = list(p.lens)
    p.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    for lens in ([1, 0, 64], [1999, 17, 1], full):
        p.len.copy_(torch.tensor(lens, dtype=torch.int32))
        p.q.normal_()
        graph.replay()
        p.lens = lens
        p.check()


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_streams(cats, kind):
    """Two streams with a workspace each, at the same time."""
    ps = [Problem(cats, [9000 + i, 3, 400], 8, 2, 128, 16, kind, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(10):
        for p, s in zip(ps, streams):
            with torch.cuda.stream(s):
                p.run()
    torch.cuda.synchronize()
    for p in ps:
        p.check()
