"""Rows into and out of the paged cache against their plain forms in 64 bits."""
import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BASE = 10000.0


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _rand(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _inputs(g, rows, heads, kv, dim, dtype, shift=0):
    """q, k, v: parts of the rows of one matrix, `shift` elements off the vector boundary."""
    wide = torch.randn(rows, (heads + 2 * kv) * dim + 24, generator=g, device="cuda").to(dtype)
    q, k, v = wide[:, shift:shift + (heads + 2 * kv) * dim].split([heads * dim, kv * dim, kv * dim], 1)
    return (q if heads else None), k, v


def _spread(n_seqs, rows):
    """(seq, pos): rows dealt out to the sequences in turn, every third position left free."""
    i = torch.arange(rows, device="cuda")
    seq = i % n_seqs
    pos = i // n_seqs
    return seq.int(), (pos + pos // 2).int()


def _state(cache):
    return [t.clone() for t in (cache.k, cache.v, cache.ks, cache.vs) if t is not None]


def _same(a, b):
    return torch.equal(a.float().nan_to_num(nan=3e38), b.float().nan_to_num(nan=3e38))


@pytest.mark.parametrize("order,pad", [("heads", 0), ("rows", 0), ("rows", 16)])
@pytest.mark.parametrize("heads,kv,dim,page,rows,shift", [(32, 32, 128, 64, 70, 0), (32, 8, 128, 16, 33, 0), (5, 5, 64, 1, 9, 1), (12, 4, 64, 24, 50, 3),
                                                            (0, 3, 128, 100, 7, 0), (64, 1, 64, 7, 64, 8), (40, 40, 128, 5, 11, 0), (130, 65, 128, 3, 4, 0)])
@pytest.mark.parametrize("kind", ["i8", "bf16"])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_append_and_read(cats, x, kind, heads, kv, dim, page, rows, shift, order, pad):
    g = _rand(heads * rows + shift)
    n_seqs = min(rows, 3)
    seq, pos = _spread(n_seqs, rows)
    longest = int(pos.max()) + 1
    cache = ref.Cache(cats, n_seqs * -(-longest // page) + 2, page, kv, dim, kind, order, pad)
    table = ref.table_for(g, [longest] * n_seqs, page, cache.n_pages)
    q, k, v = _inputs(g, rows, heads, kv, dim, TYPES[x], shift)
    before = _state(cache)
    st = cats.new_status()
    q_out = torch.full((rows, heads * dim + 8), 7.0, dtype=torch.bfloat16, device="cuda") if heads else None
    cats.cats_paged_append(cache.dev, table, seq, pos, q, k, v, BASE, q_out[:, :heads * dim] if heads else None, st)
    at = ref.places(table, page, seq, pos)
    yk, ok = ref.rotated(k, pos, BASE, dim)
    yv, ov = ref.rotated(v, pos, 0, dim)
    ref.check_cache(cache, "k", *at, yk, ok)
    ref.check_cache(cache, "v", *at, yv, ov)
    if heads:
        yq, oq = ref.rotated(q, pos, BASE, dim)
        ref.check_bf16(q_out[:, :heads * dim], yq, oq)
        assert (q_out[:, heads * dim:] == 7).all()
    # all other rows as they were
    for old, new in zip(before, _state(cache)):
        new[at] = old[at]
        assert _same(old, new)
    # and back: every type of output, rows off the vector boundary, in another order
    back = torch.randperm(rows, generator=g, device="cuda")
    at = at[0][back], at[1][back]
    for out_type in TYPES.values():
        for off in (0, 1):
            ko, vo = (torch.full((rows, kv * dim + 9), 3.0, dtype=out_type, device="cuda") for _ in range(2))
            cats.cats_paged_read(cache.dev, table, seq[back], pos[back], ko[:, off:off + kv * dim], vo[:, off:off + kv * dim], st)
            for out, name in ((ko, "k"), (vo, "v")):
                want = cache.rows(name, *at).float().to(out_type).view(rows, kv * dim)        # one rounding to fp32, one more to bf16
                assert torch.equal(out[:, off:off + kv * dim], want)
                assert (out[:, :off] == 3).all() and (out[:, off + kv * dim:] == 3).all()
    assert int(st.item()) == 0


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_sequence_i_is_row_i(cats, kind):
    """No list of sequences: row i goes to sequence i; three dimensions for the heads."""
    g = _rand(5)
    cache = ref.Cache(cats, 10, 4, 2, 64, kind)
    table = ref.table_for(g, [5, 9, 1, 16], 4, 10)
    pos = torch.tensor([4, 8, 0], dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(3, h, 64, generator=g, device="cuda") for h in (6, 2, 2))
    q_out = torch.empty(3, 6, 64, dtype=torch.bfloat16, device="cuda")
    st = cats.new_status()
    cats.cats_paged_append(cache.dev, table, None, pos, q, k, v, 500000.0, q_out, st)
    at = ref.places(table, 4, torch.arange(3, device="cuda"), pos)
    ref.check_cache(cache, "k", *at, *ref.rotated(k.flatten(1), pos, 500000.0, 64))
    ref.check_bf16(q_out, *ref.rotated(q.flatten(1), pos, 500000.0, 64))
    ko, vo = (torch.empty(3, 2, 64, device="cuda") for _ in range(2))
    cats.cats_paged_read(cache.dev, table, None, pos, ko, vo, st)
    assert torch.equal(ko, cache.rows("k", *at).float()) and torch.equal(vo, cache.rows("v", *at).float()) and int(st.item()) == 0


@pytest.mark.parametrize("base", [0.0, 10000.0, 1e6])
def test_far_positions(cats, base):
    """Positions up to 2^31 - 1: many table entries name one page."""
    g = _rand(6)
    page = 1 << 20
    cache = ref.Cache(cats, 1, page, 1, 64, "i8", "rows")
    table = torch.zeros(1, 2048, dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 1, 4095, 131070, 10 ** 6, 123456789, 2 ** 30 + 77, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    rows = pos.numel()
    q, k, v = _inputs(g, rows, 2, 1, 64, torch.float32)
    q_out = torch.empty(rows, 128, dtype=torch.bfloat16, device="cuda")
    st = cats.new_status()
    cats.cats_paged_append(cache.dev, table, torch.zeros(rows, dtype=torch.int32, device="cuda"), pos, q, k, v, base, q_out, st)
    at = torch.zeros(rows, dtype=torch.long, device="cuda"), pos.long() % page
    ref.check_cache(cache, "k", *at, *ref.rotated(k, pos, base, 64))
    ref.check_bf16(q_out, *ref.rotated(q, pos, base, 64))
    assert int(st.item()) == 0


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_rows_left_out_and_rows_outside(cats, kind):
    """A negative position leaves a row out; what is outside the tables is reported, and nothing is read or written there."""
    g = _rand(7)
    cache = ref.Cache(cats, 6, 4, 2, 64, kind)
    table = torch.tensor([[0, 1, -1, 6], [3, 4, 2 ** 30, 5]], dtype=torch.int32, device="cuda")
    good = [(0, 3), (1, 0), (0, 4)]
    left = [(0, -1), (1, -2 ** 31), (-5, -1), (9, -1)]
    bad = [(0, 8), (0, 12), (1, 8), (0, 16), (0, 2 ** 31 - 1), (2, 0), (-1, 0), (2 ** 31 - 1, 1)]
    for rows, wrong in ((good + left, False), (good + left + bad, True)):
        seq, pos = (torch.tensor(c, dtype=torch.int32, device="cuda") for c in zip(*rows))
        q, k, v = _inputs(g, len(rows), 2, 2, 64, torch.float32)
        q_out = torch.full((len(rows), 128), 5.0, dtype=torch.bfloat16, device="cuda")
        before, st = _state(cache), cats.new_status()
        cats.cats_paged_append(cache.dev, table, seq, pos, q, k, v, BASE, q_out, st)
        assert (int(st.item()) == -1) == wrong
        n = len(good)
        at = ref.places(table, 4, seq[:n], pos[:n])
        ref.check_cache(cache, "k", *at, *ref.rotated(k[:n], pos[:n], BASE, 64))
        assert (q_out[n:] == 5).all()
        for old, new in zip(before, _state(cache)):
            new[at] = old[at]
            assert _same(old, new)
        st.zero_()
        ko, vo = (torch.full((len(rows), 128), 5.0, device="cuda") for _ in range(2))
        cats.cats_paged_read(cache.dev, table, seq, pos, ko, vo, st)
        assert (int(st.item()) == -1) == wrong and (ko[n:] == 5).all() and (vo[n:] == 5).all()
        assert torch.equal(ko[:n], cache.rows("k", *at).float().view(n, 128))


def test_heads_of_zeros_tiny_and_not_finite(cats):
    g = _rand(8)
    cache = ref.Cache(cats, 2, 8, 3, 64, "i8")
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    x = torch.randn(8, 3, 64, generator=g, device="cuda")
    x[0, 0] = 0
    x[1, 1, 5] = float("inf")
    x[2, 2, 63] = float("nan")
    x[3, 0, 0] = -float("inf")
    x[4, 1] = 1e-40
    x[5, 2] = 3e38
    seq, pos = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.arange(8, dtype=torch.int32, device="cuda")
    st = cats.new_status()
    cats.cats_paged_append(cache.dev, table, seq, pos, None, x, x, 0.0, None, st)
    q, s = cache.v[1], cache.vs[1]                                            # pos is the row of page 1
    bad = torch.zeros(8, 3, dtype=torch.bool, device="cuda")
    bad[1, 1] = bad[2, 2] = bad[3, 0] = True
    assert torch.equal(torch.isnan(s), bad) and (q[bad] == 0).all()
    assert (q[0, 0] == 0).all() and (q[4, 1] == 0).all() and (q[5, 2] == 127).all()
    good = ~bad
    a, want = ref.i8.held(x.double()[good])
    assert ((q.double()[good] - want).abs() <= 0.5 + 127 * 4 * ref.U).all()
    ko, vo = (torch.empty(8, 192, device="cuda") for _ in range(2))
    cats.cats_paged_read(cache.dev, table, seq, pos, ko, vo, st)
    assert torch.equal(torch.isnan(ko.view(8, 3, 64)).all(2), bad) and torch.isfinite(ko.view(8, 3, 64)[good]).all() and int(st.item()) == 0


def test_a_contiguous_cache_is_one_page(cats):
    """The caches of the tree verification, [max_seq][heads * dim] bf16, through the same calls."""
    g = _rand(9)
    kc, vc = (torch.randn(50, 4, 64, generator=g, device="cuda").bfloat16() for _ in range(2))
    kv = cats.PagedKV(kc[None], vc[None])
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    seq, pos = torch.zeros(50, dtype=torch.int32, device="cuda"), torch.arange(50, dtype=torch.int32, device="cuda")
    ko, vo = torch.empty_like(kc), torch.empty_like(vc)
    st = cats.new_status()
    cats.cats_paged_read(kv, table, seq, pos, ko, vo, st)
    assert torch.equal(ko, kc) and torch.equal(vo, vc) and int(st.item()) == 0


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_offsets_past_32_bits(cats, kind):
    """The last page of K begins more than 2^32 elements behind the first."""
    g = _rand(10)
    n_pages = 2 ** 32 // (256 * 16 * 128) + 3
    cache = ref.Cache(cats, n_pages, 256, 16, 128, kind, fill=0)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 255, 256, 511, 512, 767], dtype=torch.int32, device="cuda")
    seq = torch.zeros_like(pos)
    q, k, v = _inputs(g, 6, 0, 16, 128, torch.bfloat16)
    st = cats.new_status()
    cats.cats_paged_append(cache.dev, table, seq, pos, None, k, v, BASE, None, st)
    at = ref.places(table, 256, seq, pos)
    ref.check_cache(cache, "k", *at, *ref.rotated(k, pos, BASE, 128))
    ref.check_cache(cache, "v", *at, *ref.rotated(v, pos, 0, 128))
    ko, vo = (torch.empty(6, 2048, device="cuda") for _ in range(2))
    cats.cats_paged_read(cache.dev, table, seq, pos, ko, vo, st)
    assert torch.equal(ko, cache.rows("k", *at).float().view(6, 2048)) and int(st.item()) == 0


def test_no_rows(cats):
    cache = ref.Cache(cats, 2, 8, 3, 64, "i8")
    table = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    x = torch.empty(0, 192, device="cuda")
    st = cats.new_status()
    cats.cats_paged_append(cache.dev, table, none, none, None, x, x, BASE, None, st)
    cats.cats_paged_read(cache.dev, table, none, none, x, x.clone(), st)
    assert cats.last_launch_count() == 0
