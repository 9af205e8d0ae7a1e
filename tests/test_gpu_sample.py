"""Drawing tokens against the plain form in 64 bits: the same token, unless the random number is nearer to another than fp64 tells."""
import numpy as np
import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _t(v, dtype=torch.float32):
    return None if v is None else torch.as_tensor(v, dtype=dtype, device="cuda").contiguous()


def draw(cats, x, u, t=None, k=None, p=None, m=None, row=None, status=0):
    """Lists or None for the settings."""
    u = _t(u)
    token, prob, st = torch.full((u.numel(),), -9, dtype=torch.int32, device="cuda"), torch.full((u.numel(),), -9.0, device="cuda"), cats.new_status()
    cats.cats_sample(x, _t(row, torch.int32), _t(t), _t(k, torch.int32), _t(p), _t(m), u, token, prob, st)
    assert int(st.item()) == status
    return token.cpu().tolist(), prob.cpu().tolist()


def check(cats, x, u, t=None, k=None, p=None, m=None, row=None):
    """The settings as fp32 holds them."""
    token, prob = draw(cats, x, u, t, k, p, m, row)
    n = len(token)
    f = [np.float32(v if v is not None else [d] * n).astype(np.float64) for v, d in ((t, 1), (p, 1), (m, 0), (u, 0))]
    x = x.double().cpu().numpy()
    sure = 0
    for i in range(n):
        want, share, near = ref.sample(x[i if row is None else row[i]], f[0][i], 0 if k is None else int(k[i]), f[1][i], f[2][i], f[3][i])
        if near < 1e-9:
            continue
        sure += 1
        assert token[i] == want, (i, token[i], want, near)
        assert abs(prob[i] - share) <= 2 * ref.U * share + 1e-9 * share, (prob[i], share)     # one rounding to fp32; sums cut at 2^-44 a token
    assert sure >= 0.9 * n
    return token


def logits(rows, vocab, dtype, seed, spread=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g, device="cuda") * spread).to(dtype)


def uniform(n, seed):
    return torch.rand(n, generator=torch.Generator().manual_seed(seed)).tolist()


VOCABS = [1, 2, 31, 33, 1000, 1023, 1025, 4099, 32000, 32001, 32768, 32769, 65537, 100003, 131073, 262144]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", VOCABS)
def test_settings(cats, vocab, dtype):
    """Every pair of filters in one call, each row with its own."""
    ks, ps, ms, ts = [0, 1, 2, 50, 1000, vocab, 2 ** 31 - 1], [1.0, 0.95, 0.5, 0.01, 0.0], [0.0, 0.05, 0.5, 1.0], [1.0, 0.3, 0.7, 2.0, 0.0]
    n = 40
    x = logits(n, vocab, dtype, vocab)
    pick = lambda v, step: [v[(i // step + i) % len(v)] for i in range(n)]      # noqa: E731
    check(cats, x, uniform(n, 1), pick(ts, 3), pick(ks, 5), pick(ps, 2), pick(ms, 7))


@pytest.mark.parametrize("which", ["none", "k", "p", "m"])
@pytest.mark.parametrize("rows", [1, 3, 150, 400])
def test_one_filter(cats, which, rows):
    x = logits(rows, 5000, torch.float32, rows)
    check(cats, x, uniform(rows, 2), k=[40] * rows if which == "k" else None, p=[0.9] * rows if which == "p" else None,
          m=[0.1] * rows if which == "m" else None)


@pytest.mark.parametrize("vocab", [700, 40000])
def test_ends_of_the_interval(cats, vocab):
    """u of 0, just below 1, 1 and past either end: the first and the last kept token."""
    x = logits(6, vocab, torch.float32, 3)
    us = [0.0, 1 - 2.0 ** -24, 1.0, 7.0, -1.0, INF]
    token, _ = draw(cats, x, us, k=[25] * 6)
    for i in range(6):
        kept = sorted(torch.sort(x[i], descending=True, stable=True)[1][:25].tolist())
        assert token[i] == (kept[0] if us[i] <= 0 else kept[-1])


@pytest.mark.parametrize("vocab", [64, 5000, 70000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_logits(cats, vocab, dtype):
    """Ties everywhere: the cut of top-k and top-p falls inside a run of equal logits and keeps the lowest indices."""
    same = torch.zeros(4, vocab, dtype=dtype, device="cuda")
    k = max(1, vocab // 3)
    token, prob = draw(cats, same, [0.0, 0.5, 1 - 2.0 ** -24, 0.25], k=[k] * 4)
    assert token == [0, k // 2, k - 1, k // 4] and all(abs(v * k - 1) <= 4 * ref.U for v in prob)
    token, _ = draw(cats, same, [1 - 2.0 ** -24] * 4, p=[0.5] * 4)
    assert token == [(vocab + 1) // 2 - 1] * 4
    coarse = (logits(4, vocab, torch.float32, 4, 1.0).round() / 2).to(dtype)
    check(cats, coarse, uniform(4, 5), k=[vocab // 2, 7, 1, vocab - 1], p=[0.7, 0.9, 1.0, 0.3])
    greedy, _ = draw(cats, coarse, [0.9] * 4, t=[0.0] * 4)
    assert greedy == [int((coarse[i] == coarse[i].max()).nonzero()[0]) for i in range(4)]


def test_signed_zeros_are_equal(cats):
    x = torch.tensor([[-1.0, -0.0, 0.0, -0.0, -5.0]], device="cuda")
    assert draw(cats, x, [0.5], t=[0.0])[0] == [1]
    assert draw(cats, x, [0.999], k=[2])[0] == [2]


@pytest.mark.parametrize("vocab", [90, 33000])
def test_masked_tokens(cats, vocab):
    """-inf weighs nothing and is never drawn, at any temperature; the type's lowest value likewise."""
    for hide in (-INF, float(torch.finfo(torch.float32).min)):
        x = logits(8, vocab, torch.float32, 6)
        x[:, ::2] = hide
        us = [0.0, 1 - 2.0 ** -24, 1.0] + uniform(5, 7)
        token, _ = draw(cats, x, us, t=[1.0, 1.0, 1.0, 5.0, 0.0, 0.1, 1.0, 1.0], k=[0, 0, vocab, 0, 0, 0, vocab - 1, 3])
        assert all(v % 2 == 1 for v in token)
    x[:, :] = -INF
    x[:, vocab // 2] = -3.0
    assert draw(cats, x, us, t=[INF] * 8)[0] == [vocab // 2] * 8
    only = torch.full((1, vocab), -INF, device="cuda")
    only[0, 3], only[0, vocab - 1] = 1.0, 2.0
    check(cats, only.repeat(3, 1), [0.1, 0.5, 0.9], t=[INF, 1.0, 3.0])


def test_any_temperature(cats):
    x = logits(9, 3001, torch.float32, 8)
    check(cats, x, uniform(9, 9), t=[1e-45, 1e-30, 1e-3, 0.1, 10.0, 1e4, 1e30, 3e38, INF])


def test_logits_of_any_size(cats):
    """Far apart, huge, tiny and subnormal."""
    for scale in (1e-42, 1e-20, 1e3, 1e30, 3e37):
        x = logits(4, 2500, torch.float32, 10, 1.0).clamp(-8, 8) * scale
        check(cats, x, uniform(4, 11), t=[1.0, scale, 0.5 * scale, 0.0], k=[0, 0, 100, 0], p=[1.0, 0.9, 1.0, 1.0])


def test_rows_by_number(cats):
    """Several draws from one row, rows out of order, draws left out."""
    x = logits(5, 2000, torch.bfloat16, 12)
    row = [4, 0, 0, 3, 0, 4, 1]
    check(cats, x, uniform(7, 13), t=[0.8] * 7, row=row)
    token, prob = draw(cats, x, [0.5] * 3, row=[-1, 2, -2 ** 31])
    assert token[0] == token[2] == -9 and prob[0] == -9 and token[1] >= 0
    token, prob = draw(cats, x, [0.5] * 3, row=[5, 2, 2 ** 31 - 1], status=-1)
    assert token[0] == token[2] == -1 and prob[0] == 0 and token[1] >= 0


@pytest.mark.parametrize("vocab", [77, 40001, 140000])
def test_rows_that_cannot_be_drawn_from(cats, vocab):
    x = logits(6, vocab, torch.float32, 14)
    good, _ = draw(cats, x, [0.3] * 6, p=[0.9] * 6)
    x[0, vocab - 1] = NAN
    x[1, 5] = INF
    x[2] = -INF
    x[4, 0] = -NAN
    token, prob = draw(cats, x, [0.3] * 6, p=[0.9] * 6, status=-1)
    assert [token[i] for i in (0, 1, 2, 4)] == [-1] * 4 and [prob[i] for i in (0, 1, 2, 4)] == [0.0] * 4
    assert token[3] == good[3] and token[5] == good[5]
    x = logits(6, vocab, torch.float32, 14)
    for bad in (dict(t=[NAN, 1, -1.0, 1, -INF, 1]), dict(p=[NAN, 1, NAN, 1, NAN, 1]), dict(m=[NAN, 0, NAN, 0, NAN, 0])):
        token, _ = draw(cats, x, [0.3] * 6, status=-1, **bad)
        assert [token[i] for i in (0, 2, 4)] == [-1] * 3 and min(token[1::2]) >= 0
    token, _ = draw(cats, x, [NAN, 0.3] * 3, status=-1)
    assert token[::2] == [-1] * 3 and min(token[1::2]) >= 0


@pytest.mark.parametrize("vocab", [1500, 50000, 200000])
def test_the_same_token_however_the_work_is_split(cats, vocab):
    """A row alone, among a few and among many; again; as a part of wider rows that start anywhere."""
    n = 300
    x = logits(n, vocab, torch.float32, 15)
    us, ts, ks = uniform(n, 16), [0.9] * n, [0, 20, 0] * 100
    ps, ms = [0.9, 1.0, 1.0] * 100, [0.0, 0.02, 0.0] * 100
    many, prob = draw(cats, x, us, ts, ks, ps, ms)
    assert (many, prob) == draw(cats, x, us, ts, ks, ps, ms)
    for lo, hi in ((0, 1), (1, 2), (2, 3), (5, 12), (20, 60)):
        assert draw(cats, x[lo:hi], us[lo:hi], ts[lo:hi], ks[lo:hi], ps[lo:hi], ms[lo:hi]) == (many[lo:hi], prob[lo:hi])
    wide = torch.full((7, vocab + 11), NAN, device="cuda")
    for off in (1, 2, 8):
        wide.fill_(NAN)
        wide[:, off:off + vocab] = x[:7]
        assert draw(cats, wide[:, off:off + vocab], us[:7], ts[:7], ks[:7], ps[:7], ms[:7])[0] == many[:7]
    half = torch.full((7, vocab + 11), NAN, dtype=torch.bfloat16, device="cuda")
    want = draw(cats, x[:7].bfloat16(), us[:7], ts[:7], ks[:7], ps[:7], ms[:7])
    for off in (1, 2, 5):
        half.fill_(NAN)
        half[:, off:off + vocab] = x[:7]
        assert draw(cats, half[:, off:off + vocab], us[:7], ts[:7], ks[:7], ps[:7], ms[:7]) == want


def test_how_often_tokens_come(cats):
    """Random numbers on an even grid: each kept token comes as often as its share says, to one."""
    x = torch.tensor([[2.0, -1.0, 0.5, 3.0, 2.0, 0.0]], device="cuda")
    n = 4096
    token, prob = draw(cats, x, [(i + 0.5) / n for i in range(n)], t=[1.3] * n, k=[4] * n, row=[0] * n)
    w = torch.softmax(x[0, [0, 2, 3, 4]].double() / 1.3, 0)
    for v, share in zip((0, 2, 3, 4), w.tolist()):
        assert abs(token.count(v) - share * n) <= 1.0
    assert token == sorted(token) and set(token) == {0, 2, 3, 4}


def test_captured_and_replayed(cats):
    """Logits, settings and random numbers are read when the graph runs."""
    x = logits(16, 32000, torch.float32, 17)
    u, t = torch.zeros(16, device="cuda"), torch.ones(16, device="cuda")
    k = torch.full((16,), 30, dtype=torch.int32, device="cuda")
    token, prob, st = torch.empty(16, dtype=torch.int32, device="cuda"), torch.empty(16, device="cuda"), cats.new_status()
    call = lambda: cats.cats_sample(x, None, t, k, None, None, u, token, prob, st)      # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (1, 2):
        x.copy_(logits(16, 32000, torch.float32, 20 + seed))
        us = uniform(16, seed)
        u.copy_(_t(us))
        k.fill_(30 * seed)
        graph.replay()
        assert token.cpu().tolist() == check(cats, x, us, k=[30 * seed] * 16)


def test_no_draws(cats):
    none = torch.empty(0, device="cuda")
    cats.cats_sample(logits(2, 10, torch.float32, 0), None, None, None, None, None, none, none.int(), None, cats.new_status())
    assert cats.last_launch_count() == 0


@pytest.mark.parametrize("weighing", [300, 900])
@pytest.mark.parametrize("vocab", [100003, 262144])
def test_top_p_after_a_top_k_that_cuts_nothing(cats, vocab, weighing):
    """Fewer tokens weigh anything than top-k asks for, over several blocks: the counts of top-k are read to their end before those of top-p begin."""
    n = 24
    x = torch.full((n, vocab), -INF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(weighing)
    at = torch.rand(n, vocab, generator=g, device="cuda").argsort(1)[:, :weighing]
    x.scatter_(1, at, torch.randn(n, weighing, generator=g, device="cuda"))
    u = uniform(n, 9)
    first = draw(cats, x, u, k=[1000] * n, p=[0.8] * n)
    check(cats, x, u, k=[1000] * n, p=[0.8] * n)
    for _ in range(20):
        assert draw(cats, x, u, k=[1000] * n, p=[0.8] * n) == first
    assert draw(cats, x, u, p=[0.8] * n) == first
