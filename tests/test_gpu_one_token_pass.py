"""The paged cache and sampling together with the operators beside them, as a program uses them: one-token passes of a batch of sequences
(norm, QKV product, append, attention, O product, LM head, draw), and a paged sequence handed to the tree attention."""
import numpy as np
import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, KV, DIM, VOCAB, PAGE, BASE = 256, 8, 2, 64, 1000, 16, 10000.0


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


class Model:
    """One layer's attention half and an LM head, 8-bit weights, buffers for a batch of rows."""

    def __init__(self, cats, rows, kind, n_pages):
        g = torch.Generator(device="cuda").manual_seed(1)
        w = lambda *shape: torch.randn(*shape, generator=g, device="cuda").bfloat16() * 0.08      # noqa: E731
        self.cats, self.rows = cats, rows
        self.embed = torch.randn(VOCAB, HIDDEN, generator=g, device="cuda")
        self.gain = (1 + 0.1 * torch.randn(HIDDEN, generator=g, device="cuda")).bfloat16()
        self.qkv, self.o, self.head = (cats.quantize_weights_i8(m) for m in (w((HEADS + 2 * KV) * DIM, HIDDEN), w(HIDDEN, HEADS * DIM), w(VOCAB, HIDDEN) * 6))
        self.cache = ref.Cache(cats, n_pages, PAGE, KV, DIM, kind, fill=0)
        self.resid = torch.empty(rows, HIDDEN, device="cuda")
        self.x, self.xs = cats.new_i8(rows, HIDDEN)
        self.a, self.sa = cats.new_i8(rows, HEADS * DIM)
        self.wide = torch.empty(rows, (HEADS + 2 * KV) * DIM, device="cuda")
        self.q = torch.zeros(rows, HEADS * DIM, dtype=torch.bfloat16, device="cuda")
        self.att = torch.empty_like(self.q)
        self.delta = torch.empty(rows, HIDDEN, device="cuda")
        self.logits = torch.empty(rows, VOCAB, device="cuda")
        self.token = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.prob = torch.empty(rows, device="cuda")
        self.ws, self.st = cats.new_workspace_paged(rows, HEADS, KV, DIM), cats.new_status()
        self.pos, self.len = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
        self.u = torch.zeros(rows, device="cuda")
        self.settings = [torch.tensor(v, device="cuda", dtype=d) for v, d in
                         (([0.8, 1.0, 0.0, 1.2, 0.7], torch.float32), ([40, 0, 0, 500, 5], torch.int32), ([0.9, 0.95, 1.0, 1.0, 1.0], torch.float32), ([0.0, 0.0, 0.0, 0.02, 0.0], torch.float32))]

    def step(self, table):
        b, n = self.cats, HEADS * DIM
        torch.index_select(self.embed, 0, self.token, out=self.resid)
        b.cats_rmsnorm_i8(self.resid, None, self.gain, 1e-5, None, self.x, self.xs)
        b.cats_linear_i8(self.x, self.xs, *self.qkv, self.wide, self.st)
        q, k, v = self.wide.split([n, KV * DIM, KV * DIM], 1)
        b.cats_paged_append(self.cache.dev, table, None, self.pos, q, k, v, BASE, self.q, self.st)
        b.cats_paged_attention(self.cache.dev, table, self.len, self.q, DIM ** -0.5, self.att, self.ws, self.st)
        b.cats_quantize_i8(self.att, self.a, self.sa)
        b.cats_linear_i8(self.a, self.sa, *self.o, self.delta, self.st)
        b.cats_rmsnorm_i8(self.resid, self.delta, self.gain, 1e-5, None, self.x, self.xs)
        b.cats_linear_i8(self.x, self.xs, *self.head, self.logits, self.st)
        b.cats_sample(self.logits, None, *self.settings, self.u, self.token, self.prob, self.st)


def _check_step(m, table, lens):
    """Every new operator of the pass against 64 bits, from the inputs that it had."""
    assert int(m.st.item()) == 0
    live = torch.tensor([i for i, n in enumerate(lens) if n > 0], device="cuda")
    pos = torch.tensor([lens[i] - 1 for i in live.tolist()], device="cuda")
    at = ref.places(table, PAGE, live, pos)
    q, k, v = m.wide[live].split([HEADS * DIM, KV * DIM, KV * DIM], 1)
    ref.check_cache(m.cache, "k", *at, *ref.rotated(k, pos, BASE, DIM))
    ref.check_cache(m.cache, "v", *at, *ref.rotated(v, pos, 0, DIM))
    ref.check_bf16(m.q[live], *ref.rotated(q, pos, BASE, DIM))
    for i, n in enumerate(lens):
        rows = torch.arange(n, device="cuda")
        rows = ref.places(table, PAGE, torch.full_like(rows, i), rows)
        ref.check_attention(m.att[i].view(HEADS, DIM), m.q[i].view(HEADS, DIM), m.cache.rows("k", *rows), m.cache.rows("v", *rows), DIM ** -0.5, m.cache.kind)
    x = m.logits.double().cpu().numpy()
    t, k, p, mn = (s.double().cpu().numpy() for s in m.settings)
    for i in range(m.rows):
        want, share, near = ref.sample(x[i], t[i], int(k[i]), p[i], mn[i], float(m.u[i]))
        if near > 1e-9:
            assert int(m.token[i]) == want and abs(float(m.prob[i]) - share) <= 2 * ref.U * share + 1e-9 * share


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_one_token_passes(cats, kind):
    """Five sequences that grow token by token from prompts of different lengths, one of them idle (a padded batch: position -1, length 0); again
    through a captured graph, with the same tokens."""
    prompts = [1, 17, 40, 0, 15]
    steps = 6
    tokens = {}
    for mode in ("eager", "graph"):
        m = Model(cats, 5, kind, 40)
        g = torch.Generator(device="cuda").manual_seed(2)
        table = ref.table_for(g, [p + steps + 1 for p in prompts], PAGE, 40)
        # the prompts' rows, all in one call
        seq = torch.repeat_interleave(torch.arange(5, device="cuda"), torch.tensor(prompts, device="cuda")).int()
        pos = torch.cat([torch.arange(p, device="cuda") for p in prompts]).int()
        kv = torch.randn(seq.numel(), 2, KV * DIM, generator=g, device="cuda")
        cats.cats_paged_append(m.cache.dev, table, seq, pos, None, kv[:, 0], kv[:, 1], BASE, None, m.st)
        m.token.copy_(torch.tensor([3, 1, 4, 1, 5], dtype=torch.int32))
        graph = None
        if mode == "graph":
            keep = m.token.clone()
            m.pos.fill_(-1)             # a pass that writes nothing, so that everything is loaded before the capture
            m.step(table)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                m.step(table)
            m.token.copy_(keep)
            m.st.zero_()
        lens = [p if p else 0 for p in prompts]
        drawn = []
        for i in range(steps):
            lens = [n + 1 if prompts[j] else 0 for j, n in enumerate(lens)]
            m.len.copy_(torch.tensor(lens, dtype=torch.int32))
            m.pos.copy_(torch.tensor([n - 1 for n in lens], dtype=torch.int32))
            m.u.copy_(torch.rand(5, generator=torch.Generator().manual_seed(i)))
            graph.replay() if graph is not None else m.step(table)
            _check_step(m, table, lens)
            drawn.append(m.token.cpu().tolist())
        tokens[mode] = drawn
        assert (m.att[3] == 0).all()
    assert tokens["eager"] == tokens["graph"]


@pytest.mark.parametrize("kind", ["i8", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_paged_sequence_to_the_tree_attention(cats, kind, dim):
    """Rows of a paged cache read back into the contiguous cache of the tree verification: the tree attention of one node over them is what the paged
    attention computes over the same values."""
    nh, n = 4, 300
    g = torch.Generator(device="cuda").manual_seed(3)
    cache = ref.Cache(cats, 25, 16, nh, dim, kind, fill=0)
    table = ref.table_for(g, [n], 16, 25)
    at = torch.arange(n, device="cuda")
    cache.fill(g, *ref.places(table, 16, torch.zeros_like(at), at))
    kc, vc = (torch.zeros(n, nh * dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st, seq, pos = cats.new_status(), torch.zeros(n, dtype=torch.int32, device="cuda"), at.int()
    cats.cats_paged_read(cache.dev, table, seq, pos, kc, vc, st)
    q = torch.randn(1, nh, dim, generator=g, device="cuda").bfloat16()
    mask = torch.tensor([[1, 0]], dtype=torch.int64, device="cuda")
    out, scale = torch.empty_like(q), dim ** -0.5
    cfg = cats.ModelCfg(nh * dim, nh, dim, 64, 128, 1, n, 1e-5, BASE)
    cats.cats_tree_attention(q, kc, vc, mask, 1, n - 1, nh, dim, nh * dim, scale, out, cats.new_workspace(cfg, 1, n), st)
    plain = cats.PagedKV(kc.view(1, n, nh, dim), vc.view(1, n, nh, dim))        # the contiguous cache as one page
    again = torch.empty_like(q)
    cats.cats_paged_attention(plain, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda"), q, scale, again,
                              cats.new_workspace_paged(1, nh, nh, dim), st)
    assert int(st.item()) == 0
    for o in (out, again):
        ref.check_attention(o[0], q[0], kc.double().view(n, nh, dim), vc.double().view(n, nh, dim), scale, "bf16")


def test_the_bonus_token_is_drawn(cats):
    """After a walk the token behind the last accepted node comes from that node's logits: its index goes to the draw on the device."""
    g = torch.Generator(device="cuda").manual_seed(4)
    T, V = 12, 3000
    logits = torch.randn(T, V, generator=g, device="cuda") * 2
    parent = torch.tensor([-1, 0, 1, 2, 0, 4, 1, 6, 7, 3, 9, 5], dtype=torch.int32, device="cuda")
    argmax = logits.argmax(1).int()
    tokens = torch.zeros(T, dtype=torch.int32, device="cuda")
    tokens[1:] = argmax[parent[1:].long()]
    tokens[4], tokens[6], tokens[9] = 0, 1, 2                       # rejected
    path, out = (torch.zeros(T, dtype=torch.int32, device="cuda") for _ in range(2))
    n, n_out, st = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(3))
    cats.cats_accept_path(parent, tokens, argmax, T, path, n, out, n_out, st)
    row = path.gather(0, n.long() - 1)
    u = torch.tensor([0.37], device="cuda")
    token, prob = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
    t, p = torch.tensor([0.7], device="cuda"), torch.tensor([0.9], device="cuda")
    cats.cats_sample(logits, row, t, None, p, None, u, token, prob, st)
    last = int(path[int(n.item()) - 1])
    assert last == 3 and int(st.item()) == 0
    want, share, near = ref.sample(logits[last].double().cpu().numpy(), float(np.float32(0.7)), 0, float(np.float32(0.9)), 0.0, float(np.float32(0.37)))
    assert near > 1e-9 and int(token.item()) == want and abs(float(prob.item()) - share) <= 3 * ref.U
