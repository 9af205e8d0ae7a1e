"""The operators of a one-token pass over a paged key/value cache, as a user calls them and in their plain form.

append   new rows of K and V into the pages of their sequences: rotated to their positions, K and V held in bf16 or in 8 bits
         with one scale per row and head, the queries beside them rotated and left in bf16; then the same rows read back
read     rows of the cache, in any order, as plain bf16 matrices (what the tree verification's contiguous cache takes)
attend   one query row per sequence over that sequence's rows of the cache
sample   one token per row of logits: temperature, top-k, top-p, min-p, and a given random number

A cache row y of one head is held in 8 bits as q = rint(127 y / a), a = max(max|y|, 2^-100), with the scale a / 127.  What is
held in 8 bits is returned as the bf16 values it stands for.
Sampling orders tokens by falling logit, equal ones by rising index.  w = exp((logit - largest) / temperature); top-k keeps the
first k of the order, top-p of those the shortest run whose w add up to p of theirs, min-p the tokens with w >= min_p; the
token is the first in index order at which the sum of the kept w exceeds u times their whole sum.  Temperature 0 takes the
first token of the order.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8}
_TINY = 2.0 ** -100
_BASE = 10000.0


def listed():
    return [
        # one-token pass of the draft stage, 7B shape, behind an 8-bit product that leaves fp32: latency counts
        dict(name="append 1 row 32/32", op="append", seqs=1, rows=1, first=512, heads=32, kv=32, dim=128, page=64, cache="i8", x="f32"),
        # one token of each of 64 users, heads in groups of four
        dict(name="append 64 rows 32/8", op="append", seqs=64, rows=64, first=4000, heads=32, kv=8, dim=128, page=16, cache="bf16", x="bf16"),
        # a prompt of odd length, 7B shape
        dict(name="append 8191 rows 32/32", op="append", seqs=1, rows=8191, first=0, heads=32, kv=32, dim=128, page=16, cache="i8", x="bf16"),
        # the prefix of a tree verification, 7B shape, out of an 8-bit cache
        dict(name="read 513 rows", op="read", seqs=1, rows=513, kv=32, dim=128, page=64, cache="i8"),
        # the longest prefix of the attention benchmark
        dict(name="read 16384 rows", op="read", seqs=1, rows=16384, kv=32, dim=128, page=64, cache="i8"),
        # one-token pass of the draft stage, 7B shape, prefix 512: latency counts
        dict(name="attend 1x513 32/32", op="attend", seqs=1, longest=513, heads=32, kv=32, dim=128, page=64, cache="i8"),
        # one user with a very long text, heads in groups of four: the cache's length has to fill the GPU
        dict(name="attend 1x131071 32/8", op="attend", seqs=1, longest=131071, heads=32, kv=8, dim=128, page=64, cache="i8"),
        # 64 users with texts of all lengths, small pages, 16-bit cache
        dict(name="attend 64x8191 32/8", op="attend", seqs=64, longest=8191, heads=32, kv=8, dim=128, page=16, cache="bf16"),
        # 48 users, 13B shape, every head with keys of its own, pages of no power of two
        dict(name="attend 48x1500 40/40", op="attend", seqs=48, longest=1500, heads=40, kv=40, dim=128, page=24, cache="i8"),
        # the bonus token of one verification: latency counts
        dict(name="sample 1x32000", op="sample", rows=1, vocab=32000, x="f32", filters="kp"),
        # the next tokens of 64 users with settings of their own
        dict(name="sample 64x32000", op="sample", rows=64, vocab=32000, x="f32", filters="mixed"),
        # 256 users over a large vocabulary of odd size, logits in 16 bits
        dict(name="sample 256x128001", op="sample", rows=256, vocab=128001, x="bf16", filters="mixed"),
    ]


def _log_between(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "sample", "sample"])
    if op == "sample":
        vocab = _log_between(rng, 500, 150000)
        return dict(op=op, rows=_log_between(rng, 1, min(512, 256 * 128001 // vocab)), vocab=vocab, x=rng.choice(["f32", "bf16"]),
                    filters=rng.choice(["none", "k", "p", "m", "kp", "mixed", "mixed"]))
    heads, kv = rng.choice([(32, 32), (40, 40), (32, 8), (40, 10), (64, 8), (16, 1), (12, 4), (5, 5)])
    c = dict(op=op, kv=kv, dim=rng.choice([128, 128, 64]), page=rng.choice([1, 16, 16, 24, 64, 64, 100, 256]), cache=rng.choice(["i8", "bf16"]))
    row = 2 * kv * c["dim"]                     # elements of a cache row, K and V
    if op == "read":
        rows = _log_between(rng, 1, 16384)
        return dict(c, seqs=rng.choice([1, min(rows, 7)]), rows=rows)
    c["heads"] = heads
    if op == "append":
        rows = _log_between(rng, 1, 8191)
        return dict(c, seqs=rng.choice([1, min(rows, 9), rows if rows <= 512 else 1]), rows=rows, first=_log_between(rng, 1, 4000) - 1, x=rng.choice(["f32", "bf16"]))
    seqs = _log_between(rng, 1, 256)
    most = 64 * 8192 * 2048 // (row * max(2, seqs))     # no more elements than the largest listed case reads
    return dict(c, seqs=seqs, longest=_log_between(rng, 1, max(1, min(131071, most))))


def _lengths(case):
    """The sequences' lengths in rising order: evenly spread up to the longest; an append adds to all but the last of them one token or an even share."""
    n = case["seqs"]
    if case["op"] == "attend":
        return [case["longest"]] if n == 1 else [1 + i * (case["longest"] - 1) // (n - 1) for i in range(n)]
    return [case["rows"] // n + (i < case["rows"] % n) for i in range(n)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def shuffled(n):
        return torch.randperm(n, generator=g, device="cuda")

    def one_of(values, n, dtype):
        return torch.tensor(values, dtype=dtype, device="cuda")[torch.randint(0, len(values), (n,), generator=g, device="cuda")]

    s = {"op": op, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if op == "sample":
        rows, vocab, filters = case["rows"], case["vocab"], case["filters"]
        x = normal(rows, vocab) * 2.5
        likely = torch.randint(0, vocab, (rows, 24), generator=g, device="cuda")       # the few tokens that the text makes likely
        x.scatter_add_(1, likely, torch.rand(rows, 24, generator=g, device="cuda") * 9)
        s["logits"] = x.to(_TYPES[case["x"]])
        s["u"] = torch.rand(rows, generator=g, device="cuda")
        mixed = filters == "mixed"
        s["temperature"] = one_of([0.0, 0.6, 0.7, 0.8, 1.0, 1.0, 1.5] if mixed else [0.7, 1.0], rows, torch.float32)
        s["top_k"] = one_of([0, 0, 1, 20, 50, 1000] if mixed else [50] if "k" in filters else [0], rows, torch.int32)
        s["top_p"] = one_of([1.0, 1.0, 0.95, 0.9, 0.5] if mixed else [0.9] if "p" in filters else [1.0], rows, torch.float32)
        s["min_p"] = one_of([0.0, 0.0, 0.0, 0.05, 0.1] if mixed else [0.05] if "m" in filters else [0.0], rows, torch.float32)
        s["token"] = torch.empty(rows, dtype=torch.int32, device="cuda")
        s["prob"] = torch.empty(rows, dtype=torch.float32, device="cuda")
        return s
    n, kv, dim, page = case["seqs"], case["kv"], case["dim"], case["page"]
    first = case.get("first", 0)
    added = torch.tensor(_lengths(case), device="cuda")[shuffled(n)]
    lens = added + first
    held = -(-lens // page)                                     # pages of each sequence
    width, n_pages = int(held.max()), int(held.sum()) + 3
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    used = torch.arange(width, device="cuda")[None, :] < held[:, None]
    table[used] = shuffled(n_pages)[:int(held.sum())].int()     # pages lie anywhere
    s["table"], s["lens"] = table, lens.int()

    def pages():
        """[page][row][head][dim] over memory in which the rows of one head of a page lie together, and their scales"""
        if case["cache"] == "bf16":
            return normal(n_pages, kv, page, dim).bfloat16().transpose(1, 2), None
        q = torch.randint(-127, 128, (n_pages, kv, page, dim), generator=g, device="cuda", dtype=torch.int8)
        return q.transpose(1, 2), (0.01 + 0.01 * torch.rand(n_pages, kv, page, generator=g, device="cuda")).transpose(1, 2)

    s["k"], s["k_scale"] = pages()
    s["v"], s["v_scale"] = pages()
    if op == "attend":
        s["q"] = normal(n, case["heads"], dim).bfloat16()
        s["out"] = torch.empty_like(s["q"])
        s["scale"] = dim ** -0.5
    else:
        seq = torch.repeat_interleave(torch.arange(n, device="cuda"), added)
        start = torch.cumsum(added, 0) - added
        s["seq"], s["pos"] = seq.int(), (torch.arange(case["rows"], device="cuda") - start[seq] + first).int()
        s["k_out"] = torch.empty(case["rows"], kv * dim, dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    if op == "append":
        heads = case["heads"]
        x = normal(case["rows"], (heads + 2 * kv) * dim).to(_TYPES[case["x"]])      # one row of the QKV projection per token
        s["q_in"], s["k_in"], s["v_in"] = x.split([heads * dim, kv * dim, kv * dim], 1)
        s["q_out"] = torch.empty(case["rows"], heads * dim, dtype=torch.bfloat16, device="cuda")
    if own:         # what a program keeps for as long as its cache lives
        from paper_2605_11186_b200 import binding
        s["cache"] = binding.PagedKV(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if op == "attend":
            s["ws"] = binding.new_workspace_paged(n, case["heads"], kv, dim)
    return s


def _run_own(s):
    from paper_2605_11186_b200 import binding
    op = s["op"]
    if op == "sample":
        binding.cats_sample(s["logits"], None, s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["u"], s["token"], s["prob"], s["status"])
        return {"token": s["token"], "prob": s["prob"]}
    if op == "attend":
        binding.cats_paged_attention(s["cache"], s["table"], s["lens"], s["q"], s["scale"], s["out"], s["ws"], s["status"])
        return {"out": s["out"]}
    out = {"k": s["k_out"], "v": s["v_out"]}
    if op == "append":
        binding.cats_paged_append(s["cache"], s["table"], s["seq"], s["pos"], s["q_in"], s["k_in"], s["v_in"], _BASE, s["q_out"], s["status"])
        out.update(q=s["q_out"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    binding.cats_paged_read(s["cache"], s["table"], s["seq"], s["pos"], s["k_out"], s["v_out"], s["status"])
    return out


def _held(y):
    """q and the scale of rows [...][dim]."""
    a = y.abs().amax(-1).clamp_min(_TINY)
    return torch.round(y * (127.0 / a)[..., None]).to(torch.int8), a / 127.0


def _rows_of(s, name, at):
    """Rows of the cache in fp32."""
    x = s[name][at].float()
    return x if s[name + "_scale"] is None else x * s[name + "_scale"][at][..., None]


def _sample(s):
    x = s["logits"].double()
    rows, vocab = x.shape
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    t, k, p, m = s["temperature"].double()[:, None], s["top_k"][:, None], s["top_p"].double()[:, None], s["min_p"].double()[:, None]
    w = torch.exp((x - x[:, :1]) / torch.where(t == 0, 1.0, t))
    rank = torch.arange(vocab, device=x.device)[None, :]
    w = torch.where((t == 0) & (rank > 0), 0.0, w)
    in_k = torch.where((k > 0) & (rank >= k), 0.0, w)
    total = in_k.cumsum(1)
    before = total - in_k                                       # a token is in while the ones before it have not reached p
    keep = (in_k > 0) & (w >= m) & ((p >= 1) | (before < p * total[:, -1:]))
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))      # back in index order
    total = w.cumsum(1)
    token = (total <= s["u"].double()[:, None] * total[:, -1:]).sum(1, keepdim=True)
    return {"token": token[:, 0].int(), "prob": (w.gather(1, token) / total[:, -1:])[:, 0].float()}


def run(state):
    if own:
        return _run_own(state)
    s, op = state, state["op"]
    if op == "sample":
        return _sample(s)
    page = s["k"].shape[1]
    if op == "attend":
        n, heads, dim = s["q"].shape
        pos = torch.arange(s["table"].shape[1] * page, device="cuda")
        live = pos[None, :] < s["lens"][:, None]
        pages = torch.where(live, s["table"].repeat_interleave(page, 1), 0)
        at = pages.long(), (pos % page).expand_as(pages)
        k, v = _rows_of(s, "k", at), _rows_of(s, "v", at)                       # [seq][row][kv head][dim]
        q = s["q"].float().view(n, k.shape[2], -1, dim)
        w = torch.einsum("ngrd,nlgd->ngrl", q, k) * s["scale"]
        w = torch.where(live[:, None, None, :], w, -math.inf)
        w = torch.exp(w - w.amax(-1, keepdim=True))
        out = torch.einsum("ngrl,nlgd->ngrd", w, v) / w.sum(-1, keepdim=True)
        return {"out": out.reshape(n, heads, dim).bfloat16()}
    seq, pos = s["seq"].long(), s["pos"].long()
    at = s["table"][seq, pos // page].long(), pos % page
    rows, kv, dim = pos.numel(), s["k"].shape[2], s["k"].shape[3]
    out = {}
    if op == "append":
        turn = pos.double()[:, None] * _BASE ** (-torch.arange(0, dim, 2, device="cuda").double() / dim)
        cos, sin = turn.cos().float()[:, None], turn.sin().float()[:, None]

        def rotated(x):
            lo, hi = x.float().view(rows, -1, dim).chunk(2, 2)
            return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], 2)

        out["q"] = rotated(s["q_in"]).view(rows, -1).bfloat16()
        k, v = rotated(s["k_in"]), s["v_in"].float().view(rows, kv, dim)
        if s["k_scale"] is None:
            s["k"][at], s["v"][at] = k.bfloat16(), v.bfloat16()
        else:
            s["k"][at], s["k_scale"][at] = _held(k)
            s["v"][at], s["v_scale"][at] = _held(v)
        out.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
    for name in ("k", "v"):
        out[name] = _rows_of(s, name, at).reshape(rows, kv * dim).bfloat16()
    return out


def work(case):
    op = case["op"]
    if op == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * _TYPES[case["x"]].itemsize + 28 * case["rows"], "flops": 4 * n}
    kv, dim = case["kv"], case["dim"]
    row = 2 * kv * (dim * _TYPES[case["cache"]].itemsize + (4 if case["cache"] == "i8" else 0))      # a row of K and of V
    if op == "attend":
        total = sum(_lengths(case))
        return {"bytes": total * row + 4 * case["seqs"] * case["heads"] * dim, "flops": 4 * total * case["heads"] * dim}
    rows, plain = case["rows"], 4 * kv * dim
    if op == "read":
        return {"bytes": rows * (row + plain), "flops": rows * 2 * kv * dim}
    heads = case["heads"]
    return {"bytes": rows * ((heads + 2 * kv) * dim * _TYPES[case["x"]].itemsize + 2 * heads * dim + row + plain), "flops": rows * (3 * (heads + kv) + 6 * kv) * dim}


def _exact_sample(s):
    """Row by row on the host: sort, cut, add up."""
    tokens, probs = [], []
    for x, t, k, p, m, u in zip(*(s[n].double().cpu().numpy() for n in ("logits", "temperature", "top_k", "top_p", "min_p", "u"))):
        order = np.argsort(-x, kind="stable")
        order = order[:1] if t == 0 else order[:int(k)] if k > 0 else order
        mass = np.exp((x[order] - x[order[0]]) / t) if t else np.ones(1)
        n = order.size if p >= 1 else min(order.size, 1 + int(np.searchsorted(np.cumsum(mass), p * mass.sum())))
        n = min(n, int(np.count_nonzero(mass >= m)))
        by_index = np.argsort(order[:n])
        along = np.cumsum(mass[:n][by_index])
        i = int(np.searchsorted(along, float(u) * along[-1], side="right"))
        tokens.append(int(order[by_index[i]]))
        probs.append(mass[by_index[i]] / along[-1])
    return {"token": np.array(tokens, dtype=np.int32), "prob": np.array(probs)}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "sample":
        return _exact_sample(s)
    page = case["page"]

    def stored(name, at):
        x = s[name][at].to(torch.float64)
        return x if case["cache"] == "bf16" else x.mul(s[name + "_scale"][at].to(torch.float64).unsqueeze(-1))

    if op == "attend":
        out = torch.zeros(case["seqs"], case["heads"], case["dim"], dtype=torch.float64, device="cuda")
        group = case["heads"] // case["kv"]
        for i, length in enumerate(s["lens"].tolist()):
            p = torch.arange(length, device="cuda")
            at = s["table"][i].long()[p.div(page, rounding_mode="floor")], p.remainder(page)
            k, v = stored("k", at).repeat_interleave(group, 1), stored("v", at).repeat_interleave(group, 1)
            score = torch.matmul(k.transpose(0, 1), s["q"][i].to(torch.float64).unsqueeze(2)).squeeze(2).mul(s["scale"])
            out[i] = torch.softmax(score, 1).unsqueeze(1).matmul(v.transpose(0, 1)).squeeze(1)
        return {"out": out}
    seq, p = s["seq"].long(), s["pos"].long()
    at = s["table"][seq, p.div(page, rounding_mode="floor")].long(), p.remainder(page)
    flat = (case["rows"], case["kv"] * case["dim"])
    if op == "read":
        return {"k": stored("k", at).reshape(flat), "v": stored("v", at).reshape(flat)}
    half = case["dim"] // 2
    angle = torch.outer(p.to(torch.float64), torch.pow(torch.tensor(_BASE, dtype=torch.float64, device="cuda"), -torch.arange(half, device="cuda").to(torch.float64) / half))
    spin = torch.polar(torch.ones_like(angle), angle).unsqueeze(1)

    def turned(x):
        x = x.to(torch.float64).unflatten(1, (-1, case["dim"]))
        z = torch.complex(x[..., :half], x[..., half:]) * spin
        return torch.cat([z.real, z.imag], 2)

    found = {"q": turned(s["q_in"]).flatten(1)}
    for name, y in (("k", turned(s["k_in"])), ("v", s["v_in"].to(torch.float64).unflatten(1, (-1, case["dim"])))):
        if case["cache"] == "bf16":
            found[name], found[name + "_scale"] = y.reshape(flat), None
            continue
        step = torch.maximum(y.amax(2), -y.amin(2)).clamp(min=_TINY).div(127)
        found[name] = y.div(step.unsqueeze(2)).round().mul(step.unsqueeze(2)).reshape(flat)
        found[name + "_scale"] = s[name + "_scale"].to(torch.float64).index_put(at, step)
    return found
