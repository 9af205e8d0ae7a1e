"""Plain 64-bit forms of the paged-cache operators and of sampling, and how far a correct kernel may be from them.

u = 2^-24: half a step of fp32, relative."""
import math

import numpy as np
import torch

import i8_reference as i8

U = 2.0 ** -24
BF16 = 2.0 ** -8             # half a step of bf16, relative


class Cache:
    """Pages with chosen strides: order "heads" keeps the rows of one head of a page together, "rows" the heads of a row."""

    def __init__(self, cats, n_pages, page, kv, dim, kind, order="heads", pad=0, fill=None):
        dtype = {"bf16": torch.bfloat16, "i8": torch.int8}[kind]
        self.n_pages, self.page, self.kv, self.dim, self.kind = n_pages, page, kv, dim, kind

        def pages(last, dtype, value):
            a, b = (kv, page) if order == "heads" else (page, kv)
            t = torch.full((n_pages, a, b) + ((last + pad,) if last else ()), value, dtype=dtype, device="cuda")
            t = t[..., :last] if last else t
            return t.transpose(1, 2) if order == "heads" else t
        value = fill if fill is not None else (0 if kind == "i8" else float("nan"))
        self.k, self.v = pages(dim, dtype, value), pages(dim, dtype, value)
        self.ks = self.vs = None
        if kind == "i8":
            self.ks, self.vs = pages(0, torch.float32, float("nan")), pages(0, torch.float32, float("nan"))
        self.dev = cats.PagedKV(self.k, self.v, self.ks, self.vs)

    def rows(self, name, page, at):
        """fp64 values of rows [n][kv][dim]."""
        x = getattr(self, name)[page, at].double()
        return x if self.kind == "bf16" else x * getattr(self, name + "s")[page, at].double()[..., None]

    def fill(self, g, page, at):
        """Random rows at (page, at); everything else stays as it was."""
        for name in ("k", "v"):
            shape = (page.numel(), self.kv, self.dim)
            if self.kind == "bf16":
                getattr(self, name)[page, at] = torch.randn(*shape, generator=g, device="cuda").bfloat16()
            else:
                getattr(self, name)[page, at] = torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)
                getattr(self, name + "s")[page, at] = 0.02 * torch.rand(*shape[:2], generator=g, device="cuda")


def table_for(g, lens, page, n_pages, spare=1):
    """Pages of each sequence drawn without order; entries that no row needs name no page."""
    held = [-(-n // page) for n in lens]
    assert sum(held) <= n_pages
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    t = torch.full((len(lens), max(held + [0]) + spare), -7, dtype=torch.int32, device="cuda")
    first = 0
    for i, h in enumerate(held):
        t[i, :h] = order[first:first + h]
        first += h
    return t


def places(table, page, seq, pos):
    return table[seq.long(), pos.long() // page].long(), pos.long() % page


def rotated(x, pos, base, dim):
    """x fp64 [rows][heads * dim] at positions pos, and a bound on the error of an fp32 rotation: cos and sin are off by 2^-22 and what
    an fp64 angle of that many turns loses, and two products and a sum are rounded."""
    rows = x.shape[0]
    x = x.double().view(rows, -1, dim)
    if base == 0:
        return x, torch.zeros_like(x)
    half = dim // 2
    angle = pos.double()[:, None] * base ** (-2.0 * torch.arange(half, device=x.device).double() / dim)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    lo, hi = x[..., :half], x[..., half:]
    y = torch.cat([lo * c - hi * s, hi * c + lo * s], 2)
    off = 2.0 ** -22 + 3 * U + pos.double()[:, None, None] * 2.0 ** -50
    size = (lo.abs() + hi.abs()) * off
    return y, torch.cat([size, size], 2)


def check_bf16(got, want, off):
    got = got.double().view_as(want)
    bad = ~((got - want).abs() <= BF16 * (want.abs() + off) + off + 2.0 ** -133)
    assert not bad.any(), (int(bad.sum()), (got - want).abs().max().item())


def check_cache(cache, name, page, at, want, off):
    """Rows of the cache against fp64 rows [n][kv][dim] that are off by at most `off`."""
    if cache.kind == "bf16":
        return check_bf16(getattr(cache, name)[page, at], want, off)
    q, scale = getattr(cache, name)[page, at].reshape(-1, cache.dim), getattr(cache, name + "s")[page, at].reshape(-1)
    y = want.reshape(-1, cache.dim)
    a, steps = i8.held(y)
    rel = (off.reshape(-1, cache.dim).amax(1) / a)                       # of the largest, and of every value in units of it
    assert ((scale.double() - a / 127).abs() <= (rel + 2 * U) * a / 127).all()
    assert ((q.double() - steps).abs() <= 0.5 + 127 * (2 * rel + 4 * U)[:, None]).all()


def attention(q, k, v, scale):
    """q [heads][dim], k, v fp64 [n][kv][dim]: out [heads][dim], sum p |v|, and the largest sum |q k scale| and |score|."""
    heads, dim = q.shape
    n, kv = k.shape[:2]
    if n == 0:
        z = torch.zeros(heads, dim, dtype=torch.float64, device=q.device)
        return z, z, 0.0, 0.0
    q = q.double().view(kv, heads // kv, dim)
    s = torch.einsum("grd,lgd->grl", q, k) * scale
    size = torch.einsum("grd,lgd->grl", q.abs(), k.abs()).amax().item() * abs(scale)
    p = torch.softmax(s, -1)
    out = torch.einsum("grl,lgd->grd", p, v).reshape(heads, dim)
    return out, torch.einsum("grl,lgd->grd", p, v.abs()).reshape(heads, dim), size, s.abs().amax().item()


def attention_off(kind, n, dim, size, score):
    """Error of the kernel's fp32 result in units of sum p |v|.  A score: dim products (exact, the int8 scale and the softmax scale round) added
    in fp32 by instructions that may cut instead of round (2 u each): (dim + 3) 2 u size; times log2 e and less the maximum: 3 u of
    2 |score| more; 2^x: 4 u.  Twice all that, for numerator and denominator.  The probability enters the second product with 2^-17
    (two bf16 parts) or 2^-12 (fp16, after one more product and one rescale per step of the running maximum: 4 u).  Sums: every
    term passes at most n / 64 + 64 additions of 2 u: a warp adds 16 rows or more at once, and at least four share a row's length."""
    p = 2 * ((dim + 3) * 2 * U * size + 6 * U * 2 * score + 8 * U)
    return p + (2.0 ** -17 if kind == "bf16" else 2.0 ** -12 + 4 * U) + (n / 64 + 64) * 2 * U * 2


def check_attention(got, q, k, v, scale, kind):
    want, size_v, size, score = attention(q, k, v, scale)
    off = attention_off(kind, k.shape[0], q.shape[1], size, score) * size_v
    check_bf16(got, want, off)


def sample(x, t, k, p, m, u):
    """One draw from fp64 logits, and how near u came to another answer (in parts of the whole)."""
    order = np.argsort(-x, kind="stable")
    if t == 0:
        return int(order[0]), 1.0, 1.0
    top = x[order[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(np.isneginf(x), 0.0, np.exp((x - top) / t) if not math.isinf(t) else 1.0)
    if k > 0:
        order = order[:k]
    mass = np.cumsum(w[order])
    near = 1.0
    if p < 1:
        want = p * mass[-1]
        n = 1 + int(np.searchsorted(mass, want))
        near = float(np.abs(mass - want).min() / mass[-1])
        order = order[:n]
    n = max(1, int(np.count_nonzero(w[order] >= m)))
    if m > 0:
        near = min(near, float(np.abs(w[order] - m).min()) if m != 1 else 1.0)
    kept = np.sort(order[:n])
    along = np.cumsum(w[kept])
    r = min(max(u, 0.0), 1.0) * along[-1]
    i = min(int(np.searchsorted(along, r, side="right")), int(np.searchsorted(along, along[-1])))
    if 0 < u < 1:
        near = min(near, float(np.abs(along[:-1] - r).min() / along[-1]) if kept.size > 1 else 1.0)
    return int(kept[i]), float(w[kept[i]] / along[-1]), near
