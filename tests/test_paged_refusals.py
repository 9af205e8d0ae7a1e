"""What the paged-cache and sampling entry points refuse, through the C ABI and without a GPU: a refused call launches nothing."""
import ctypes as C

import pytest
import torch

A = 1 << 20                     # an address that is aligned to anything; never dereferenced
F32, BF16, I8 = 0, 1, 2
INVALID, UNSUPPORTED, WORKSPACE = -1, -3, -4


@pytest.fixture(scope="module")
def b():
    from paper_2605_11186_b200 import binding
    return binding


def _kv(b, **change):
    a = dict(k=A, v=A, ks=A, vs=A, type=I8, n_pages=10, page_size=16, n_kv=4, hd=64, page=16 * 256, row=256, head=64, s_page=64, s_row=4, s_head=1)
    a.update(change)
    return b.PagedKVDesc(*a.values())


CACHE = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ks=None), INVALID), (dict(vs=None), INVALID), (dict(k=A + 8), INVALID), (dict(v=A + 4), INVALID),
         (dict(ks=A + 2), INVALID), (dict(type=0), INVALID), (dict(type=3), INVALID), (dict(n_pages=0), INVALID), (dict(page_size=0), INVALID), (dict(n_kv=0), INVALID),
         (dict(page=-16), INVALID), (dict(row=250), INVALID), (dict(head=72), INVALID), (dict(s_row=-1), INVALID), (dict(hd=96), UNSUPPORTED), (dict(hd=0), UNSUPPORTED),
         (dict(page=2 ** 33), UNSUPPORTED), (dict(page=2 ** 62), UNSUPPORTED), (dict(s_page=2 ** 30), UNSUPPORTED), (dict(page_size=2 ** 26 + 1), UNSUPPORTED),
         (dict(type=BF16, page=2 ** 32), UNSUPPORTED), (dict(type=BF16, row=260), INVALID)]
TABLE = [(dict(table=None), INVALID), (dict(table=A + 2), INVALID), (dict(width=0), INVALID), (dict(ld=3), INVALID), (dict(n_seqs=-1), INVALID)]


def _append(b, kv, **change):
    a = dict(table=A, ld=4, width=4, n_seqs=3, seq=A, pos=A, rows=2, q=A, ldq=512, heads=8, k=A, ldk=256, v=A, ldv=256, type=F32, base=10000.0, qo=2 * A, ldqo=512, st=A)
    a.update(change)
    rc = b.lib.cats_paged_append(kv if kv is None else C.byref(kv), *a.values(), None)
    assert b.lib.cats_last_launch_count() == 0
    return rc


def _read(b, kv, **change):
    a = dict(table=A, ld=4, width=4, n_seqs=3, seq=A, pos=A, rows=2, k=A, ldk=256, v=A, ldv=256, type=F32, st=A)
    a.update(change)
    rc = b.lib.cats_paged_read(kv if kv is None else C.byref(kv), *a.values(), None)
    assert b.lib.cats_last_launch_count() == 0
    return rc


def _attend(b, kv, **change):
    a = dict(table=A, ld=4, width=4, len=A, n_seqs=3, q=A, ldq=512, heads=8, scale=0.1, o=A, ldo=512, ws=A, n=None, st=A)
    a.update(change)
    if a["n"] is None:
        a["n"] = b.lib.cats_paged_workspace_bytes(max(a["n_seqs"], 1), 8, 4, 64)
    rc = b.lib.cats_paged_attention(kv if kv is None else C.byref(kv), *a.values(), None)
    assert b.lib.cats_last_launch_count() == 0
    return rc


@pytest.mark.parametrize("call", [_append, _read, _attend])
def test_cache_and_table(b, call):
    assert call(b, None) == INVALID
    for change, code in CACHE:
        assert call(b, _kv(b, **change)) == code, change
    for change, code in TABLE:
        assert call(b, _kv(b), **change) == code, change


@pytest.mark.parametrize("change", [dict(pos=None), dict(pos=A + 1), dict(seq=A + 2), dict(seq=None, rows=4), dict(rows=-1), dict(k=None), dict(v=None), dict(k=A + 2),
                                    dict(ldk=255), dict(ldv=255), dict(ldq=511), dict(ldqo=511), dict(type=I8), dict(base=-1.0), dict(base=float("nan")),
                                    dict(base=float("inf")), dict(heads=0), dict(heads=-1), dict(qo=None), dict(q=A, qo=A), dict(qo=A + 1), dict(q=A + 2), dict(st=None)])
def test_append(b, change):
    assert _append(b, _kv(b), **change) == INVALID


@pytest.mark.parametrize("change", [dict(pos=None), dict(seq=None, rows=4), dict(rows=-1), dict(k=None), dict(v=None), dict(k=A + 2), dict(type=BF16, v=A + 1), dict(ldk=255),
                                    dict(ldv=255), dict(type=I8), dict(st=None)])
def test_read(b, change):
    assert _read(b, _kv(b), **change) == INVALID


@pytest.mark.parametrize("change,code", [(dict(len=None), INVALID), (dict(len=A + 2), INVALID), (dict(q=None), INVALID), (dict(q=A + 8), INVALID), (dict(o=None), INVALID),
                                         (dict(o=A + 2), INVALID), (dict(ldq=504), INVALID), (dict(ldq=516), INVALID), (dict(ldo=511), INVALID), (dict(ldo=513), INVALID),
                                         (dict(heads=0), INVALID), (dict(heads=6), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
                                         (dict(st=None), INVALID), (dict(ws=None), INVALID), (dict(ws=A + 512), WORKSPACE), (dict(n=0), WORKSPACE),
                                         (dict(heads=1 << 20, ldq=1 << 26, ldo=1 << 26), UNSUPPORTED)])
def test_attention(b, change, code):
    assert _attend(b, _kv(b), **change) == code


def test_workspace_size(b):
    size = b.lib.cats_paged_workspace_bytes
    assert size(1, 32, 32, 128) > 0 and size(1, 32, 32, 128) % 1024 == 0 and size(0, 8, 1, 64) > 0
    assert size(1, 6, 4, 64) == 0 and size(1, 0, 1, 64) == 0 and size(1, 4, 0, 64) == 0 and size(-1, 4, 4, 64) == 0 and size(1, 4, 4, 96) == 0
    assert size(1 << 20, 32, 32, 128) == 0


@pytest.mark.parametrize("change,code", [(dict(x=None), INVALID), (dict(x=A + 2), INVALID), (dict(t=I8), INVALID), (dict(ld=99), INVALID), (dict(n=-1), INVALID),
                                         (dict(vocab=0), INVALID), (dict(rows=-1), INVALID), (dict(rows=6), INVALID), (dict(u=None), INVALID), (dict(u=A + 2), INVALID),
                                         (dict(row=A + 1), INVALID), (dict(temp=A + 1), INVALID), (dict(k=A + 1), INVALID), (dict(p=A + 1), INVALID), (dict(m=A + 1), INVALID),
                                         (dict(tok=None), INVALID), (dict(tok=A + 3), INVALID), (dict(prob=A + 1), INVALID), (dict(st=None), INVALID),
                                         (dict(vocab=262145, ld=262145), UNSUPPORTED), (dict(rows=2 ** 27 + 1, n=2 ** 27 + 1), UNSUPPORTED)])
def test_sample(b, change, code):
    a = dict(x=A, t=F32, ld=100, n=5, vocab=100, row=None, rows=5, temp=A, k=A, p=A, m=A, u=A, tok=A, prob=A, st=A)
    a.update(change)
    assert b.lib.cats_sample(*a.values(), None) == code
    assert b.lib.cats_last_launch_count() == 0


def test_no_rows_is_no_work(b):
    """Nothing to do: accepted, nothing launched, no pointer of a row looked at."""
    kv = _kv(b)
    assert _append(b, kv, rows=0, pos=None, k=None, v=None) == 0 and _read(b, kv, rows=0, pos=None, k=None, v=None) == 0
    assert _attend(b, kv, n_seqs=0, len=None, q=None, o=None, table=None) == 0
    assert b.lib.cats_sample(None, F32, 100, 0, 100, None, 0, None, None, None, None, None, None, None, None, None) == 0


def test_paged_kv(b):
    """Tensors that do not make a cache."""
    def t(*shape, dtype=torch.int8):
        return torch.zeros(*shape, dtype=dtype)
    s = [t(3, 8, 2, dtype=torch.float32) for _ in range(2)]
    k, v = t(3, 8, 2, 64), t(3, 8, 2, 64)
    kv = b.PagedKV(k, v, *s)
    assert len(kv.desc) == C.sizeof(b.PagedKVDesc) and (kv.struct.n_pages, kv.struct.page_size, kv.struct.n_kv_heads, kv.struct.head_dim) == (3, 8, 2, 64)
    for bad in ((k, v), (k, v, s[0]), (k, t(3, 8, 2, 32), *s), (k, v.bfloat16(), *s), (k.float(), v.float(), *s), (k.bfloat16(), v.bfloat16(), *s), (k[0], v[0], *s),
                (k, v, s[0], s[1].double()), (k, v, s[0][:2], s[1][:2]), (None, v, *s), (k, None, *s), (k, t(3, 2, 8, 64).transpose(1, 2), *s),
                (t(3, 8, 64, 2).transpose(2, 3), t(3, 8, 64, 2).transpose(2, 3), *s)):
        with pytest.raises(ValueError):
            b.PagedKV(*bad)


def test_tensors_of_the_calls(b):
    """Host tensors and things that are no cache are refused by the binding."""
    kv = b.new_paged_kv(2, 8, 2, 64, device="cpu")
    i, x = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 128)
    for cache in (kv, None, x):
        with pytest.raises(ValueError):
            b.cats_paged_append(cache, i[None], None, i, None, x, x, 0.0, None, i)
        with pytest.raises(ValueError):
            b.cats_paged_read(cache, i[None], None, i, x, x, i)
        with pytest.raises(ValueError):
            b.cats_paged_attention(cache, i[None], i, x, 1.0, x, i, i)
    with pytest.raises(ValueError):
        b.cats_sample(x, None, None, None, None, None, x[0, :1], i, None, i)
    with pytest.raises(TypeError):
        b._marshal().sample(x)
