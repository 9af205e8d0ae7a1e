"""Caches without pages, rows, heads or channels: refused before anything is divided by their sizes.  On the CPU."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2605_11186_b200 import binding
    return binding


@pytest.mark.parametrize("shape", [(0, 8, 2, 64), (3, 0, 2, 64), (3, 8, 0, 64), (3, 8, 2, 0), (0, 0, 0, 0)])
@pytest.mark.parametrize("dtype", [torch.int8, torch.bfloat16])
def test_no_cache_is_made(b, shape, dtype):
    scales = [torch.zeros(shape[:3]) for _ in range(2)] if dtype == torch.int8 else []
    with pytest.raises(ValueError, match="empty"):
        b.PagedKV(torch.zeros(shape, dtype=dtype), torch.zeros(shape, dtype=dtype), *scales)


@pytest.mark.parametrize("change", [dict(n_kv_heads=0), dict(head_dim=0), dict(n_kv_heads=-1), dict(head_dim=-64)])
def test_no_call_takes_one(b, change):
    """A cache made another way: the calls refuse it by its sizes, before they look at a tensor."""
    kv = b.new_paged_kv(2, 8, 2, 64, device="cpu")
    for name, value in change.items():
        setattr(kv.struct, name, value)
    kv.desc = bytes(kv.struct)
    assert len(kv.desc) == C.sizeof(b.PagedKVDesc)
    i, x = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 128)
    for call in (lambda: b.cats_paged_append(kv, i[None], None, i, x, x, x, 0.0, x, i), lambda: b.cats_paged_read(kv, i[None], None, i, x, x, i),
                 lambda: b.cats_paged_attention(kv, i[None], i, x, 1.0, x, i, i)):
        with pytest.raises(ValueError, match="no heads"):
            call()
