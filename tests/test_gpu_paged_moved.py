"""A cache whose tensors lie elsewhere than when it was made is refused: the calls know the old addresses only."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _calls(cats, kv):
    i = torch.zeros(1, dtype=torch.int32, device="cuda")
    x, y = (torch.zeros(1, 128, device="cuda") for _ in range(2))
    q = torch.zeros(1, 128, dtype=torch.bfloat16, device="cuda")
    ws = cats.new_workspace_paged(1, 2, 2, 64)
    st = cats.new_status()
    return [lambda: cats.cats_paged_append(kv, i[None], None, i, None, x, x, 0.0, None, st),
            lambda: cats.cats_paged_read(kv, i[None], None, i, x, y, st),
            lambda: cats.cats_paged_attention(kv, i[None], i + 1, q, 1.0, torch.empty_like(q), ws, st)]


@pytest.mark.parametrize("dtype", [torch.int8, torch.bfloat16])
@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale"])
@pytest.mark.parametrize("how", ["data", "attribute", "storage", "device"])
def test_moved(cats, dtype, name, how):
    kv = cats.new_paged_kv(2, 8, 2, 64, dtype=dtype)
    for call in _calls(cats, kv):
        call()
    t = getattr(kv, name)
    if t is None:
        if how != "attribute":
            return
        setattr(kv, name, torch.zeros(2, 8, 2, device="cuda"))          # scales that the cache was not made with
    elif how == "data":
        t.data = t.clone()
    elif how == "attribute":
        setattr(kv, name, t.clone())
    elif how == "storage":
        t.untyped_storage().resize_(0)
    else:
        setattr(kv, name, t.cpu())
    for call in _calls(cats, kv):
        with pytest.raises(ValueError, match="cache"):
            call()
    torch.cuda.synchronize()
