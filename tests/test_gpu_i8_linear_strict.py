"""The 8-bit product element by element, with checks that fail on NaN, and rows and channels that are not finite in every kernel of it."""
import pytest
import torch

import i8_strict
from test_gpu_i8_linear import SIZES

pytestmark = pytest.mark.gpu

# few tokens, whole tiles, tiles shared by a cluster, pairs
KERNELS = [(1, 300, 77), (3, 4096, 200), (40, 256, 64), (64, 11008, 512), (77, 640, 20000), (700, 512, 3000)]


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _problem(rows, cols, outs, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def whole(r):
        t = torch.empty(r, -(-cols // 16) * 16, dtype=torch.int8, device="cuda")[:, :cols]
        return t.copy_(torch.randint(-127, 128, (r, cols), generator=g, device="cuda"))

    def scales(n):
        return torch.rand(n, generator=g, device="cuda") * 0.03 + 1e-3
    return whole(rows), scales(rows), whole(outs), scales(outs)


def _run(cats, x, sx, w, sw, kind):
    out, st = torch.full((x.shape[0], w.shape[0]), float("nan"), dtype=kind, device="cuda"), cats.new_status()
    cats.cats_linear_i8(x, sx, cats.pack_weights_i8(w), sw, out, st)
    assert int(st.item()) == 0
    return out


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,outs", SIZES)
def test_every_element(cats, rows, cols, outs, kind):
    """The output starts as NaN: an element that is left out is found."""
    p = _problem(rows, cols, outs, 100 + rows)
    i8_strict.product(_run(cats, *p, kind), *p)


@pytest.mark.parametrize("rows,cols,outs", KERNELS)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_row_and_channel(cats, rows, cols, outs, value):
    x, sx, w, sw = _problem(rows, cols, outs, 7)
    t, n = rows * 2 // 3, outs * 3 // 5
    sx[t], sw[n] = value, value
    out = _run(cats, x, sx, w, sw, torch.float32)
    assert not torch.isfinite(out[t]).any() and not torch.isfinite(out[:, n]).any()
    rows_left = [i for i in range(rows) if i != t]
    outs_left = [i for i in range(outs) if i != n]
    if rows_left:
        i8_strict.product(out[rows_left][:, outs_left], x[rows_left], sx[rows_left], w[outs_left], sw[outs_left])
