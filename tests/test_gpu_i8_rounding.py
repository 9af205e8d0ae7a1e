"""What the row operators round to: q = rint(127 y / a), ties to even, wherever y itself is exact.

For a bf16 row, or an fp32 row of values with eight significant bits, y = Y 2^i and a = A 2^j with whole numbers Y, A below 256
and i <= j.  If 127 y / a is not a half-integer h, then 127 y / a - h = (254 Y - 2 h A 2^(j-i)) 2^(i-j) / (2 A) with a whole number
in brackets that is not zero, so it is at least 2^(i-j) / 510, and 127 y / a <= 127 * 255 / 128 * 2^(i-j): the distance from a tie
is at least 2^-17 of the quotient.  fp32 (2^-24) and fp64 both tell such quotients from ties, which both hold exactly: the
rounded quotient has one right value, equal in both.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

# a row of one warp, one, two and four vectors per thread, rows too long for the registers; whole and ragged; few and many rows
SHAPES = [(1, 8), (3, 7), (65, 64), (9, 1000), (64, 4096), (700, 4096), (40, 4100), (33, 5120), (2, 11008), (300, 11008), (5, 13825),
          (2, 16392), (3, 40000)]


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _rows(rows, cols, seed, spread=0.0):
    """Normal bf16 rows; spread: their sizes vary by up to 2^spread either way."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    size = torch.exp2(torch.round((torch.rand(rows, 1, generator=g, device="cuda") * 2 - 1) * spread))
    return (x * size).bfloat16()


def _want(y):
    """(q, scale) in 64 bits.  A quotient of two fp32 values rounded to fp64 and then to fp32 is rounded correctly (53 >= 2 * 24 + 2)."""
    a = y.double().abs().amax(1).clamp_min(2.0 ** -100)
    return torch.round(127.0 * y.double() / a[:, None]).to(torch.int8), (a / 127.0).float()


def test_such_rows_have_ties(cats):
    """What the tests below are about occurs in their inputs: about one element of a normal bf16 row in a thousand is a tie."""
    y = _rows(64, 4096, 1).double()
    t = 127.0 * y / y.abs().amax(1, keepdim=True)
    assert ((t - t.floor()) == 0.5).sum().item() > 64


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize(cats, rows, cols, kind):
    for seed, spread in ((1, 0.0), (2, 60.0)):
        y = _rows(rows, cols, seed, spread)
        q, scale = cats.new_i8(rows, cols)
        cats.cats_quantize_i8(y.to(kind), q, scale)
        want, want_scale = _want(y)
        assert torch.equal(q, want), (q != want).sum().item()
        assert torch.equal(scale, want_scale)


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_of_exact_rows(cats, rows, cols):
    """The row factor cancels in 127 y / a, so with a gain of powers of two the norm of a bf16 row is rounded from the row itself."""
    x = _rows(rows, cols, 3)
    gain = torch.exp2((torch.arange(cols, device="cuda") % 3).float()).bfloat16()
    q, scale = cats.new_i8(rows, cols)
    for kind in (torch.bfloat16, torch.float32):
        cats.cats_rmsnorm_i8(x.to(kind), None, gain, 1e-5, None, q, scale)
        want, _ = _want(x.double() * gain.double())
        assert torch.equal(q, want), (q != want).sum().item()


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_full_precision_rows(cats, rows, cols):
    """fp32 rows: the quotient is fp32, 127 y and its division rounded once each (2^-24 of at most 127 apiece), so nothing further than
    127 * 2^-23 from a tie may go the other way.  (The correction of the quotient leaves 2^-46 of it, covered by the 1.01.)"""
    g = torch.Generator(device="cuda").manual_seed(4)
    y = torch.randn(rows, cols, generator=g, device="cuda")
    q, scale = cats.new_i8(rows, cols)
    cats.cats_quantize_i8(y, q, scale)
    want, want_scale = _want(y)
    t = 127.0 * y.double() / y.double().abs().amax(1, keepdim=True)
    near = ((t - t.floor()) - 0.5).abs() <= 1.01 * 127 * 2.0 ** -23
    assert torch.equal(torch.where(near, want, q), want) and torch.equal(scale, want_scale)


def test_largest_and_smallest_rows(cats):
    """Rows at both ends of the exponent range, where 127 y overflows and y / 2 is subnormal."""
    for size in (2.0 ** 126, 2.0 ** 100, 2.0 ** -60, 2.0 ** -92, 2.0 ** -104):
        y = (_rows(20, 600, 5).clamp(-1.99, 1.99).double() * size).bfloat16()
        for kind in (torch.bfloat16, torch.float32):
            q, scale = cats.new_i8(20, 600)
            cats.cats_quantize_i8(y.to(kind), q, scale)
            want, want_scale = _want(y)
            assert torch.equal(q, want) and torch.equal(scale, want_scale), size


def test_weights(cats):
    """A weight matrix goes through the same rounding once and for all."""
    w = (_rows(300, 1000, 6).float() * 0.02).bfloat16()
    _, scale = cats.quantize_weights_i8(w)
    want, want_scale = _want(w)
    assert torch.equal(scale, want_scale)
    q, _ = cats.new_i8(300, 1000)
    cats.cats_quantize_i8(w, q, scale)
    assert torch.equal(q, want)
