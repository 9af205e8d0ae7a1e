"""The row operators of the 8-bit path (norm, SwiGLU, quantise, dequantise) against their plain forms in 64 bits."""
import pytest
import torch

import i8_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# one vector, a row of one warp, ragged ends, one and several vectors per thread, rows too long for the registers
SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (2, 127), (7, 688), (9, 1024), (4, 1025), (3, 1032), (64, 4096), (130, 4100), (1, 5120),
          (2, 11008), (3, 13825), (2, 16384), (2, 16392), (1, 40000), (1, 131071)]


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _guarded(rows, cols, dtype, pad, fill):
    """A [rows][cols] view inside a larger buffer, and a function that says whether everything around it is as it was."""
    buf = torch.full((rows + 2, cols + pad), fill, dtype=dtype, device="cuda")
    view = buf[1:rows + 1, :cols]

    def intact():
        return bool((buf[0] == fill).all() and (buf[-1] == fill).all() and (buf[1:rows + 1, cols:] == fill).all())
    return view, intact


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_and_back(cats, rows, cols, kind):
    x = _normal((rows, cols), TYPES[kind], 1, 3.0)
    q, scale = cats.new_i8(rows, cols)
    cats.cats_quantize_i8(x, q, scale)
    ref.check_held(q, scale, x.double(), 0.0)
    for out_type in TYPES.values():
        out, intact = _guarded(rows, cols, out_type, 3, 5.0)
        cats.cats_dequantize_i8(q, scale, out)
        want = (q.double() * scale.double()[:, None]).float()         # one rounding to fp32, one more to bf16
        assert torch.equal(out, want.to(out_type)) and intact()


@pytest.mark.parametrize("resid,delta", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", None), ("bf16", None)])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_rmsnorm(cats, rows, cols, resid, delta):
    x = _normal((rows, cols), TYPES[resid], 2, 4.0)
    d = None if delta is None else _normal((rows, cols), TYPES[delta], 3)
    gain = _normal((cols,), torch.bfloat16, 4) + 1
    r, y = ref.rmsnorm(x, d, gain, 1e-5)
    q, scale = cats.new_i8(rows, cols)
    out = torch.empty_like(x)
    cats.cats_rmsnorm_i8(x, d, gain, 1e-5, out, q, scale)
    ref.check_held(q, scale, y, ref.norm_error(cols))
    step = ref.U if resid == "f32" else 2.0 ** -8 * (1 + 2.0 ** -15)
    assert ((out.double() - r).abs() <= step * r.abs()).all()
    # in place, and without the sum: the same bits
    q2, scale2 = cats.new_i8(rows, cols)
    x2 = x.clone()
    cats.cats_rmsnorm_i8(x2, d, gain, 1e-5, x2, q2, scale2)
    assert torch.equal(x2, out) and torch.equal(q2, q) and torch.equal(scale2, scale)
    cats.cats_rmsnorm_i8(x, d, gain, 1e-5, None, q2, scale2)
    assert torch.equal(q2, q) and torch.equal(scale2, scale)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_swiglu(cats, rows, cols, kind):
    x = _normal((rows, 2 * cols), TYPES[kind], 5, 2.0)
    q, scale = cats.new_i8(rows, cols)
    cats.cats_swiglu_i8(x, q, scale)
    ref.check_held(q, scale, ref.swiglu(x), ref.swiglu_error(x))


@pytest.mark.parametrize("offset", [0, 1, 4])
@pytest.mark.parametrize("cols", [96, 100, 4096, 4099])
def test_strides_and_neighbours(cats, cols, offset):
    """Rows of wider buffers, starting on and off the vector boundary; nothing around an output is touched."""
    rows = 5
    wide = _normal((rows, 2 * cols + 29), torch.bfloat16, 6)
    x, gu = wide[:, offset:offset + cols], wide[:, offset:offset + 2 * cols]
    gain = _normal((cols,), torch.bfloat16, 7)
    out, out_ok = _guarded(rows, cols, torch.bfloat16, offset, 9.0)
    for call, y, rel in ((lambda q, s: cats.cats_quantize_i8(x, q, s), x.double(), 0.0),
                         (lambda q, s: cats.cats_swiglu_i8(gu, q, s), ref.swiglu(gu), ref.swiglu_error(gu)),
                         (lambda q, s: cats.cats_rmsnorm_i8(x, x, gain, 1e-6, out, q, s), ref.rmsnorm(x, x, gain, 1e-6)[1], ref.norm_error(cols))):
        q, intact = _guarded(rows, cols, torch.int8, offset + 3, 55)
        scale, scale_ok = _guarded(1, rows, torch.float32, 1, 7.0)
        call(q, scale[0])
        ref.check_held(q, scale[0], y, rel)
        assert intact() and scale_ok()
    assert out_ok() and torch.equal(out, (x.float() * 2).bfloat16())


@pytest.mark.parametrize("cols", [64, 100, 4096, 20000])
def test_rows_of_zeros_tiny_and_not_finite(cats, cols):
    inf, nan = float("inf"), float("nan")
    x = _normal((8, cols), torch.float32, 8)
    x[1] = 0
    x[2] = 0
    x[2, cols // 2] = 1e-38                 # below the smallest maximum: q = 0 at the scale of 2^-100
    x[3, cols - 1] = inf
    x[4, 0] = -inf
    x[5, cols // 3] = nan
    x[6] = 1e-40                            # subnormal
    x[7] = 3e38
    q, scale = cats.new_i8(8, cols)
    cats.cats_quantize_i8(x, q, scale)
    good = [0, 1, 2, 6, 7]
    ref.check_held(q[good], scale[good], x[good].double(), 0.0)
    assert (q[[1, 2, 6]] == 0).all() and (q[7] == 127).all()
    assert torch.isnan(scale[3:6]).all() and (q[3:6] == 0).all()
    out = torch.empty(8, cols, dtype=torch.bfloat16, device="cuda")
    cats.cats_dequantize_i8(q, scale, out)
    assert torch.isnan(out[3:6]).all() and torch.isfinite(out[good]).all()
    # the norm: a row of zeros, and rows that are not finite in the residual stream, the delta or the gain
    gain = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    x[7] = 1.0
    d = torch.zeros_like(x)
    d[7, 5] = inf
    cats.cats_rmsnorm_i8(x, d, gain, 1e-5, None, q, scale)
    ref.check_held(q[:3], scale[:3], ref.rmsnorm(x[:3], None, gain, 1e-5)[1], ref.norm_error(cols))
    assert torch.isnan(scale[[3, 4, 5, 7]]).all() and (q[[3, 4, 5, 7]] == 0).all() and (q[1] == 0).all()
    gain[3] = nan
    cats.cats_rmsnorm_i8(x, None, gain, 1e-5, None, q, scale)
    assert torch.isnan(scale).all() and (q == 0).all()
    # SwiGLU far out on both sides of the gate: silu(-200) = 0, silu(200) = 200
    gu = torch.ones(2, 2 * cols, device="cuda")
    gu[0, :cols] = -200
    gu[1, :cols] = 200
    gu[1, 0] = -200
    cats.cats_swiglu_i8(gu, q[:2], scale[:2])
    assert (q[0] == 0).all() and q[1, 0] == 0 and (q[1, 1:] == 127).all()
    assert abs(scale[1].item() * 127 / 200 - 1) < 1e-6
    gu[1, cols + 2] = nan
    cats.cats_swiglu_i8(gu, q[:2], scale[:2])
    assert torch.isnan(scale[1]) and (q[1] == 0).all() and torch.isfinite(scale[0])


def test_no_rows(cats):
    x = torch.empty(0, 64, device="cuda")
    q, scale = cats.new_i8(0, 64)
    cats.cats_quantize_i8(x, q, scale)
    cats.cats_rmsnorm_i8(x, None, torch.ones(64, dtype=torch.bfloat16, device="cuda"), 1e-5, x, q, scale)
    cats.cats_dequantize_i8(q, scale, x)


def test_offsets_past_32_bits(cats):
    """A row stride that takes the last row past 2^31 elements and 2^32 bytes (three rows of one 5 GB buffer)."""
    stride, cols = (1 << 30) + (1 << 28), 264
    buf = torch.empty(2 * stride + cols, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, cols), (stride, 1))
    x.copy_(_normal((3, cols), torch.bfloat16, 9))
    q, scale = cats.new_i8(3, cols)
    cats.cats_quantize_i8(x, q, scale)
    ref.check_held(q, scale, x.double(), 0.0)
    x.zero_()
    cats.cats_dequantize_i8(q, scale, x)
    assert torch.equal(x, (q.float() * scale[:, None]).bfloat16())


def test_wrong_shapes_and_types_are_refused(cats):
    x = torch.zeros(4, 64, device="cuda")
    q, scale = cats.new_i8(4, 64)
    gain = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: cats.cats_quantize_i8(x.half(), q, scale), lambda: cats.cats_quantize_i8(x, q[:3], scale),
                lambda: cats.cats_quantize_i8(x, q, scale[:3]), lambda: cats.cats_quantize_i8(x.cpu(), q, scale),
                lambda: cats.cats_quantize_i8(x.t(), q.t(), scale), lambda: cats.cats_quantize_i8(x, q.view(torch.uint8), scale),
                lambda: cats.cats_rmsnorm_i8(x, x[:, :32], gain, 1e-5, None, q, scale),
                lambda: cats.cats_rmsnorm_i8(x, None, gain.float(), 1e-5, None, q, scale),
                lambda: cats.cats_rmsnorm_i8(x, None, gain, 1e-5, x.bfloat16(), q, scale),
                lambda: cats.cats_swiglu_i8(x, q, scale), lambda: cats.cats_dequantize_i8(q, scale, x.double())):
        with pytest.raises(ValueError):
            bad()
