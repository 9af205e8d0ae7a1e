"""One set of buffers used again and again without a synchronisation: every kernel overlaps the one that fills its inputs, and blocks
of a third call may share an SM with those of the first.  Whatever is read has to be what the call in front wrote."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _inputs(n, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    return [torch.randn(rows, cols, generator=g, device="cuda") * 2.0 ** (i % 7 - 3) for i in range(n)]


@pytest.mark.parametrize("rows,cols", [(1, 64), (16, 1000), (64, 4096), (300, 4099), (2000, 512)])
def test_quantize_then_dequantize(cats, rows, cols):
    xs = _inputs(24, rows, cols)
    q, s = cats.new_i8(rows, cols)
    outs = [torch.empty(rows, cols, device="cuda") for _ in xs]
    want = []
    for x in xs:
        cats.cats_quantize_i8(x, q, s)
        torch.cuda.synchronize()
        want.append(q.float() * s[:, None])
    for _ in range(5):
        for x, o in zip(xs, outs):
            cats.cats_quantize_i8(x, q, s)
            cats.cats_dequantize_i8(q, s, o)
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.parametrize("rows,cols,outs", [(1, 512, 256), (4, 4096, 600), (37, 1024, 1000), (128, 2048, 512), (600, 512, 1024)])
def test_quantize_then_product(cats, rows, cols, outs):
    xs = _inputs(16, rows, cols)
    g = torch.Generator(device="cuda").manual_seed(3)
    w, sw = cats.quantize_weights_i8(torch.randn(outs, cols, generator=g, device="cuda"))
    q, s = cats.new_i8(rows, cols)
    st = cats.new_status()
    got, want = [torch.empty(rows, outs, device="cuda") for _ in xs], [torch.empty(rows, outs, device="cuda") for _ in xs]
    for x, o in zip(xs, want):
        cats.cats_quantize_i8(x, q, s)
        torch.cuda.synchronize()
        cats.cats_linear_i8(q, s, w, sw, o, st)
        torch.cuda.synchronize()
    for _ in range(5):
        for x, o in zip(xs, got):
            cats.cats_quantize_i8(x, q, s)
            cats.cats_linear_i8(q, s, w, sw, o, st)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and int(st.item()) == 0


def test_gains_and_channel_scales_written_by_the_call_in_front(cats):
    """Operands that are constant in a model may be an earlier call's output all the same: the dequantised gain of a norm, the channel
    scales that a quantisation of the weights has just written."""
    rows, cols, outs = 24, 2048, 768
    gains, mats, xs = _inputs(12, 1, cols), _inputs(12, outs, cols), _inputs(12, rows, cols)
    gq, gs = cats.new_i8(1, cols)
    gain = torch.empty(1, cols, dtype=torch.bfloat16, device="cuda")
    wq, sw = cats.new_i8(outs, cols)
    packed = torch.empty(cats.pack_weights_i8(wq.zero_()).numel(), dtype=torch.uint8, device="cuda")
    q, s = cats.new_i8(rows, cols)
    st = cats.new_status()

    def run(sync):
        res = []
        for g, m, x in zip(gains, mats, xs):
            out = torch.empty(rows, outs, device="cuda")
            packed.copy_(cats.pack_weights_i8(wq))                      # the weights as they are; their scales change below
            cats.cats_quantize_i8(g, gq, gs)
            cats.cats_dequantize_i8(gq, gs, gain)
            if sync:
                torch.cuda.synchronize()
            cats.cats_rmsnorm_i8(x, None, gain[0], 1e-5, None, q, s)
            cats.cats_quantize_i8(m, wq, sw)
            if sync:
                torch.cuda.synchronize()
            cats.cats_linear_i8(q, s, packed, sw, out, st)
            if sync:
                torch.cuda.synchronize()
            res += [out, q.clone(), s.clone()]
        torch.cuda.synchronize()
        return res
    wq.zero_()
    want = run(True)
    for _ in range(3):
        wq.zero_()
        assert all(torch.equal(a, b) for a, b in zip(run(False), want)) and int(st.item()) == 0
