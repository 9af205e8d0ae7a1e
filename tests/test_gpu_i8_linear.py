"""The 8-bit product against whole-number sums in 64 bits."""
import pytest
import torch

import i8_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _whole(rows, cols, seed, lo=-127, hi=127):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.int8, device="cuda")[:, :cols]
    return q.copy_(torch.randint(lo, hi + 1, (rows, cols), generator=g, device="cuda"))


def _scales(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.rand(n, generator=g, device="cuda") * 0.03 + 1e-3


def _run(cats, x, sx, w, sw, dtype, pad=0):
    rows, outs = x.shape[0], w.shape[0]
    buf = torch.full((rows + 2, outs + pad), 3.0, dtype=dtype, device="cuda")
    out = buf[1:rows + 1, :outs]
    st = cats.new_status()
    cats.cats_linear_i8(x, sx, cats.pack_weights_i8(w), sw, out, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert (buf[0] == 3).all() and (buf[-1] == 3).all() and (buf[:, outs:] == 3).all()      # nothing beside the output
    return out


# (tokens, columns, channels): one of everything, ragged everywhere, tree sizes, several token blocks, several tiles per SM
SIZES = [(1, 1, 1), (1, 16, 8), (1, 128, 16), (2, 127, 15), (3, 129, 17), (8, 256, 768), (9, 688, 256), (16, 4096, 100), (17, 1000, 1001),
         (37, 256, 1376), (64, 4096, 4096), (77, 5120, 1536), (128, 11008, 4096), (127, 640, 40000), (129, 384, 300), (200, 2048, 512),
         (256, 256, 256), (300, 512, 2000), (513, 1024, 1111), (1000, 128, 8000), (1, 11008, 4096), (5, 40000, 48), (2500, 320, 2500),
         (257, 2048, 12296), (1024, 4096, 4096), (2049, 200, 5000), (4093, 130, 300),
         (700, 2001, 5003), (1500, 1000, 6001), (391, 8000, 3500), (2047, 1111, 7777), (513, 6000, 2000),
         (1, 4096, 22016), (1, 131, 5003), (3, 4096, 4100), (4, 1000, 77), (4, 8192, 4096), (2, 17, 9)]


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,outs", SIZES)
def test_product(cats, rows, cols, outs, kind):
    x, w, sx, sw = _whole(rows, cols, 1), _whole(outs, cols, 2), _scales(rows, 3), _scales(outs, 4)
    ref.check_linear(_run(cats, x, sx, w, sw, kind), ref.linear(x, sx, w, sw))


@pytest.mark.parametrize("pad", [1, 4, 8])
def test_output_strides(cats, pad):
    x, w, sx, sw = _whole(33, 300, 5), _whole(96, 300, 6), _scales(33, 7), _scales(96, 8)
    for kind in (torch.float32, torch.bfloat16):
        ref.check_linear(_run(cats, x, sx, w, sw, kind, pad), ref.linear(x, sx, w, sw))


def test_input_rows_of_a_wider_buffer(cats):
    """Columns behind the matrix hold other data: they must not enter the sums."""
    wide = _whole(70, 512, 9)
    x, sx = wide[:, 32:32 + 200], _scales(70, 10)
    w, sw = _whole(500, 232, 11)[:, 16:216], _scales(500, 12)
    ref.check_linear(_run(cats, x, sx, w, sw, torch.float32), ref.linear(x, sx, w, sw))


def test_largest_sums(cats):
    """Every product -128 * -128 at the longest row: the sum is 2^31 - 2^14, still exact."""
    cols = 131071
    x = torch.full((2, 131072), -128, dtype=torch.int8, device="cuda")[:, :cols]
    w = torch.full((24, 131072), -128, dtype=torch.int8, device="cuda")[:, :cols]
    w[1] = 127
    one = torch.ones(24, device="cuda")
    ref.check_linear(_run(cats, x, one[:2], w, one, torch.float32), ref.linear(x, one[:2], w, one))


def test_a_row_that_is_not_finite_stays_one_row(cats):
    x, w, sx, sw = _whole(40, 256, 13), _whole(64, 256, 14), _scales(40, 15), _scales(64, 16)
    sx[7] = float("nan")
    out = _run(cats, x, sx, w, sw, torch.float32)
    assert torch.isnan(out[7]).all()
    keep = [i for i in range(40) if i != 7]
    ref.check_linear(out[keep], ref.linear(x[keep], sx[keep], w, sw))


def test_same_bits_every_time_and_on_other_streams(cats):
    x, w, sx, sw = _whole(64, 4096, 17), _whole(4096, 4096, 18), _scales(64, 19), _scales(4096, 20)
    packed, st = cats.pack_weights_i8(w), cats.new_status()
    want = torch.empty(64, 4096, device="cuda")
    cats.cats_linear_i8(x, sx, packed, sw, want, st)
    outs = [torch.empty(64, 4096, device="cuda") for _ in range(8)]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):                        # several calls in flight at once: they share nothing
        with torch.cuda.stream(streams[i % 4]):
            cats.cats_linear_i8(x, sx, packed, sw, o, st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs) and int(st.item()) == 0


def test_several_threads_at_once(cats):
    """Four host threads, a stream each, different sizes (few tokens, whole tiles, clusters, pairs): each gets its own bits."""
    import threading
    jobs = []
    for i, (rows, cols, outs) in enumerate([(1, 4096, 4096), (64, 1024, 4096), (64, 11008, 2048), (700, 2048, 4096)]):
        x, w, sx, sw = _whole(rows, cols, 40 + i), _whole(outs, cols, 50 + i), _scales(rows, 60 + i), _scales(outs, 70 + i)
        jobs.append((x, sx, cats.pack_weights_i8(w), sw, _run(cats, x, sx, w, sw, torch.float32).clone()))
    wrong = []

    def work(x, sx, packed, sw, want):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            outs, st = [torch.empty_like(want) for _ in range(20)], cats.new_status()
            for o in outs:
                cats.cats_linear_i8(x, sx, packed, sw, o, st)
        stream.synchronize()
        if int(st.item()) or not all(torch.equal(o, want) for o in outs):
            wrong.append(tuple(want.shape))
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_captured_and_replayed(cats):
    """norm -> product -> SwiGLU -> product -> norm in a graph, replayed on other inputs: the bits of the calls themselves."""
    T, H, F = 21, 512, 1376
    g = torch.Generator(device="cuda").manual_seed(21)
    resid = torch.randn(T, H, generator=g, device="cuda")
    gain = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    gu, s_gu = cats.quantize_weights_i8(torch.randn(2 * F, H, generator=g, device="cuda") * 0.05)
    dn, s_dn = cats.quantize_weights_i8(torch.randn(H, F, generator=g, device="cuda") * 0.05)
    q, s = cats.new_i8(T, H)
    qa, sa = cats.new_i8(T, F)
    wide, delta, st = torch.empty(T, 2 * F, device="cuda"), torch.empty(T, H, device="cuda"), cats.new_status()
    q_out, s_out = cats.new_i8(T, H)

    def run():
        cats.cats_rmsnorm_i8(resid, None, gain, 1e-5, None, q, s)
        cats.cats_linear_i8(q, s, gu, s_gu, wide, st)
        cats.cats_swiglu_i8(wide, qa, sa)
        cats.cats_linear_i8(qa, sa, dn, s_dn, delta, st)
        cats.cats_rmsnorm_i8(resid, delta, gain, 1e-5, resid, q_out, s_out)
    start = resid.clone()
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in (1, 2):
        start = torch.randn(T, H, generator=g, device="cuda")
        resid.copy_(start)
        run()
        want = [t.clone() for t in (resid, q_out, s_out)]
        resid.copy_(start)
        q_out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((resid, q_out, s_out), want))
    assert int(st.item()) == 0


def test_captured_between_copies_and_on_two_branches(cats):
    """In a graph whose nodes in front are copies, fills and another stream's kernels, not only kernels of this library."""
    T, K, N = 70, 640, 1000
    src = torch.randn(T, K, device="cuda")
    x, out_a, out_b = torch.empty_like(src), torch.empty(T, N, device="cuda"), torch.empty(T, N, device="cuda")
    (qa, sa), (qb, sb) = cats.new_i8(T, K), cats.new_i8(T, K)
    w, sw = cats.quantize_weights_i8(torch.randn(N, K, device="cuda"))
    st, side = cats.new_status(), torch.cuda.Stream()

    def run():
        main = torch.cuda.current_stream()
        x.copy_(src)
        qa.zero_()
        side.wait_stream(main)
        cats.cats_quantize_i8(x, qa, sa)
        with torch.cuda.stream(side):
            cats.cats_quantize_i8(x * -2, qb, sb)
            cats.cats_linear_i8(qb, sb, w, sw, out_b, st)
        out_a.fill_(7)
        cats.cats_linear_i8(qa, sa, w, sw, out_a, st)
        main.wait_stream(side)
        cats.cats_dequantize_i8(qb, sb, x)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        src.copy_(torch.randn(T, K, device="cuda"))
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (out_a, out_b, x)]
        for t in (out_a, out_b, x):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out_a, out_b, x), want))
    assert int(st.item()) == 0


@pytest.mark.parametrize("rows,cols,outs", [(64, 4096, 12288), (37, 1024, 50000), (64, 11008, 4096), (1000, 2048, 4096), (3000, 1024, 8192)])
def test_a_wait_that_runs_out(cats, rows, cols, outs):
    """Whole tiles, tiles shared by a cluster, CTA pairs: the last copy of x is announced but withheld by the host's order.  The
    call returns, says so, writes nothing beside its output, and the next call is right."""
    x, w, sx, sw = _whole(rows, cols, 26), _whole(outs, cols, 27), _scales(rows, 28), _scales(outs, 29)
    packed = cats.pack_weights_i8(w)
    want = _run(cats, x, sx, w, sw, torch.float32).clone()
    buf, st = torch.full((rows + 2, outs), 3.0, device="cuda"), cats.new_status()
    cats.wait_limit_ns(2_000_000)
    try:
        cats.inject_fault(3)
        cats.cats_linear_i8(x, sx, packed, sw, buf[1:-1], st)
        torch.cuda.synchronize()
    finally:
        cats.inject_fault(0)
        cats.wait_limit_ns(0)
    assert int(st.item()) == -6 and (buf[0] == 3).all() and (buf[-1] == 3).all()
    st.zero_()
    cats.cats_linear_i8(x, sx, packed, sw, buf[1:-1], st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and torch.equal(buf[1:-1], want)


def test_wrong_shapes_and_types_are_refused(cats):
    x, w, sx, sw = _whole(4, 64, 1), _whole(32, 64, 2), _scales(4, 3), _scales(32, 4)
    p, out, st = cats.pack_weights_i8(w), torch.empty(4, 32, device="cuda"), cats.new_status()
    for bad in (lambda: cats.cats_linear_i8(x[:, :32], sx, cats.pack_weights_i8(_whole(40, 64, 2)), sw, out, st),
                lambda: cats.cats_linear_i8(x, sx[:3], p, sw, out, st), lambda: cats.cats_linear_i8(x, sx, p, sw, out.half(), st),
                lambda: cats.cats_linear_i8(x, sx, p, sw, out[:, :16], st), lambda: cats.cats_linear_i8(x, sx, p, sw.cpu(), out, st)):
        with pytest.raises(ValueError):
            bad()
    off = torch.zeros(4, 80, dtype=torch.int8, device="cuda")
    for bad in (off[:, 8:72], torch.zeros(4, 72, dtype=torch.int8, device="cuda")[:, :64]):     # rows that do not start on 16 bytes
        with pytest.raises(cats.CatsError) as e:
            cats.cats_linear_i8(bad, sx, p, sw, out, st)
        assert e.value.status == -1


def test_weights_past_4_gb(cats):
    """Byte offsets into the packed weights past 2^32, in each of the kernels; the last and some other channels are checked."""
    cols, outs = 12288, 360000
    g = torch.Generator(device="cuda").manual_seed(30)
    w = torch.randint(-127, 128, (outs, cols), generator=g, device="cuda", dtype=torch.int8)
    packed, sw, st = cats.pack_weights_i8(w), _scales(outs, 31), cats.new_status()
    assert packed.numel() > 1 << 32
    some = torch.cat([torch.arange(0, outs, 997, device="cuda"), torch.arange(outs - 600, outs, device="cuda")])
    for rows in (1, 16, 300):
        x, sx = _whole(rows, cols, 32), _scales(rows, 33)
        out = torch.empty(rows, outs, device="cuda")
        cats.cats_linear_i8(x, sx, packed, sw, out, st)
        ref.check_linear(out[:, some], ref.linear(x, sx, w[some], sw[some]))
    assert int(st.item()) == 0


@pytest.mark.parametrize("cols", [64, 640])
def test_outputs_past_2_31_elements(cats, cols):
    rows, outs = 4100, 530000
    x, w, sx, sw, st = _whole(rows, cols, 34), _whole(outs, cols, 35), _scales(rows, 36), _scales(outs, 37), cats.new_status()
    out = torch.empty(rows, outs, dtype=torch.bfloat16, device="cuda")
    assert out.numel() > 1 << 31
    cats.cats_linear_i8(x, sx, cats.pack_weights_i8(w), sw, out, st)
    for some in (torch.arange(0, rows, 411, device="cuda"), torch.arange(rows - 5, rows, device="cuda")):
        ref.check_linear(out[some], ref.linear(x[some], sx[some], w, sw))
    assert int(st.item()) == 0


def test_a_token_does_not_depend_on_its_batch(cats):
    """Whole-number sums have no order: any share of the tokens, whatever tiles it runs in, gives the same bits."""
    x, w, sx, sw = _whole(400, 1536, 22), _whole(2000, 1536, 23), _scales(400, 24), _scales(2000, 25)
    want = _run(cats, x, sx, w, sw, torch.float32)
    for lo, hi in ((0, 1), (5, 12), (100, 164), (37, 165), (130, 400)):
        assert torch.equal(_run(cats, x[lo:hi], sx[lo:hi], w, sw, torch.float32), want[lo:hi])
