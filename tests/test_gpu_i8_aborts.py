"""The 8-bit product after a bounded wait has run out: no copy and no MMA of a CTA is in flight when it goes away.

Nothing is provoked but the end of waits, by the host's order: a copy that is withheld, and warps that give up while everything is
on its way as usual."""
import pytest
import torch

import i8_reference as ref

pytestmark = pytest.mark.gpu

# whole tiles, one and several per SM; tiles shared by a cluster; CTA pairs, one and several tiles per pair
SIZES = [(64, 4096, 12288), (37, 1024, 50000), (64, 11008, 4096), (128, 11008, 4096), (300, 512, 2000), (1000, 2048, 4096), (3000, 1024, 8192)]
TIMEOUT = -6


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _problem(cats, rows, cols, outs):
    g = torch.Generator(device="cuda").manual_seed(rows + cols + outs)

    def whole(r, c):
        return torch.randint(-127, 128, (r, c), generator=g, device="cuda", dtype=torch.int8)

    def scales(n):
        return torch.rand(n, generator=g, device="cuda") * 0.03 + 1e-3
    x, w, sx, sw = whole(rows, cols), whole(outs, cols), scales(rows), scales(outs)
    packed, st = cats.pack_weights_i8(w), cats.new_status()
    want = torch.empty(rows, outs, device="cuda")
    cats.cats_linear_i8(x, sx, packed, sw, want, st)
    ref.check_linear(want, ref.linear(x, sx, w, sw))
    assert torch.isfinite(want).all() and int(st.item()) == 0
    return (x, sx, packed, sw), want, st


@pytest.mark.parametrize("rows,cols,outs", SIZES)
def test_a_withheld_copy_is_waited_for(cats, rows, cols, outs):
    """The wait for the last copy of x expires after 2 ms, long after every copying warp has issued its last stage.  The announced
    copies are then waited for, 10 ms at most: with one that never comes the call takes those 10 ms too."""
    args, want, st = _problem(cats, rows, cols, outs)
    out = torch.empty_like(want)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    cats.wait_limit_ns(2_000_000)
    try:
        cats.inject_fault(3)
        begin.record()
        cats.cats_linear_i8(*args, out, st)
        end.record()
        torch.cuda.synchronize()
    finally:
        cats.inject_fault(0)
        cats.wait_limit_ns(0)
    assert int(st.item()) == TIMEOUT
    assert begin.elapsed_time(end) >= 2 + 10 - 0.5      # the timer that the limits are read from steps by up to 32 us
    st.zero_()
    cats.cats_linear_i8(*args, out, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and torch.equal(out, want)


@pytest.mark.parametrize("rows,cols,outs", SIZES)
def test_giving_up_while_copies_are_under_way(cats, rows, cols, outs):
    """The MMA warps give up before their first wait, the copying warps when the ring is full and nothing empties it: they stop at different
    stages, the second CTA of a pair 2 ms after the first.  The call returns well before the 10 ms that are kept for copies
    that never come, so every barrier told that its copies had landed; it writes nothing beside its output, and the kernel that takes
    its SMs over next computes what it always does."""
    args, want, st = _problem(cats, rows, cols, outs)
    g = torch.Generator(device="cuda").manual_seed(1)
    a, b = torch.randn(2048, 2048, generator=g, device="cuda").bfloat16(), torch.randn(2048, 2048, generator=g, device="cuda").bfloat16()
    product = a @ b
    buf = torch.full((rows + 2, outs), 3.0, device="cuda")
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(5):
        st.zero_()
        cats.wait_limit_ns(2_000_000)
        try:
            cats.inject_fault(4)
            begin.record()
            cats.cats_linear_i8(*args, buf[1:-1], st)
            end.record()
            after = a @ b
            torch.cuda.synchronize()
        finally:
            cats.inject_fault(0)
            cats.wait_limit_ns(0)
        assert int(st.item()) == TIMEOUT and torch.equal(after, product)
        assert (buf[0] == 3).all() and (buf[-1] == 3).all()
        assert begin.elapsed_time(end) < 8
    st.zero_()
    cats.cats_linear_i8(*args, buf[1:-1], st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and torch.equal(buf[1:-1], want)
