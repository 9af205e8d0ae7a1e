"""The largest caches: K and V of exactly 2^36 bytes, whose last 16-byte unit is 2^32 - 1.  On the CPU; nothing is launched."""
import ctypes as C

import pytest

from test_paged_refusals import _attend, _kv, b  # noqa: F401


def _span(kind, n_pages, page, row, head, page_size, n_kv, hd):
    """One of several layouts that end exactly `2^36` bytes behind their beginning."""
    return dict(type=kind, n_pages=n_pages, page=page, row=row, head=head, page_size=page_size, n_kv=n_kv, hd=hd, s_page=page_size * n_kv, s_row=1, s_head=page_size)


@pytest.mark.parametrize("kind,elements", [(2, 2 ** 36), (1, 2 ** 35)])
def test_the_limit_itself(b, kind, elements):  # noqa: F811
    """2^36 bytes are accepted (no sequences: nothing is launched), 16 bytes more are not."""
    unit = 16 if kind == 2 else 8
    pages = elements // (16 * 128)
    assert _attend(b, _kv(b, **_span(kind, pages, 16 * 128, 128, 0, 16, 1, 128)), n_seqs=0, table=None, ldq=1024, ldo=1024) == 0
    two = elements - 4 * 16 * 64            # two pages, the second at the very end
    assert _attend(b, _kv(b, **_span(kind, 2, two, 64, 16 * 64, 16, 4, 64)), n_seqs=0, table=None) == 0
    assert _attend(b, _kv(b, **_span(kind, 2, two + unit, 64, 16 * 64, 16, 4, 64)), n_seqs=0, table=None) == -3


@pytest.mark.parametrize("pieces", [4, 8, 16])
def test_rows_that_follow_each_other(b, pieces):  # noqa: F811
    """A tile whose last rows are in the last page and whose next are in page 0 is no run of rows that follow each other."""
    f = b.lib.cats_debug_paged_lies_behind
    f.argtypes = [C.c_uint32] * 3
    top = 2 ** 32
    for lanes_before in (1, 16, 31):
        at0 = top - lanes_before * pieces
        for lane in range(32):
            at = (at0 + lane * pieces) % top            # where the row is if the page behind the last one is page 0
            assert f(at0, at, lane * pieces) == (1 if lane < lanes_before else 0), (lanes_before, lane)
    for at0 in (0, 5 * pieces, top - 32 * pieces):
        for lane in range(32):
            assert f(at0, at0 + lane * pieces, lane * pieces) == 1
            assert f(at0, (at0 + (lane + 1) * pieces) % top, lane * pieces) == 0
