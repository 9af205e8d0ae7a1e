"""The paged-cache and sampling kernels, too, start while the kernel in front of them writes their inputs: no read-only loads (see
test_i8_coherent_loads.py)."""
import pytest

from test_i8_coherent_loads import _code, _functions


@pytest.mark.parametrize("source,kernels", [("cats_paged.cu", 2), ("cats_paged_attn.cu", 1), ("cats_sample.cu", 1)])
def test_no_read_only_loads_behind_a_programmatic_wait(source, kernels):
    functions = list(_functions(_code(source)))
    waits = [n for n, text in functions if text.startswith("__global__") and "pdl_wait()" in text]
    assert len(waits) == kernels
    bad = [n for n, text in functions if "__ldg(" in text or "__restrict__" in text or "ld.global.nc" in text]
    assert not bad, bad


@pytest.mark.parametrize("source", ["cats_paged.cu", "cats_paged_attn.cu", "cats_sample.cu"])
def test_no_memory_is_touched_before_the_wait(source):
    """Every one of these calls is one launch that may overlap what runs before it: nothing but parameters and shared memory until the wait."""
    for name, text in _functions(_code(source)):
        if text.startswith("__global__"):
            head = text[text.index("{"):text.index("pdl_wait()")]
            assert "p." not in head.replace("p.vocab", "") and "r." not in head and "c." not in head and "a." not in head, (name, head)
