"""Kernels of the 8-bit path start while the kernel in front of them still writes their inputs.  The read-only data path (__ldg, or
a load that the compiler may turn into one because of const __restrict__) is defined for data that nobody writes while the kernel
runs, so no kernel that waits with griddepcontrol.wait may use it."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_11186_b200", "csrc")


def _code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def _functions(code):
    """(name, text) of everything at brace depth zero or one that ends with a brace at that depth."""
    for m in re.finditer(r"__global__|__device__", code):
        start = code.find("{", m.start())
        depth, i = 0, start
        while True:
            depth += {"{": 1, "}": -1}.get(code[i], 0)
            i += 1
            if depth == 0:
                break
        head = code[m.start():start]
        name = re.findall(r"(\w+)\s*\(", head)
        yield (name[-1] if name else "?"), code[m.start():i]


@pytest.mark.parametrize("source", ["cats_i8_rows.cu", "cats_i8_linear.cu"])
def test_no_read_only_loads_behind_a_programmatic_wait(source):
    functions = list(_functions(_code(source)))
    waits = [n for n, text in functions if text.startswith("__global__") and "pdl_wait()" in text]
    assert waits, "the kernels were not found"
    plain = {n for n, text in functions if text.startswith("__global__") and "pdl_wait()" not in text}      # ordered as ever: may use it
    bad = [n for n, text in functions if n not in plain and ("__ldg(" in text or "__restrict__" in text or "ld.global.nc" in text)]
    assert not bad, bad
