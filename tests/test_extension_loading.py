"""The extension that marshals the 8-bit calls (csrc/cats_py.cpp) is needed by those calls only, and is the one its sources and the
installed torch make.  Run in copies of the package, on the CPU: an 8-bit call on CPU tensors is refused by the extension itself."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = "paper_2605_11186_b200"

USE_16_BIT = """
from paper_2605_11186_b200 import binding as b
assert b.lib.cats_version() >= 100 and b.lib.cats_packed_weight_i8_bytes(8, 128) == 1024
"""
USE_8_BIT = """
import torch
from paper_2605_11186_b200 import binding as b
x, (q, s) = torch.zeros(2, 16), b.new_i8(2, 16, device="cpu")
try:
    b.cats_quantize_i8(x, q, s)
except ValueError as e:
    print("refused:", e)
"""


@pytest.fixture()
def copy(tmp_path):
    """The package without its extension; the library itself is the one that is built."""
    from paper_2605_11186_b200 import build
    build.build()
    shutil.copytree(os.path.join(ROOT, PKG), tmp_path / PKG, ignore=shutil.ignore_patterns("*.so", "__pycache__"))
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    os.symlink(build.LIB, tmp_path / PKG / "libcats.so")
    return tmp_path


def _run(where, code, path=None):
    env = dict(os.environ, PYTHONPATH=str(where))
    if path is not None:
        env["PATH"] = str(path)
    return subprocess.run([sys.executable, "-c", code], cwd=where, env=env, capture_output=True, text=True)


def test_without_a_compiler_everything_but_the_8_bit_calls_works(copy):
    empty = copy / "empty"
    empty.mkdir()
    r = _run(copy, USE_16_BIT, empty)
    assert r.returncode == 0, r.stderr
    r = _run(copy, USE_8_BIT, empty)
    assert r.returncode != 0 and "RuntimeError" in r.stderr and "8-bit" in r.stderr.strip().splitlines()[-1], r.stderr


def test_an_extension_of_other_sources_is_built_again(copy):
    """Whatever the files' times say: a checkout or a copy may set them at will."""
    so = copy / PKG / "_cats_py.so"
    r = _run(copy, USE_8_BIT)
    assert r.returncode == 0 and "refused: cats_quantize_i8: x" in r.stdout, r.stderr
    first = so.read_bytes()
    r = _run(copy, USE_8_BIT)
    assert r.returncode == 0 and so.read_bytes() == first          # built once
    header = copy / "include" / "cats.h"
    header.write_text(header.read_text() + "\n/* another interface */\n")
    os.utime(header, (1, 1))
    assert _run(copy, USE_16_BIT).returncode == 0 and so.read_bytes() == first
    r = _run(copy, USE_8_BIT)
    assert r.returncode == 0 and "refused" in r.stdout and so.read_bytes() != first
    so.write_bytes(b"not a library")
    r = _run(copy, USE_8_BIT)
    assert r.returncode == 0 and "refused" in r.stdout, r.stderr
