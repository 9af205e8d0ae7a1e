"""Compile the CUDA library ``libcats.so`` (sm_100a) in-tree with nvcc."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcats.so")
PY_EXT = os.path.join(HERE, "_cats_py.so")
SOURCES = ["cats_api.cu", "cats_small_kernels.cu", "cats_gemm.cu", "cats_attn.cu", "cats_i8_rows.cu", "cats_i8_linear.cu"]
HEADERS = ["cats_common.cuh", "cats_kernels.cuh", os.path.join("..", "..", "include", "cats.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "--shared", "-cudart", "static"]


def _stale(lib=LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def _python_stamp() -> str:
    """What the extension depends on: its sources, the interpreter and the installed torch."""
    import hashlib
    import sysconfig

    import torch
    h = hashlib.sha256()
    for f in (os.path.join(CSRC, "cats_py.cpp"), os.path.join(HERE, "..", "include", "cats.h")):
        with open(f, "rb") as src:
            h.update(src.read())
    h.update(("%s %s %s" % (torch.__version__, torch._C._GLIBCXX_USE_CXX11_ABI, sysconfig.get_config_var("SOABI"))).encode())
    return "cats_py_stamp:" + h.hexdigest()


def build_python(force: bool = False) -> str:
    """The CPython extension that marshals the 8-bit calls' tensors (csrc/cats_py.cpp), for the torch that is installed.  Built if
    there is none that carries the stamp of its sources and that torch (not by the files' times, which a copy may set at will)."""
    import sysconfig

    import torch
    stamp = _python_stamp()
    if not force and os.path.exists(PY_EXT):
        with open(PY_EXT, "rb") as f:
            if stamp.encode() in f.read():
                return PY_EXT
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    tmp = PY_EXT + ".tmp.%d" % os.getpid()
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
                           '-DCATS_PY_STAMP="%s"' % stamp,
                           "-I" + sysconfig.get_paths()["include"], "-I" + os.path.join(root, "include"),
                           "-I" + os.path.join(root, "include", "torch", "csrc", "api", "include"), "-I" + os.path.join(cuda, "include"),
                           os.path.join(CSRC, "cats_py.cpp"), "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
                           "-lc10_cuda", "-o", tmp])
    os.replace(tmp, PY_EXT)
    return PY_EXT


TIMELINE_LIB = os.path.join(HERE, "libcats_timeline.so")


def build(force: bool = False, verbose: bool = False, timeline: bool = False) -> str:
    """timeline: build the measurement variant (``-DCATS_TIMELINE``, see cats_debug_timeline) as libcats_timeline.so."""
    out = TIMELINE_LIB if timeline else LIB
    if not force and not _stale(out):
        return out
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = out + ".tmp.%d" % os.getpid()
    cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + (["-DCATS_TIMELINE"] if timeline else []) + \
        [os.path.join(CSRC, f) for f in SOURCES] + ["-ldl", "-o", tmp]
    subprocess.check_call(cmd)
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
    print(build_python(force=True))
