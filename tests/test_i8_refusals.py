"""What the 8-bit entry points refuse, through the C ABI and without a GPU: a refused call launches nothing."""
import ctypes as C

import pytest

A = 1 << 20                     # an address that is aligned to anything; never dereferenced
F32, BF16 = 0, 1
INVALID, UNSUPPORTED, WORKSPACE = -1, -3, -4


@pytest.fixture(scope="module")
def lib():
    from paper_2605_11186_b200 import binding
    return binding.lib


def test_packed_size(lib):
    size = lib.cats_packed_weight_i8_bytes
    assert size(1, 1) == 1024
    assert size(8, 128) == 1024 and size(9, 128) == 2048 and size(8, 129) == 2048
    assert size(22016, 4096) == 22016 * 4096
    assert size(0, 128) == 0 and size(8, 0) == 0 and size(8, 131072) == 0 and size(-1, 8) == 0


@pytest.mark.parametrize("change", [dict(x=None), dict(t=7), dict(ldx=63), dict(rows=-1), dict(cols=0), dict(q=None), dict(ldq=63),
                                    dict(s=None), dict(x=A + 2), dict(s=A + 2)])
def test_quantize(lib, change):
    a = dict(x=A, t=F32, ldx=64, rows=2, cols=64, q=A, ldq=64, s=A)
    a.update(change)
    assert lib.cats_quantize_i8(a["x"], a["t"], a["ldx"], a["rows"], a["cols"], a["q"], a["ldq"], a["s"], None) == INVALID
    assert lib.cats_last_launch_count() == 0


@pytest.mark.parametrize("change", [dict(q=None), dict(s=None), dict(o=None), dict(t=2), dict(ldq=63), dict(ldo=63), dict(rows=-2),
                                    dict(cols=0), dict(o=A + 1)])
def test_dequantize(lib, change):
    a = dict(q=A, ldq=64, s=A, rows=2, cols=64, o=A, t=BF16, ldo=64)
    a.update(change)
    assert lib.cats_dequantize_i8(a["q"], a["ldq"], a["s"], a["rows"], a["cols"], a["o"], a["t"], a["ldo"], None) == INVALID


@pytest.mark.parametrize("change", [dict(x=None), dict(xt=3), dict(ldr=63), dict(dt=9), dict(ldd=10), dict(d=A + 2), dict(g=None),
                                    dict(g=A + 1), dict(eps=-1.0), dict(eps=float("nan")), dict(ldo=63), dict(o=A + 2), dict(ldq=63),
                                    dict(s=None), dict(q=None), dict(o=A, x=A, ldo=128), dict(cols=0)])
def test_rmsnorm(lib, change):
    a = dict(x=A, xt=F32, ldr=64, d=A, dt=F32, ldd=64, g=A, eps=1e-5, rows=2, cols=64, o=2 * A, ldo=64, q=A, ldq=64, s=A)
    a.update(change)
    assert lib.cats_rmsnorm_i8(a["x"], a["xt"], a["ldr"], a["d"], a["dt"], a["ldd"], a["g"], a["eps"], a["rows"], a["cols"], a["o"],
                               a["ldo"], a["q"], a["ldq"], a["s"], None) == INVALID
    assert lib.cats_last_launch_count() == 0


@pytest.mark.parametrize("change", [dict(x=None), dict(t=2), dict(ld=127), dict(rows=-1), dict(cols=0), dict(q=None), dict(ldq=63), dict(s=None)])
def test_swiglu(lib, change):
    a = dict(x=A, t=BF16, ld=128, rows=2, cols=64, q=A, ldq=64, s=A)
    a.update(change)
    assert lib.cats_swiglu_i8(a["x"], a["t"], a["ld"], a["rows"], a["cols"], a["q"], a["ldq"], a["s"], None) == INVALID


@pytest.mark.parametrize("change,code", [(dict(x=None), INVALID), (dict(x=A + 8), INVALID), (dict(ldx=72), INVALID), (dict(ldx=48), INVALID),
                                         (dict(sx=None), INVALID), (dict(w=None), INVALID), (dict(w=A + 512), INVALID),
                                         (dict(sw=None), INVALID), (dict(rows=-1), INVALID), (dict(cols=0), INVALID),
                                         (dict(outs=0), INVALID), (dict(o=None), INVALID), (dict(o=A + 2), INVALID), (dict(t=5), INVALID),
                                         (dict(ldo=31), INVALID), (dict(st=None), INVALID),
                                         (dict(cols=131072, ldx=131072), UNSUPPORTED)])
def test_linear(lib, change, code):
    a = dict(x=A, ldx=64, sx=A, w=A, sw=A, rows=2, cols=64, outs=32, o=A, t=F32, ldo=32, st=A)
    a.update(change)
    assert lib.cats_linear_i8(a["x"], a["ldx"], a["sx"], a["w"], a["sw"], a["rows"], a["cols"], a["outs"], a["o"], a["t"], a["ldo"],
                              a["st"], None) == code
    assert lib.cats_last_launch_count() == 0


def test_pack(lib):
    assert lib.cats_pack_weights_i8(None, 64, 8, 64, A, None) == INVALID
    assert lib.cats_pack_weights_i8(A, 63, 8, 64, A, None) == INVALID
    assert lib.cats_pack_weights_i8(A, 64, 8, 64, A + 512, None) == INVALID
    assert lib.cats_pack_weights_i8(A, 64, 0, 64, A, None) == INVALID


def test_sizes_that_are_not_supported(lib):
    n = 131072
    assert lib.cats_quantize_i8(A, F32, n, 2, n, A, n, A, None) == UNSUPPORTED
    assert lib.cats_dequantize_i8(A, n, A, 2, n, A, F32, n, None) == UNSUPPORTED
    assert lib.cats_rmsnorm_i8(A, F32, n, None, F32, 0, A, 1e-5, 2, n, None, 0, A, n, A, None) == UNSUPPORTED
    assert lib.cats_swiglu_i8(A, F32, 2 * n, 2, n, A, n, A, None) == UNSUPPORTED
    big = (1 << 30) + 1
    assert lib.cats_linear_i8(A, 64, A, A, A, big, 64, 8, A, F32, 8, A, None) == UNSUPPORTED
    assert lib.cats_linear_i8(A, 64, A, A, A, 2, 64, big, A, F32, big, A, None) == UNSUPPORTED
    assert lib.cats_packed_weight_i8_bytes(big, 64) == 0
    assert lib.cats_last_launch_count() == 0


def test_no_rows_is_no_work(lib):
    """Zero rows: accepted, nothing launched, no pointer looked at."""
    assert lib.cats_quantize_i8(None, F32, 64, 0, 64, None, 64, None, None) == 0
    assert lib.cats_dequantize_i8(None, 64, None, 0, 64, None, F32, 64, None) == 0
    assert lib.cats_rmsnorm_i8(None, F32, 64, None, F32, 0, None, 1e-5, 0, 64, None, 0, None, 64, None, None) == 0
    assert lib.cats_swiglu_i8(None, F32, 128, 0, 64, None, 64, None, None) == 0
    assert lib.cats_linear_i8(None, 64, None, None, None, 0, 64, 32, None, F32, 32, None, None) == 0
    assert lib.cats_last_launch_count() == 0


def test_layer(lib):
    from paper_2605_11186_b200 import binding as b
    cfg = b.ModelCfg(256, 4, 64, 688, 1024, 1, 160, 1e-5, 10000.0)
    need = lib.cats_workspace_i8_bytes(C.byref(cfg), 37)
    assert need > 0 and need % 1024 == 0
    assert lib.cats_workspace_i8_bytes(C.byref(cfg), 129) == 0 and lib.cats_workspace_i8_bytes(C.byref(cfg), 0) == 0
    assert lib.cats_workspace_i8_bytes(C.byref(b.ModelCfg(256, 4, 96, 688, 1024, 1, 160, 1e-5, 10000.0)), 4) == 0

    def call(w=None, resid=A, kc=A, vc=A, mask=A, pos=A, T=37, P=77, ws=A, n=need, st=A):
        if w is None:
            w = b.LayerWeightsI8(*[A] * 10)
        return lib.cats_verify_layer_i8(C.byref(cfg), C.byref(w), resid, kc, vc, mask, pos, T, P, ws, n, st, None)
    for bad in (dict(resid=None), dict(kc=None), dict(vc=None), dict(mask=None), dict(pos=None), dict(ws=None), dict(st=None), dict(T=0),
                dict(T=129), dict(P=-1), dict(P=124), dict(P=2 ** 31 - 1), dict(resid=A + 8), dict(kc=A + 8)):
        assert call(**bad) == INVALID, bad
    assert call(n=need - 1) == WORKSPACE and call(ws=A + 512) == WORKSPACE
    for i in range(10):
        fields = [A] * 10
        fields[i] = None
        assert call(w=b.LayerWeightsI8(*fields)) == INVALID, i
        fields[i] = A + 2
        assert call(w=b.LayerWeightsI8(*fields)) == INVALID, i
    assert lib.cats_last_launch_count() == 0
