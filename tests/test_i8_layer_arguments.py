"""What the binding of the 8-bit layer and of the weight packing refuses before a pointer leaves it.  On the CPU: the current device is
said to be the CPU, and every call here is refused or launches nothing."""
import pytest
import torch

H, D, F = 64, 128, 200


@pytest.fixture()
def cats(monkeypatch):
    from paper_2605_11186_b200 import binding
    monkeypatch.setattr(binding, "_device", lambda: torch.device("cpu"))
    return binding


def _packed(cats, **change):
    def mat(outs, cols):
        n = int(cats.lib.cats_packed_weight_i8_bytes(outs, cols))
        t = torch.zeros(n + 1024, dtype=torch.uint8)
        return t[-t.data_ptr() % 1024:][:n]
    w = {"attn_norm": torch.ones(H, dtype=torch.bfloat16), "mlp_norm": torch.ones(H, dtype=torch.bfloat16),
         "wqkv": mat(3 * D, H), "wo": mat(H, D), "w_gate_up": mat(2 * F, H), "w_down": mat(H, F),
         "s_qkv": torch.ones(3 * D), "s_o": torch.ones(H), "s_gate_up": torch.ones(2 * F), "s_down": torch.ones(H)}
    w.update(change)
    return w


def test_a_layer_that_fits(cats):
    w = _packed(cats)
    s = cats.layer_weights_i8(w)
    assert s.wqkv == w["wqkv"].data_ptr() and s.s_down == w["s_down"].data_ptr()
    # the struct holds addresses: it keeps the tensors behind them
    address = s.s_down
    del w
    assert any(t.data_ptr() == address for t in s.tensors)


@pytest.mark.parametrize("change", [
    dict(s_qkv=torch.ones(3 * D - 1)), dict(s_qkv=torch.ones(3 * D + 1)), dict(s_o=torch.ones(H - 1)), dict(s_gate_up=torch.ones(2 * F - 16)),      # (one channel less is a layer of its own: the packed matrices are padded)
   
    dict(s_gate_up=torch.ones(2 * F - 1)), dict(s_down=torch.ones(H + 8)), dict(s_o=torch.ones(H, dtype=torch.bfloat16)),
    dict(s_o=torch.ones(2 * H)[::2]), dict(attn_norm=torch.ones(H)), dict(mlp_norm=torch.ones(H - 8, dtype=torch.bfloat16)),
    dict(mlp_norm=None), dict(wqkv=torch.zeros(1024, dtype=torch.uint8)), dict(wo=torch.zeros(1024, dtype=torch.int8)),
    dict(w_down=torch.zeros(64 * 256 - 1, dtype=torch.uint8)), dict(s_down=torch.ones(H, device="meta"))])
def test_a_layer_that_does_not_fit_is_refused(cats, change):
    with pytest.raises(ValueError):
        cats.layer_weights_i8(_packed(cats, **change))


def test_a_missing_weight_is_refused(cats):
    w = _packed(cats)
    del w["s_o"]
    with pytest.raises(ValueError):
        cats.layer_weights_i8(w)


def _call(cats, cfg=None, **change):
    T, P, max_seq = 5, 3, 16
    cfg = cfg or cats.ModelCfg(H, 2, D // 2, F, 256, 1, max_seq, 1e-5, 10000.0)
    a = dict(w=cats.layer_weights_i8(_packed(cats)), resid=torch.zeros(T, H), kcache=torch.zeros(max_seq, D, dtype=torch.bfloat16),
             vcache=torch.zeros(max_seq, D, dtype=torch.bfloat16), mask=torch.zeros(T, 2, dtype=torch.int64),
             pos=torch.zeros(T, dtype=torch.int32), T=T, prefix_len=P, ws=torch.zeros(8, dtype=torch.uint8), status=torch.zeros(1, dtype=torch.int32))
    a.update(change)
    return cats.cats_verify_layer_i8(cfg, a["w"], a["resid"], a["kcache"], a["vcache"], a["mask"], a["pos"], a["T"], a["prefix_len"], a["ws"], a["status"])


@pytest.mark.parametrize("change", [
    dict(resid=torch.zeros(4, H)), dict(resid=torch.zeros(5, H, dtype=torch.bfloat16)), dict(kcache=torch.zeros(15, D, dtype=torch.bfloat16)),
    dict(vcache=torch.zeros(16, D - 8, dtype=torch.bfloat16)), dict(kcache=torch.zeros(16, D)), dict(mask=torch.zeros(4, 2, dtype=torch.int64)),
    dict(mask=torch.zeros(5, 2, dtype=torch.int32)), dict(pos=torch.zeros(4, dtype=torch.int32)), dict(pos=torch.zeros(5, dtype=torch.int64)),
    dict(status=torch.zeros(0, dtype=torch.int32)), dict(resid=torch.zeros(H, 5).t()), dict(pos=torch.zeros(5, dtype=torch.int32, device="meta")),
    dict(ws=torch.zeros(8, dtype=torch.uint8, device="meta")), dict(resid=None)])
def test_operands_of_the_layer_that_do_not_fit_are_refused(cats, change):
    with pytest.raises(ValueError):
        _call(cats, **change)


@pytest.mark.parametrize("change", [dict(hidden=128), dict(ffn=208), dict(n_heads=4)])
def test_weights_of_another_model_are_refused(cats, change):
    cfg = cats.ModelCfg(H, 2, D // 2, F, 256, 1, 16, 1e-5, 10000.0)
    for k, v in change.items():
        setattr(cfg, k, v)
    with pytest.raises(ValueError):
        _call(cats, cfg)


def test_what_fits_reaches_the_library(cats, monkeypatch):
    """The workspace here is too small, which is the library's to say: status -4, nothing launched."""
    monkeypatch.setattr(cats, "_stream", lambda: None)
    with pytest.raises(cats.CatsError) as e:
        _call(cats)
    assert e.value.status == -4 and cats.lib.cats_last_launch_count() == 0


@pytest.mark.parametrize("w", [torch.zeros(4, 64, dtype=torch.int8, device="meta"), torch.zeros(4, 64), torch.zeros(64, dtype=torch.int8),
                               torch.zeros(64, 4, dtype=torch.int8).t(), torch.zeros(4, 64, dtype=torch.uint8), None])
def test_packing_refuses(cats, w):
    with pytest.raises(ValueError):
        cats.pack_weights_i8(w)


def test_a_matrix_of_another_device_is_not_packed():
    from paper_2605_11186_b200 import binding
    with pytest.raises(ValueError):
        binding.pack_weights_i8(torch.zeros(4, 64, dtype=torch.int8))
