"""cats_verify_layer_i8 stage by stage: every stage of the layer against the public call of the same operator on the layer's own inputs,
bit for bit, and the one stage that has no call of its own (rotation and KV append) against 64 bits.  No tolerance of one stage
hides a lost scale, head, row or channel of another."""
import numpy as np
import pytest
import torch

import i8_strict
import oracle
from paper_2605_11186_b200 import inputs as gen

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _gain(m, *key):
    return (1 + gen.normal_bf16((m.hidden,), 0.2, "cuda", *key).float()).bfloat16()


def _setup(cats, m, T, P, tag):
    """Everything from the key's own streams: a failure can be repeated."""
    max_seq = P + T + 5
    w = {k: v.cuda() for k, v in gen.make_layer(m, tag, 0, device="cuda").items()}
    w["attn_norm"], w["mlp_norm"] = _gain(m, tag, "attn_norm"), _gain(m, tag, "mlp_norm")
    kc, vc = gen.make_kv_prefix(m, 1, max_seq, P, tag)
    resid = gen.normal_bf16((T, m.hidden), 1.0, "cuda", tag, T, "resid").float()
    _, mask, pos, _ = oracle.build_tree_mask(gen.tree_random(T, 7) if T > 1 else np.array([-1], np.int32), P)
    return dict(w=w, kc=kc[0].cuda(), vc=vc[0].cuda(), resid=resid, mask=torch.from_numpy(mask.view(np.int64)).cuda(),
                pos=torch.from_numpy(pos).cuda(), cfg=cats.model_cfg(m, max_seq, 1))


def _rotated(t, pos, m):
    """fp64 rotation of fp32 [T][n_heads * head_dim], and the size that its fp32 rounding errors are relative to."""
    hd = m.head_dim
    x = t.double().view(len(pos), m.n_heads, 2, hd // 2)
    freq = m.rope_base ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
    ang = (pos.double()[:, None] * freq)[:, None]
    lo, hi = x[:, :, 0], x[:, :, 1]
    c, s = ang.cos(), ang.sin()
    size = lo.abs() + hi.abs()
    return torch.stack([lo * c - hi * s, hi * c + lo * s], 2).reshape(t.shape), torch.stack([size, size], 2).reshape(t.shape)


def _check_rotated(got, want, size):
    """One rounding to bf16 (2^-8); before it cosine and sine, two products and their sum are rounded once each: 3 u of |lo| + |hi|."""
    assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 3.03 * U * size).all()


SHAPES = {"tiny": gen.TINY, "odd": gen.TINY.replace(hidden=320, n_heads=5, head_dim=64, ffn=1000),
          "wide": gen.TINY.replace(hidden=1152, n_heads=9, head_dim=128, ffn=2752), "7b": gen.LLAMA_7B}


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("T,P", [(1, 0), (1, 300), (3, 20), (37, 77), (64, 512), (128, 130)])
def test_every_stage(cats, shape, T, P):
    m, tag = SHAPES[shape], "i8_stages_" + shape
    s = _setup(cats, m, T, P, tag)
    H, D, F, w, cfg = m.hidden, m.n_heads * m.head_dim, m.ffn, s["w"], s["cfg"]
    p = cats.pack_layer_i8(w)
    resid, kc, vc = s["resid"].clone(), s["kc"].clone(), s["vc"].clone()
    ws, st = cats.new_workspace_i8(cfg, T), cats.new_status()
    ws.fill_(0x7F)
    cats.cats_verify_layer_i8(cfg, cats.layer_weights_i8(p), resid, kc, vc, s["mask"], s["pos"], T, P, ws, st)
    at = cats.workspace_i8_layout(cfg, T)

    def buf(name, rows, cols, kind, stride=None):
        size = torch.empty(0, dtype=kind).element_size()
        flat = ws[at[name]:at[name] + rows * (stride or cols) * size].view(kind)
        return flat.view(rows, stride or cols)[:, :cols]

    def new(cols):
        return torch.full((T, cols), float("nan"), device="cuda")
    # norm, QKV projection, rotation and append
    q8, sc = cats.new_i8(T, H)
    cats.cats_rmsnorm_i8(s["resid"], None, w["attn_norm"], m.rms_eps, None, q8, sc)
    qkv = new(3 * D)
    cats.cats_linear_i8(q8, sc, p["wqkv"], p["s_qkv"], qkv, st)
    q, k, v = qkv.split(D, 1)
    _check_rotated(buf("q", T, D, torch.bfloat16), *_rotated(q.contiguous(), s["pos"], m))
    _check_rotated(kc[P:P + T], *_rotated(k.contiguous(), s["pos"], m))
    assert torch.equal(vc[P:P + T], v.bfloat16())
    for cache, before in ((kc, s["kc"]), (vc, s["vc"])):
        assert torch.equal(cache[:P], before[:P]) and torch.equal(cache[P + T:], before[P + T:])
    # attention on the layer's own q and caches
    o = torch.full((T, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    cats.cats_tree_attention(buf("q", T, D, torch.bfloat16).contiguous(), kc, vc, s["mask"], T, P, m.n_heads, m.head_dim, D,
                             float(np.float32(1) / np.sqrt(np.float32(m.head_dim))), o, cats.new_workspace(cfg, T, P), st)
    assert torch.equal(o, buf("o", T, D, torch.bfloat16))
    # O projection; norm with its sum; gate and up; SwiGLU; down; the last sum
    oq, osc = cats.new_i8(T, D)
    cats.cats_quantize_i8(o, oq, osc)
    delta, mid = new(H), new(H)
    cats.cats_linear_i8(oq, osc, p["wo"], p["s_o"], delta, st)
    cats.cats_rmsnorm_i8(s["resid"], delta, w["mlp_norm"], m.rms_eps, mid, q8, sc)
    assert torch.equal(mid, s["resid"] + delta)
    wide = new(2 * F)
    cats.cats_linear_i8(q8, sc, p["w_gate_up"], p["s_gate_up"], wide, st)
    assert torch.equal(wide, buf("wide", T, 2 * F, torch.float32))
    aq, asc = cats.new_i8(T, F)
    cats.cats_swiglu_i8(wide, aq, asc)
    assert torch.equal(aq, buf("x", T, F, torch.int8, at["ldx"])) and torch.equal(asc, buf("scale", 1, T, torch.float32)[0])
    down = new(H)
    cats.cats_linear_i8(aq, asc, p["w_down"], p["s_down"], down, st)
    assert torch.equal(down, buf("delta", T, H, torch.float32))
    assert torch.equal(resid, mid + down) and int(st.item()) == 0
    # and one of the products itself, element by element
    raw, ch = cats.new_i8(H, F)
    cats.cats_quantize_i8(w["w_down"], raw, ch)
    assert torch.equal(ch, p["s_down"])
    i8_strict.product(down, aq, asc, raw, ch)


@pytest.mark.parametrize("shape", ["tiny", "wide", "7b"])
@pytest.mark.parametrize("T,P", [(1, 300), (64, 512)])
def test_eight_bits_against_sixteen(cats, shape, T, P):
    """The layer beside cats_verify_layer on the same bf16 weights.  A row held in 8 bits is off by steps of a / 127, uniformly: h / sqrt(12)
    in the 2-norm with h = a / 127 of a deviation, a <= 5 for rows of a few thousand normal values, gains up to 1.6: h <= 6.3 / 127.
    Eight matrices and rows take part, all independent: (attention) Q, K, V and O with their inputs, (MLP) gate / up and down with
    theirs, at most sqrt(8) h / sqrt(12) = 4.1e-2 of the contribution if each passed on in full, doubled for the products of a gate
    and an up value, both off."""
    m, tag = SHAPES[shape], "i8_against_16_" + shape
    s = _setup(cats, m, T, P, tag)
    st = cats.new_status()
    r8, r16 = s["resid"].clone(), s["resid"].clone()
    cats.cats_verify_layer_i8(s["cfg"], cats.layer_weights_i8(cats.pack_layer_i8(s["w"])), r8, s["kc"].clone(), s["vc"].clone(), s["mask"], s["pos"],
                              T, P, cats.new_workspace_i8(s["cfg"], T), st)
    packed = cats.pack_layer(s["w"])
    cats.cats_verify_layer(s["cfg"], cats.layer_weights(packed), r16, s["kc"].clone(), s["vc"].clone(), s["mask"], s["pos"], T, P,
                           cats.new_workspace(s["cfg"], T, P), st)
    torch.cuda.synchronize()
    part = (r16 - s["resid"]).double()
    err = (r8 - r16).double()
    print("8 against 16 bits, %s T=%d P=%d: %.2e of the layer's contribution" % (shape, T, P, (err.norm() / part.norm()).item()))
    assert int(st.item()) == 0 and (err.norm() / part.norm()).item() < 8.2e-2
    # no channel and no token on its own is off by more than several times that: one that is lost would be off by all of it
    assert (err.norm(dim=1) / part.norm(dim=1)).max().item() < 0.33
    if T >= 64:
        assert (err.norm(dim=0) / part.norm(dim=0)).max().item() < 0.33
