"""cats_verify_layer_i8 against a layer computed in 64 bits from the same 8-bit weights."""
import numpy as np
import pytest
import torch

import i8_reference as ref
import oracle
from paper_2605_11186_b200 import inputs as gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cats():
    from paper_2605_11186_b200 import binding
    assert torch.cuda.is_available()
    return binding


def _values(y):
    """The values that the rows' 8-bit form stands for, in 64 bits."""
    a, want = ref.held(y)
    return torch.round(want) * (a / 127)[:, None]


def _weight(cats, mats):
    w = torch.cat(mats).cuda()
    q, scale = cats.new_i8(*w.shape)
    cats.cats_quantize_i8(w, q, scale)
    ref.check_held(q, scale, w.double(), 0.0)
    return q.double() * scale.double()[:, None]


def _layer64(cats, m, w, resid, kc, vc, mask, pos, T, P):
    """One layer in 64 bits with the path's rounding points: 8-bit projection inputs; bf16 q, k, v and attention output."""
    D, nh, hd = m.n_heads * m.head_dim, m.n_heads, m.head_dim
    x = resid.double()
    qkv = _values(ref.rmsnorm(x, None, w["attn_norm"].cuda(), m.rms_eps)[1]) @ _weight(cats, [w["wq"], w["wk"], w["wv"]]).t()
    q, k, v = (t.view(T, nh, hd) for t in qkv.split(D, 1))
    freq = m.rope_base ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
    ang = pos.double()[:, None] * freq
    c, s = ang.cos()[:, None], ang.sin()[:, None]

    def rotate(t):
        lo, hi = t.chunk(2, -1)
        return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)
    q, k, v = (t.bfloat16().double() for t in (rotate(q), rotate(k), v))
    keys = torch.cat([kc[:P].double().view(P, nh, hd), k])
    vals = torch.cat([vc[:P].double().view(P, nh, hd), v])
    see = torch.ones(T, P + T, dtype=torch.bool, device="cuda")
    for j in range(T):
        see[:, P + j] = (mask[:, j >> 6] >> (j & 63)) & 1 == 1
    score = torch.einsum("thd,khd->htk", q, keys) / hd ** 0.5
    p = torch.softmax(score.masked_fill(~see, float("-inf")), -1)
    o = torch.einsum("htk,khd->thd", p, vals).reshape(T, D).bfloat16().double()
    x = x + _values(o) @ _weight(cats, [w["wo"]]).t()
    y = _values(ref.rmsnorm(x, None, w["mlp_norm"].cuda(), m.rms_eps)[1])
    act = ref.swiglu(y @ _weight(cats, [w["w_gate"], w["w_up"]]).t())
    return x + _values(act) @ _weight(cats, [w["w_down"]]).t(), k.reshape(T, D), v.reshape(T, D)


SHAPES = {"tiny": gen.TINY, "odd": gen.TINY.replace(hidden=320, n_heads=5, head_dim=64, ffn=1000),
          "wide": gen.TINY.replace(hidden=1152, n_heads=9, head_dim=128, ffn=2752)}


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("T,P", [(1, 0), (1, 300), (37, 77), (64, 512), (128, 130)])
def test_layer(cats, shape, T, P):
    m, tag = SHAPES[shape], "i8_" + shape
    max_seq = P + T + 5
    w = {k: v.cuda() for k, v in gen.make_layer(m, tag, 0).items()}
    w["attn_norm"] = (1 + 0.2 * torch.randn(m.hidden, device="cuda")).bfloat16()
    w["mlp_norm"] = (1 + 0.2 * torch.randn(m.hidden, device="cuda")).bfloat16()
    kc, vc = gen.make_kv_prefix(m, 1, max_seq, P, tag)
    kc, vc = kc[0].cuda(), vc[0].cuda()
    kc0, vc0 = kc.clone(), vc.clone()
    resid = gen.normal_bf16((T, m.hidden), 1.0, "cuda", tag, "resid").float()
    start = resid.clone()
    _, mask, pos, _ = oracle.build_tree_mask(gen.tree_random(T, 7) if T > 1 else np.array([-1], np.int32), P)
    mask, pos = torch.from_numpy(mask.view(np.int64)).cuda(), torch.from_numpy(pos).cuda()
    cfg = cats.model_cfg(m, max_seq, 1)
    packed = cats.pack_layer_i8(w)
    ws, st = cats.new_workspace_i8(cfg, T), cats.new_status()
    cats.cats_verify_layer_i8(cfg, cats.layer_weights_i8(packed), resid, kc, vc, mask, pos, T, P, ws, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    want, k, v = _layer64(cats, m, w, start, kc0, vc0, mask, pos, T, P)
    # the cache: the prefix and the rows behind the tree as they were, the tree's rows rotated and appended.
    assert torch.equal(kc[:P], kc0[:P]) and torch.equal(kc[P + T:], kc0[P + T:])
    assert torch.equal(vc[:P], vc0[:P]) and torch.equal(vc[P + T:], vc0[P + T:])
    # A row's step is a / 127 with a <= 6 deviations (4 of 1152 normal values, gains up to 1.5), so h = 6 / 127 of a deviation.
    # The norm's quotients are within 127 * 2 * 2^-19 = 5e-4 of the 64-bit ones, so at most one in 1e3 of the T * hidden inputs
    # (and a handful where that is less than one) lies that near a tie and comes out one step apart: a relative 2-norm of
    # h sqrt((3 + T hidden / 1e3) / (T hidden)) before and, the weights being independent of it, after the projection.  A bf16
    # tie may then go the other way for what moved: 4e-3 on at most a twentieth of the values, 1e-3.
    n, h = T * m.hidden, 6 / 127
    for got, exp in ((kc[P:P + T], k), (vc[P:P + T], v)):
        assert ((got.double() - exp).norm() / exp.norm()).item() < h * ((3 + n / 1e3) / n) ** 0.5 + 1e-3
    # The layer's contribution.  Wherever two rounded rows part, they differ by at most two independent roundings to steps of h,
    # sqrt(2) h / sqrt(12) in the 2-norm; four rounded inputs on the way: 2 sqrt(2) h / sqrt(12) = 3.9e-2.  A lost scale, head,
    # row or rotation is of the order of 1.
    err = ((resid.double() - want).norm() / (want - start.double()).norm()).item()
    print("layer %s T=%d P=%d: %.2e of its contribution" % (shape, T, P, err))
    assert err < 3.9e-2
    # the same call on a workspace that holds another call's leftovers gives the same bits
    kc2, vc2, resid2 = kc0.clone(), vc0.clone(), start.clone()
    ws.fill_(0x7F)
    cats.cats_verify_layer_i8(cfg, cats.layer_weights_i8(packed), resid2, kc2, vc2, mask, pos, T, P, ws, st)
    torch.cuda.synchronize()
    assert torch.equal(resid2, resid) and torch.equal(kc2, kc) and torch.equal(vc2, vc) and int(st.item()) == 0


def test_a_stack_of_8_bit_layers_to_the_accepted_path(cats):
    """Embedding, two 8-bit layers, the bf16 head, the walk and the compaction, as a decoding cycle runs them."""
    m = gen.TINY
    T, P, max_seq = 16, 64, 96
    model = gen.make_model(m, "i8_stack")
    kc, vc = gen.make_kv_prefix(m, m.n_layers, max_seq, P, "i8_stack")
    kc, vc = kc.cuda(), vc.cuda()
    parent = torch.from_numpy(gen.tree_random(T, 3)).cuda()
    tokens = torch.arange(T, dtype=torch.int32, device="cuda") * 7 % m.vocab
    cfg = cats.model_cfg(m, max_seq)
    st = cats.new_status()
    mask, pos = torch.zeros((T, 2), dtype=torch.int64, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    resid = torch.zeros((T, m.hidden), device="cuda")
    cats.cats_build_tree_mask(parent, P, mask, pos, None, st)
    cats.cats_embed_tokens(model["embed"].cuda(), tokens, resid, st)
    want = resid.clone()
    ws8, ws = cats.new_workspace_i8(cfg, T), cats.new_workspace(cfg, T, P)
    for l in range(m.n_layers):
        w = {k: v.cuda() for k, v in model["layers"][l].items()}
        packed = cats.pack_layer_i8(w)
        want, _, _ = _layer64(cats, m, w, want, kc[l].clone(), vc[l].clone(), mask, pos, T, P)
        cats.cats_verify_layer_i8(cfg, cats.layer_weights_i8(packed), resid, kc[l], vc[l], mask, pos, T, P, ws8, st)
    torch.cuda.synchronize()
    assert ((resid.double() - want).norm() / want.norm()).item() < 3e-2
    dm = cats.pack_model({"layers": [], "final_norm": model["final_norm"].cuda(), "w_lm": model["w_lm"].cuda()})
    amax = torch.zeros(T, dtype=torch.int32, device="cuda")
    cats.cats_lm_head_argmax(cfg, dm["final_norm"], dm["w_lm"], resid, T, None, amax, ws, st)
    children = [i for i in range(1, T) if int(parent[i]) == 0]
    tokens[children[0]] = amax[0]                       # one child that the target accepts
    path, out = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    sc = torch.zeros(3, dtype=torch.int32, device="cuda")
    cats.cats_accept_path(parent, tokens, amax, T, path, sc[0:1], out, sc[1:2], st)
    row = kc[:, P + children[0]].clone()
    cats.cats_compact_kv(kc, vc, m.n_layers, max_seq * m.n_heads * m.head_dim, m.n_heads * m.head_dim, P, path, sc[0:1], sc[2:3], None, None, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and int(sc[0]) >= 2 and int(path[1]) == children[0] and torch.equal(kc[:, P + 1], row)
