"""The 8-bit integer operators of a decoder layer, as a user calls them and in their plain form.

rmsnorm_i8   residual + delta, root-mean-square norm, int8 with one scale per token
linear_i8    int8 x int8 product with one scale per token and one per output channel
swiglu_i8    silu(gate) * up, int8 with one scale per token
quantize_i8  int8 with one scale per row (attention output; a weight matrix, one scale per channel)

A row y is held as q = rint(127 y / a), a = max(max|y|, 2^-100), and its scale a / 127.  What is held in 8 bits is
returned as the bf16 values it stands for.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_TINY = 2.0 ** -100
_EPS = 1e-5


def listed():
    return [
        # one-token pass of the draft stage, 7B shape: latency counts
        dict(name="norm 1x4096", op="rmsnorm_i8", rows=1, cols=4096, resid="f32", delta="f32"),
        # a draft tree of 64 nodes, 13B shape
        dict(name="norm 64x5120", op="rmsnorm_i8", rows=64, cols=5120, resid="f32", delta="bf16"),
        # a ragged batch of prompt tokens, residual stream kept in bf16
        dict(name="norm 8191x4096", op="rmsnorm_i8", rows=8191, cols=4096, resid="bf16", delta="bf16"),
        # O projection of a one-token pass
        dict(name="linear 1x4096x4096", op="linear_i8", rows=1, cols=4096, outs=4096, out="bf16"),
        # QKV projection of a ragged tree, 13B shape
        dict(name="linear 77x5120x15360", op="linear_i8", rows=77, cols=5120, outs=15360, out="f32"),
        # gate and up projections of a tree of 64 nodes, 7B shape
        dict(name="linear 64x4096x22016", op="linear_i8", rows=64, cols=4096, outs=22016, out="bf16"),
        # down projection of the largest tree, 7B shape
        dict(name="linear 128x11008x4096", op="linear_i8", rows=128, cols=11008, outs=4096, out="f32"),
        # gate and up projections over a prompt of odd length: bound by the matrix instructions
        dict(name="linear 4093x4096x22016", op="linear_i8", rows=4093, cols=4096, outs=22016, out="bf16"),
        # the activation of a tree of 64 nodes, 7B shape
        dict(name="swiglu 64x11008", op="swiglu_i8", rows=64, cols=11008, x="bf16"),
        # the activation of a prompt, 7B shape
        dict(name="swiglu 4096x11008", op="swiglu_i8", rows=4096, cols=11008, x="bf16"),
        # attention output of a tree of 64 nodes
        dict(name="quantize 64x4096", op="quantize_i8", rows=64, cols=4096, x="bf16"),
        # the stacked gate and up matrices, one scale per channel
        dict(name="quantize 22016x4096", op="quantize_i8", rows=22016, cols=4096, x="bf16"),
    ]


def _log_between(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["rmsnorm_i8", "linear_i8", "linear_i8", "swiglu_i8", "quantize_i8"])
    rows = _log_between(rng, 1, 4096)
    step = rng.choice([1, 8, 64, 128])      # column counts that are odd, in whole vectors, in whole heads
    cols = max(step, _log_between(rng, 64, 13824) // step * step)
    if op == "rmsnorm_i8":
        return dict(op=op, rows=rows, cols=cols, resid=rng.choice(["f32", "bf16"]), delta=rng.choice(["f32", "bf16", "none"]))
    if op == "linear_i8":
        outs = max(step, _log_between(rng, 64, 32000) // step * step)
        return dict(op=op, rows=rows, cols=cols, outs=min(outs, 4093 * 4096 * 22016 // (rows * cols)), out=rng.choice(["f32", "bf16"]))
    return dict(op=op, rows=rows, cols=cols, x=rng.choice(["f32", "bf16"]))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols, op = case["rows"], case["cols"], case["op"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def scales(n):
        return torch.rand(n, generator=g, device="cuda") * 0.02 + 0.002

    def whole(r, c):
        t = torch.empty(r, -(-c // 16) * 16, dtype=torch.int8, device="cuda")[:, :c]     # rows start on 16 bytes
        return t.copy_(normal(r, c).mul_(32).round_().clamp_(-127, 127))

    s = {"op": op}
    if op == "rmsnorm_i8":
        loud = torch.ones(cols, device="cuda")
        loud[torch.randint(0, cols, (max(1, cols // 512),), generator=g, device="cuda")] = 20.0   # the loud channels of a residual stream
        s["resid"] = (normal(rows, cols) * loud).to(_TYPES[case["resid"]])
        s["delta"] = None if case["delta"] == "none" else normal(rows, cols).to(_TYPES[case["delta"]])
        s["gain"] = (1 + 0.2 * normal(cols)).bfloat16()
        s["resid_out"] = torch.empty_like(s["resid"])
    elif op == "linear_i8":
        s["x"], s["x_scale"] = whole(rows, cols), scales(rows)
        s["w"], s["w_scale"] = whole(case["outs"], cols), scales(case["outs"])
        s["out"] = torch.empty(rows, case["outs"], dtype=_TYPES[case["out"]], device="cuda")
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        if own:     # weights are laid out once, when a model is loaded
            from paper_2605_11186_b200 import binding
            s["packed"] = binding.pack_weights_i8(s["w"])
    else:
        s["x"] = normal(rows, cols * 2 if op == "swiglu_i8" else cols).to(_TYPES[case["x"]])
    if op != "linear_i8":
        s["q"] = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.int8, device="cuda")[:, :cols]
        s["scale"] = torch.empty(rows, dtype=torch.float32, device="cuda")
        s["values"] = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    return s


def _held(y):
    """The values that a row's 8-bit form stands for, and its scale."""
    a = y.abs().amax(1).clamp_min(_TINY)
    q = torch.round(y * (127.0 / a)[:, None])
    scale = a / 127.0
    return (q * scale[:, None]).bfloat16(), scale


def run(state):
    op = state["op"]
    if own:
        from paper_2605_11186_b200 import binding
        if op == "linear_i8":
            binding.cats_linear_i8(state["x"], state["x_scale"], state["packed"], state["w_scale"], state["out"], state["status"])
            return {"out": state["out"]}
        if op == "rmsnorm_i8":
            binding.cats_rmsnorm_i8(state["resid"], state["delta"], state["gain"], _EPS, state["resid_out"], state["q"], state["scale"])
        elif op == "swiglu_i8":
            binding.cats_swiglu_i8(state["x"], state["q"], state["scale"])
        else:
            binding.cats_quantize_i8(state["x"], state["q"], state["scale"])
        binding.cats_dequantize_i8(state["q"], state["scale"], state["values"])
        out = {"values": state["values"], "scale": state["scale"]}
        if op == "rmsnorm_i8":
            out["resid"] = state["resid_out"]
        return out
    if op == "linear_i8":
        sums = state["x"].double() @ state["w"].double().t()        # whole numbers past 2^24
        out = sums * state["x_scale"].double()[:, None] * state["w_scale"].double()
        return {"out": out.to(state["out"].dtype)}
    if op == "rmsnorm_i8":
        r = state["resid"].float()
        if state["delta"] is not None:
            r = r + state["delta"].float()
        y = r * torch.rsqrt((r * r).mean(1, keepdim=True) + _EPS) * state["gain"].float()
        values, scale = _held(y)
        return {"values": values, "scale": scale, "resid": r.to(state["resid"].dtype)}
    x = state["x"].float()
    if op == "swiglu_i8":
        gate, up = x.chunk(2, 1)
        x = gate / (1 + torch.exp(-gate)) * up
    values, scale = _held(x)
    return {"values": values, "scale": scale}


def work(case):
    rows, cols, op = case["rows"], case["cols"], case["op"]
    size = {"f32": 4, "bf16": 2, "none": 0}
    n = rows * cols
    if op == "linear_i8":
        outs = case["outs"]
        return {"bytes": n + outs * cols + 4 * (rows + outs) + rows * outs * size[case["out"]], "flops": 2 * n * outs}
    held = n + 4 * rows
    if op == "rmsnorm_i8":
        return {"bytes": n * (2 * size[case["resid"]] + size[case["delta"]]) + 2 * cols + held, "flops": 7 * n}
    if op == "swiglu_i8":
        return {"bytes": 2 * n * size[case["x"]] + held, "flops": 8 * n}
    return {"bytes": n * size[case["x"]] + held, "flops": 3 * n}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "linear_i8":
        x = s["x"].to(torch.float64).mul_(s["x_scale"].to(torch.float64).unsqueeze(1))
        w = s["w"].to(torch.float64).mul_(s["w_scale"].to(torch.float64).unsqueeze(1))
        return {"out": torch.einsum("tk,nk->tn", x, w)}
    found = {}
    if op == "rmsnorm_i8":
        y = s["resid"].to(torch.float64)
        if s["delta"] is not None:
            y = y.add(s["delta"].to(torch.float64))
        found["resid"] = y
        length = y.square().sum(dim=1, keepdim=True).div(case["cols"]).add(_EPS).sqrt()
        y = s["gain"].to(torch.float64) * y / length
    elif op == "swiglu_i8":
        y = s["x"].to(torch.float64)
        y = y[:, :case["cols"]].sigmoid().mul(y[:, :case["cols"]]).mul(y[:, case["cols"]:])
    else:
        y = s["x"].to(torch.float64)
    step = torch.maximum(y.max(dim=1).values, -y.min(dim=1).values).clamp(min=_TINY).div(127)
    found["scale"] = step
    found["values"] = y.div(step.unsqueeze(1)).round().mul(step.unsqueeze(1))
    return found
