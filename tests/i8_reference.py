"""Plain 64-bit forms of the 8-bit operators, and how far a correct kernel may be from them.

Rounding steps: u = 2^-24 (half a step of fp32, relative), 2^-8 of bf16."""
import torch

U = 2.0 ** -24
TINY = 2.0 ** -100


def held(y):
    """(a, 127 y / a) of fp64 rows: what q is the rounding of."""
    a = y.abs().amax(1).clamp_min(TINY)
    return a, 127.0 * y / a[:, None]


def rmsnorm(resid, delta, gain, eps):
    r = resid.double() if delta is None else resid.double() + delta.double()
    return r, r / torch.sqrt((r * r).mean(1, keepdim=True) + eps) * gain.double()


def swiglu(gate_up):
    g, u = gate_up.double().chunk(2, 1)
    return g * torch.sigmoid(g) * u


def norm_error(cols):
    """Relative error of y: the sum of squares has at most cols / 512 + 16 roundings on any term's way (a thread's own terms,
    then nine or ten levels of pairwise sums), halved by the root; rsqrt 2 ulp (4 u); residual sum, two products, the mean's
    division, + eps: 6 u."""
    return (0.5 * (cols / 512 + 16 + 2) + 4 + 6) * U


def swiglu_error(gate_up):
    """__expf is off by 2 + 1.173 |g| ulp (an ulp is 2 u), the quotient by 2 ulp, the sum and the product by u each."""
    g = gate_up.double().chunk(2, 1)[0].abs().amax().item()
    return (2 * (2 + 1.173 * g) + 4 + 2) * U


def check_held(q, scale, y, rel):
    """q and scale against fp64 rows y; rel: relative error of the kernel's own fp32 y.  127 y / a as the kernel takes it is
    off by y's error, a's, and two roundings; the nearest whole number is at most 1/2 away from that."""
    a, want = held(y)
    assert ((scale.double() - a / 127).abs() <= (rel + 2 * U) * a / 127).all()
    off = (q.double() - want).abs().max().item()
    assert off <= 0.5 + 127 * (2 * rel + 4 * U), off
    assert q.abs().max().item() <= 127


def linear(x, sx, w, sw):
    return (x.double() @ w.double().t()) * sx.double()[:, None] * sw.double()


def check_linear(out, want):
    """The sums are exact; conversion and two products round once each (3 u), and bf16 once more."""
    rel = 3.01 * U if out.dtype == torch.float32 else 2.0 ** -8 * (1 + 2.0 ** -12)
    bad = ((out.double() - want).abs() > rel * want.abs())
    assert not bad.any(), (int(bad.sum()), (out.double() - want).abs().max().item())
