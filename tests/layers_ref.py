"""Reference of the layer operators in 64 bits, with bounds on how far fp32
arithmetic and one final rounding may be from it.

A sum of n products in fp32, in any order, is within n u S of the exact one,
u = 2^-24, S the sum of the products' absolute values (bf16 factors multiply
exactly).  A few more roundings (bias, residual, scale) are covered by n + 8.
Rounding to p significant bits adds 2^-p of the value (bf16 has 8, fp32 24).  An activation's own
arithmetic (an exponential or erf, a quotient, a few products) is taken as good
to 2^-20 (1 + |z|), and passes an error of z on with a slope below 1.2.
"""
import math

import torch

U = 2.0 ** -24
ACT_TOL = 2.0 ** -20
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_C = math.sqrt(2 / math.pi)


def act(z, name):
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(_C * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def act_grad(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        t = torch.tanh(_C * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * _C * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def f64(t):
    return None if t is None else t.detach().cpu().double()


def linear_forward(x, w, b, r, name, out_dtype):
    """(z, bound of z, y, bound of y), the bounds including the outputs' rounding."""
    x, w, b, r = f64(x), f64(w), f64(b), f64(r)
    z, s = x @ w, x.abs() @ w.abs()
    if b is not None:
        z, s = z + b, s + b.abs()
    ez = (x.shape[1] + 8) * U * s
    y = act(z, name)
    ey = ez if name == "none" else 1.2 * ez + ACT_TOL * (1 + z.abs())
    if r is not None:
        y = y + r
        ey = ey + 2 * U * (y.abs() + r.abs())
    q = ROUND[out_dtype]
    return z, ez + q * (z.abs() + ez), y, ey + q * (y.abs() + ey)


def linear_backward(dy, x, w, z, name, dtype):
    """{"dx", "dw", "db"}: (value, bound)."""
    dy, x, w, z = f64(dy), f64(x), f64(w), f64(z)
    q = ROUND[dtype]
    if name == "none":
        dz, e = dy, torch.zeros_like(dy)
        ezr = e
    else:
        dz = dy * act_grad(z, name)
        e = dy.abs() * ACT_TOL * (1 + z.abs())
        ezr = e + q * dz.abs()   # dz as the products read it, rounded to dtype
    n, m = w.shape[1], x.shape[0]

    def close(v, s, err, terms):
        err = err + (terms + 8) * U * s
        return v, err + q * (v.abs() + err) + 1e-300

    return {"dx": close(dz @ w.t(), (dz.abs() + ezr) @ w.abs().t(), ezr @ w.abs().t(), n),
            "dw": close(x.t() @ dz, x.abs().t() @ (dz.abs() + ezr), x.abs().t() @ ezr, m),
            "db": close(dz.sum(0), dz.abs().sum(0), e.sum(0), m)}


def check(got, want, bound, what=""):
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs() - bound
    bad = ~(off <= 0)   # (NaN counts)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} outside the bound, worst "
                           f"{float((got - want).abs()[bad].max())} at {torch.nonzero(bad)[0].tolist()}")


def norm(x, w, b, eps, mean=None, rstd=None):
    """(y, mean, rstd, h) in 64 bits."""
    x, w, b = f64(x), f64(w), f64(b)
    if mean is None:
        mean = x.mean(1)
        rstd = 1 / torch.sqrt((x - mean[:, None]).pow(2).mean(1) + eps)
    h = (x - mean[:, None]) * rstd[:, None]
    y = h if w is None else h * w
    return (y if b is None else y + b), mean, rstd, h
