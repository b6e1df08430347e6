"""What the activations lose in fp32 arithmetic, relative to their value: far out
on the negative side they are small, and an error that is small next to 1 is not
small next to them.

u = 2^-24.  GELU z Phi(z), z exact: -z^2 / 2 is within 2 u z^2 / 2 after two
roundings, its exponential within that, relatively, and the few u of the
exponential's own argument (u z^2 / 2 once more) and result; the argument of the
remaining factor moves it by less.  2 z^2 + 40 units u hold that with room for some ten
roundings of a polynomial, a reciprocal and the products.  Beyond |z|, Phi is 1 less such a tail.
SiLU and the tanh form are z s(v), s(v) = 1 / (1 + exp(-v)): v is within 4 u |v|, so
exp(-v) within 4 u |v| and the same few terms: 8 |v| + 40.
Rounding to bf16 adds 2^-8 of the value."""
import math

import pytest
import torch

import layers_ref as R
from paper_2606_27153_amd import layers

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _forward_and_slope(z, act):
    one = torch.ones(1, 1, dtype=z.dtype, device=DEV)
    y = layers.linear_forward(one, z, activation=act)
    _, slope, _ = layers.linear_backward(torch.ones_like(z), one, z, preactivation=z, activation=act)
    return y.double()[0], slope.double()[0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=lambda v: str(v).replace("torch.", ""))
def test_gelu_is_good_relative_to_its_value(dtype):
    z = torch.cat([torch.linspace(-12, 12, 96001, device=DEV), 10 ** torch.linspace(-6, 0, 999, device=DEV),
                   -10 ** torch.linspace(-6, 0, 1000, device=DEV)])[None].to(dtype)
    y, slope = _forward_and_slope(z, "gelu")
    t = z.double()[0]
    cdf = 0.5 * torch.special.erfc(-t * math.sqrt(0.5))   # (torch.special.ndtr is 0 from -9 on)
    density = torch.exp(-t * t / 2) / math.sqrt(2 * math.pi)
    rel = (2 * t * t + 40) * R.U
    q = R.ROUND[dtype]
    want = t * cdf
    assert ((y - want).abs() <= want.abs() * (rel + q * (1 + rel))).all(), \
        float(((y - want).abs() / want.abs()).max())
    want, err = cdf + t * density, rel * (cdf + t.abs() * density)
    assert ((slope - want).abs() <= err + q * (want.abs() + err)).all(), float((slope - want).abs().max())


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_sigmoid_forms_are_good_relative_to_their_value(act):
    z = torch.linspace(-80, 80, 100001, device=DEV)[None] if act == "silu" else \
        torch.linspace(-9, 9, 100001, device=DEV)[None]
    y, _ = _forward_and_slope(z, act)
    t = z.double()[0]
    v = t if act == "silu" else 2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3)
    want = t * torch.special.expit(v)
    assert ((y - want).abs() <= want.abs() * (8 * v.abs() + 40) * R.U).all(), \
        float(((y - want).abs() / want.abs()).max())
