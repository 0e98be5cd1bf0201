"""Activations and their slopes far below zero, where they are small: relative errors, in half steps e = 2^-24 of fp32.

z is the bias alone (x = 0), y fp32, and dbias of one row with dy = 1 the slope, so that nothing but the activation is rounded.
- gelu_tanh: z sigmoid(a), a = 2 sqrt(2 / pi) (z + 0.044715 z^3), is off by 5 e |a| of the exponent (a's four roundings and the
  factor's), 2 e for exp2, e for the sum, 2 e for the reciprocal and e for the product: (5 |a| + 7) e.  Its slope is s + z s (1 - s) a':
  s as above, the other term by three such factors, (15 |a| + 24) e, and e.
- gelu: z times half the weight of the tail, p(t) e^(-z^2/2): 1.5 z^2 e of the exponent's three factors and 2 e for exp2, 4 e in
  t, which count at most twice, 16 e for the eight terms, 1.4 e for the fit, 3 e of products: (1.5 z^2 + 32) e; above zero that of
  the tail, in 1 - tail, and 2 e.  Its slope adds z e^(-z^2/2) / sqrt(2 pi), off by (1.5 z^2 + 8) e, and e.
- silu: z sigmoid(z) likewise with 3 e |z| of the exponent: (3 |z| + 7) e.
"""
import math

import pytest
import torch

import paper_2606_05597_amd as grpo
from tests.test_gpu_linear import BF16, E, F32, act64

pytestmark = pytest.mark.gpu


def values(act, z):
    """y and the slope of act at z, as the kernel forms them."""
    N = z.numel()
    x, w = torch.zeros((1, 8), dtype=BF16, device="cuda"), torch.zeros((8, N), dtype=BF16, device="cuda")
    y, kept = grpo.grpo_linear(x, w, z, act=act, out_dtype=F32, keep_z=True)
    assert torch.equal(kept[0], z)
    slope = torch.empty_like(z)
    grpo.grpo_linear_bwd(torch.ones((1, N), device="cuda"), x, w, kept, act=act, dx=False, dw=False, dbias=slope)
    return y[0].double(), slope.double()


def near(got, want, bound, z):
    off = (got - want).abs()
    i = int((off - bound).argmax())
    assert (off <= bound).all(), (float(z[i]), float(got[i]), float(want[i]), float(bound[i]))


def test_gelu_tanh():
    z = torch.linspace(-9.4, 9.4, 6001, device="cuda")
    y, slope = values("gelu_tanh", z)
    zd = z.double()
    k = 2 * math.sqrt(2 / math.pi)
    a, da = k * (zd + 0.044715 * zd**3), k * (1 + 3 * 0.044715 * zd**2)
    s = torch.sigmoid(a)
    near(y, zd * s, 1.01 * (5 * a.abs() + 7) * E * (zd * s).abs(), z)
    rest = zd * s * torch.sigmoid(-a) * da
    near(slope, s + rest, 1.01 * E * ((5 * a.abs() + 7) * s + (15 * a.abs() + 24) * rest.abs() + (s + rest).abs()), z)


def test_gelu():
    z = torch.linspace(-12, 12, 6001, device="cuda")
    y, slope = values("gelu", z)
    zd = z.double()
    tail = 0.5 * torch.special.erfc(zd.abs() * math.sqrt(0.5))
    cdf = torch.where(zd < 0, tail, 1 - tail)
    off = (1.5 * zd**2 + 32) * E * tail + torch.where(zd < 0, 0.0, 2 * E)
    near(y, zd * cdf, 1.01 * (zd.abs() * off + E * (zd * cdf).abs()), z)
    rest = zd * torch.exp(-0.5 * zd**2) / math.sqrt(2 * math.pi)
    near(slope, cdf + rest, 1.01 * (off + (1.5 * zd**2 + 8) * E * rest.abs() + E * (cdf + rest).abs()), z)


def test_silu():
    z = torch.linspace(-80, 20, 6001, device="cuda")
    y, _ = values("silu", z)
    want = act64("silu", z.double())
    near(y, want, 1.01 * (3 * z.double().abs() + 7) * E * want.abs(), z)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_far_out(act):
    """Beyond the tails y is z or 0 and the slope 1 or 0."""
    z = torch.tensor([-3e38, -1e30, -1e8, -200.0, 200.0, 1e8, 1e30, 3e38], device="cuda")
    y, slope = values(act, z)
    assert torch.equal(y[4:], z[4:].double()) and (y[:4].abs() <= 1e-30).all()
    assert (slope[4:] == 1).all() and (slope[:4].abs() <= 1e-30).all()
