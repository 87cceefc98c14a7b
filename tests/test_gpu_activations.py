"""The group norm's activations by themselves: with a weight of zero, z is the bias, y = act(z), and the bias' gradient for grad_y = 1
over one position is act'(z).  u = 2^-24.

Tolerances.  GELU: Phi(z) is 1 or 0 plus or minus a tail of at most 1/2 whose formula is off by 7.5e-8 (half of erf's 1.5e-7), and which
passes some eight roundings (4 u): 7.5e-8 + 5 u with the last subtraction, times |z|, and u for the product; the slope adds z times
the density (0.25 at most, ten roundings: 3 u).  Far below zero the formula keeps a relative 2^-6.  SiLU: the exponent -z log2 e is
rounded twice (2 |z| u of the exponential) and six operations follow; its slope p (1 + z (1 - p)) sums terms of |z| p."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def values():
    """z, and what the library gives for it: {activation: (value, slope)}."""
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2510_03426_amd import Goom
    g = Goom(0)
    z = torch.cat([torch.linspace(-8, 8, 4091), torch.tensor([-3.0, -5.0, -7.0, 0.0, 1e-4])]).cuda()
    x = torch.randn(1, z.numel(), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    out = {}
    for act in ("silu", "gelu"):
        y, mean, rstd = g.group_norm(x, 8, torch.zeros_like(z), z, activation=act, want_stats=True)
        slope = g.group_norm_backward(x, torch.ones_like(x), mean, rstd, 8, torch.zeros_like(z), z, activation=act)[2]
        out[act] = y[0].double().cpu().numpy(), slope.double().cpu().numpy()
    z = z.double().cpu().numpy()
    g.close()
    return z, out


def test_gelu(values):
    z, out = values
    y, slope = out["gelu"]
    cdf = np.array([0.5 * math.erfc(-t / math.sqrt(2)) for t in z])
    density = np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    assert (np.abs(y - z * cdf) <= np.abs(z) * (7.5e-8 + 5 * U) + U * np.abs(z * cdf)).all()
    assert (np.abs(slope - cdf - z * density) <= 7.5e-8 + 9 * U).all()
    far = z <= -3
    assert (np.abs(y - z * cdf)[far] <= 2.0 ** -6 * np.abs(z * cdf)[far]).all()


def test_silu(values):
    z, out = values
    y, slope = out["silu"]
    p = 1 / (1 + np.exp(-z))
    assert (np.abs(y - z * p) <= (2 * np.abs(z) + 8) * U * np.abs(z * p)).all()
    assert (np.abs(slope - p * (1 + z * (1 - p))) <= (2 * np.abs(z) + 12) * U * p * (1 + np.abs(z) * (1 - p))).all()
