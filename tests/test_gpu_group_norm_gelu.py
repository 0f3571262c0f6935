"""The GELU of the group norm by itself, against the error function in 64 bits.

With gamma = 0 the activation's argument is beta, whatever x holds, so a channel gives one value, and with a single position and d_y = 1
its d_beta is the slope there.  (Grouped over all channels: more than 1024 channels go through the passes over memory, fewer are held
by a workgroup.)

Tolerances.  Relative, of the integral of the normal distribution up to z (where it is small it is a product of an exponential, a
reciprocal and a polynomial): 1.1e-7 the polynomial's, 1.2e-7 for each of the hardware's exponential and reciprocal, some ten roundings of
6e-8 that add up to no more than 4e-7: 1e-6 in all; the exponential's argument z^2 / 2 is rounded twice, 6e-8 of it each, which
makes 6e-8 z^2 of the value; twice that is allowed.  Root mean square over a normal distribution: 1.5 times that of the formula by
fp32 torch, which rounds as often."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _gelu(lp, z, shape=(1, 1)):
    c = z.numel()
    gen = torch.Generator().manual_seed(c)
    x = torch.randn(*shape, c, generator=gen).cuda()
    norm = lp.GroupNorm(1, torch.zeros(c, device="cuda"), z.cuda(), lp.LP_ACT_GELU)
    y, stats = lp.group_norm_fwd(norm, x)
    _, _, slope = lp.group_norm_bwd(norm, x, stats, torch.ones_like(x))
    return y.view(-1, c).double().cpu(), slope.double().cpu()


def _exact(z):
    z = z.double()
    integral = 0.5 * torch.erfc(-z / math.sqrt(2))
    return integral, z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("count", [1024, 65536])
def test_relative_error(lp, count):
    """Down to -10, where the integral is 8e-24."""
    z = torch.linspace(-10, 10, count)
    z[0], z[1], z[2], z[3], z[4], z[5] = 0.0, 1.0, -1.0, math.nextafter(1.0, 0.0), 1e-20, -1e-6
    y, _ = _gelu(lp, z)
    want = _exact(z)[0] * z.double()
    assert float(((y[0] - want).abs() - (1e-6 + 1.2e-7 * z.double() ** 2) * want.abs()).max()) <= 0


@pytest.mark.parametrize("count", [1024, 65536])
def test_mean_error_is_that_of_the_formula_in_fp32(lp, count):
    z = torch.randn(count, generator=torch.Generator().manual_seed(3))
    y, slope = _gelu(lp, z)
    integral, more = _exact(z)
    half = 0.5 * (1 + torch.erf(z / math.sqrt(2.0)))
    plain = (z * half).double(), (half + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)).double()
    for got, by_torch, want in ((y[0], plain[0], z.double() * integral), (slope, plain[1], integral + more)):
        assert float((got - want).square().mean().sqrt()) <= 1.5 * float((by_torch - want).square().mean().sqrt())
    assert float((slope - integral - more).abs().max()) <= 4e-7   # (1e-6 of terms that are at most 0.25, and a rounding near 1)


def test_ends(lp):
    z = torch.tensor([1e4, -1e4, 3e38, -3e38, float("inf"), 20.0, -20.0, float("nan")])
    y, slope = _gelu(lp, z)
    assert y[0, 0] == 1e4 and y[0, 2] == float(z[2]) and y[0, 4] == float("inf") and y[0, 5] == 20.0
    assert y[0, 1] == 0 and y[0, 3] == 0 and abs(float(y[0, 6])) < 1e-80 and math.isnan(float(y[0, 7]))
    assert slope[0] == 1 and slope[1] == 0 and slope[2] == 1 and slope[3] == 0 and math.isnan(float(slope[7]))
