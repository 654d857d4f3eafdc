"""Activation functions of fp32 tensors, and their gradients, to fp32's accuracy; ends
of the range in both types.

Tolerances, with u = 2^-24 (half a step of fp32, relative), a = |z|, Q(a) the upper
tail of the normal distribution and phi its density.  The device library's erfcf is off
by up to 2 units in the last place (4 u), expf by 1 (2 u).
GELU: a / sqrt 2 is off by 2 u (constant, product), which erfc multiplies by up to
a^2 + 1, so that Q is off by (6 + 2 a^2) u; the last sum rounds once, and its other term
is at most as large as twice the result: (8 + 2 a^2) u of the value.
GELU': Q as above, 1 - Q one rounding, the exponent a^2 / 2 one rounding, its exponential
2 u, constant and products 3 u: (7 + 2 a^2) Q + (6 + a^2 / 2) a phi + 1 for z > 0, and
two roundings of the result (the sum, and the product with da), in u.
SiLU: 2 u, a sum and a quotient: 5 u.  SiLU': s = 1 / (1 + e^-z) is off by 4 u, 1 - s
by 7 u, its product with z by 8 u; the sum, and the product with s, round once more: 9 s
a (1 - s) + 7 times the result, in u.  e^-z passes fp32 below z = -88.7, where SiLU is
below 3e-37: + 1e-36."""

import math

import pytest
import torch

from paper_2606_19163_amd import ops

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def _values(dtype):
    """Both tails, the bend, and the zero of GELU'."""
    z = torch.cat([torch.linspace(-14, 14, 4096), torch.linspace(-100, 100, 2048),
                   torch.linspace(-1, 1, 2048), 10.0 ** torch.linspace(-30, 30, 1024),
                   -(10.0 ** torch.linspace(-30, 30, 1024))])
    return z.to(dtype).view(-1, 64)


def _tail(z):
    a = z.abs()
    return a, 0.5 * torch.erfc(a / math.sqrt(2.0)), torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)


def _gelu(z):
    a, q, phi = _tail(z)
    return torch.where(z > 0, z - a * q, -a * q), torch.where(z > 0, 1 - q, q) + z * phi


def _silu(z):
    s = torch.sigmoid(z)
    return z * s, s * (1 + z * torch.sigmoid(-z))


def _run(act, x, dtype):
    plan = ops.Checkpoint(64, act=act, dtype=dtype)
    a, kept = plan.forward(x.cuda())
    z = plan.load(kept).cpu().double()
    da = 1 + torch.rand(x.shape, generator=torch.Generator().manual_seed(1))
    da = da.to(dtype)
    return a.cpu().double(), z, da.double(), plan.backward(da.cuda(), kept).cpu().double()


def _check(off, bound):
    assert bool((off <= bound).all()), float((off / bound).max())


def test_gelu_fp32():
    x = _values(F32)
    got, z, da, dx = _run("gelu", x, F32)
    ref, _ = _gelu(x.double())
    _check((got - ref).abs(), (8 + 2 * x.double() ** 2).clamp(max=1e9) * U * ref.abs() + 1e-37)
    _, d = _gelu(z)
    a, q, phi = _tail(z)
    a2 = (a * a).clamp(max=1e9)
    _check((dx - da * d).abs(), 1.01 * U * da * ((7 + 2 * a2) * q + (z > 0) +
                                                 (6 + a2 / 2) * a * phi + 2 * d.abs()) + 1e-37)


def test_silu_fp32():
    x = _values(F32)
    got, z, da, dx = _run("silu", x, F32)
    ref, _ = _silu(x.double())
    _check((got - ref).abs(), 5 * U * ref.abs() + 1e-36)
    _, d = _silu(z)
    s = torch.sigmoid(z)
    _check((dx - da * d).abs(),
           1.01 * U * da * (9 * s * z.abs() * torch.sigmoid(-z) + 7 * d.abs()) + 1e-36)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_ends(dtype):
    x = torch.zeros(4, 64, dtype=dtype)
    x[0, 0], x[1, 0], x[2, 0], x[3, 0] = float("nan"), float("inf"), -float("inf"), -300.0
    a = ops.Checkpoint(64, act="gelu", dtype=dtype).forward(x.cuda())[0].cpu()
    assert bool(torch.isnan(a[0, 0])) and float(a[1, 0]) == float("inf")
    assert float(a[2, 0]) == 0 and float(a[3, 0]) == 0 and not bool(torch.isnan(a[1:]).any())
    a = ops.Checkpoint(64, act="silu", dtype=dtype).forward(x.cuda())[0].cpu()
    assert bool(torch.isnan(a[0, 0])) and float(a[1, 0]) == float("inf") and float(a[3, 0]) == 0
    for act in ("gelu", "silu"):
        plan = ops.Checkpoint(64, act=act, dtype=dtype)
        big = torch.full((1, 64), torch.finfo(dtype).max, dtype=dtype)
        for v, want in ((big, 1.0), (-big, 0.0)):
            dx = plan.backward(torch.ones_like(v).cuda(), plan.save(v.cuda()))
            assert bool((dx == want).all())
