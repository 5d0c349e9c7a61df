"""GELU as closely as the header states it: Phi(-|z|) within 1.5e-6 relative for |z| <= 4, 5e-6 to 9 and 1e-5 to 12, in
calls of either type, against the complementary error function in 64 bits.

Products with the identity leave z as it is, so act(z) is seen alone. An fp32 output adds the roundings of z Phi and of
the store, 2^-24 each. A bf16 output would hide all of it behind 2^-8, so the residual there is minus the bf16 value next to
the exact one: the sum that is stored is small, exact before its rounding (both have the same exponent or neighbouring
ones), and rounded by 2^-8 of its own size only."""
import math

import pytest
import torch

from paper_2512_16928_amd import binding
from paper_2512_16928_amd.binding import ACT_GELU

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def lower_tail(z):
    """Phi(-|z|) in 64 bits, on the CPU."""
    return torch.tensor([0.5 * math.erfc(abs(v) / math.sqrt(2.0)) for v in z.double().reshape(-1).tolist()],
                        dtype=torch.float64).reshape(z.shape)


def phi_bound(z):
    a = z.double().abs()
    return torch.where(a <= 4, 1.5e-6, torch.where(a <= 9, 5e-6, 1e-5))


def values(rows, dtype):
    """[rows, 64] of -12 to 12, denser about 0, each a value of the type."""
    u = torch.linspace(-1.0, 1.0, rows * 64, dtype=torch.float64)
    return (12.0 * u * u.abs()).to(dtype).view(rows, 64)


@pytest.mark.parametrize("dtype,rows", [(F32, 8), (F32, 640), (F32, 5000), (BF, 32), (BF, 640), (BF, 5000)])
def test_gelu_is_as_exact_as_stated(hip_device, dtype, rows):
    z = values(rows, dtype)
    tail = lower_tail(z)
    phi = torch.where(z > 0, 1.0 - tail, tail)
    want = z.double() * phi
    off = z.double().abs() * (tail * phi_bound(z) + 2.0 ** -24 * phi) + 2.0 ** -24 * want.abs()
    R = None
    if dtype is BF:
        R = (-want).to(BF)
        want = want + R.double()
    Y = torch.empty((rows, 64), dtype=dtype, device="cuda")
    binding.dion2_linear_forward(Y, z.cuda(), torch.eye(64, device="cuda").to(dtype), act=ACT_GELU,
                                 residual=None if R is None else R.cuda())
    lim = off + (2.0 ** -8 if dtype is BF else 2.0 ** -24) * (want.abs() + off) + 1e-37
    err = (Y.cpu().double() - want).abs()
    worst = int((err / lim).argmax())
    assert bool((err <= lim).all()), (float(z.view(-1)[worst]), float(err.view(-1)[worst]), float(lim.view(-1)[worst]))


@pytest.mark.parametrize("rows", [8, 640])
def test_gelu_slope_is_as_exact(hip_device, rows):
    """Phi(z) + z phi(z) in fp32: for -|z| both terms share the exponential whose error Phi's bound is made of; the
    subtraction, the step to positive z and the product with dY round by 2^-24 each."""
    z = values(rows, F32)
    d, tail = z.double(), lower_tail(z)
    density = d.abs() * torch.exp(-0.5 * d * d) / math.sqrt(2.0 * math.pi)
    low = tail - density
    want = torch.where(z > 0, 1.0 - low, low)
    dZ = torch.empty((rows, 64), device="cuda")
    binding.dion2_activation_backward(dZ, torch.ones((rows, 64), device="cuda"), z.cuda(), ACT_GELU)
    lim = (tail + density) * (phi_bound(z) + 2.0 ** -23) + 2.0 ** -23 * want.abs() + 1e-37
    err = (dZ.cpu().double() - want).abs()
    worst = int((err / lim).argmax())
    assert bool((err <= lim).all()), (float(z.view(-1)[worst]), float(err.view(-1)[worst]), float(lim.view(-1)[worst]))
