"""Layer norm's stored mean is the row's mean rounded once."""
import pytest
import torch

from paper_2512_16928_amd import binding

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("t,c", [(3, 5), (7, 264), (1200, 264), (1500, 2048), (40, 4096), (33, 8448), (9, 11008), (5, 16390)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_mean_is_rounded_once(hip_device, dtype, t, c):
    """Rows whose mean is small beside their entries, which have a hundredth of channels twenty times the others: the sum in 64
    bits is off by c 2^-53 of the sum of magnitudes, and the mean stored by half a step of fp32 more."""
    g = torch.Generator(device="cuda")
    g.manual_seed(t * 100003 + c)
    loud = 1.0 + 19.0 * (torch.rand(c, generator=g, device="cuda") < 0.01)
    x = (torch.randn((t, c), generator=g, device="cuda") * loud + 0.5 * torch.randn((1, c), generator=g, device="cuda"))
    x = (x * torch.exp(0.5 * torch.randn((t, 1), generator=g, device="cuda"))).to(dtype)
    y, mean, rstd = torch.empty_like(x), torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
    binding.dion2_layernorm_forward(y, x, mean=mean, rstd=rstd)
    want = x.double().mean(1)
    off = 2 * c * 2.0 ** -53 * x.double().abs().mean(1)
    err = (mean.double() - want).abs()
    lim = off + 2.0 ** -24 * (want.abs() + off)
    assert bool((err <= lim).all()), float((err / lim).max())


@pytest.mark.parametrize("c", [9, 1000, 2048, 20000])
def test_rows_far_from_zero_keep_their_spread(hip_device, c):
    """fp32 rows of spread 1 around 2^20: entries are multiples of 2^-3 and their mean is not. rstd is that of the entries'
    own spread: x - mean is exact, what the mean leaves (2^-4 at most) is known to 2^-28, d is rounded by 2^-24 of itself, its
    square and the sum of c of them by at most (c + 2) 2^-24."""
    g = torch.Generator(device="cuda")
    g.manual_seed(c)
    x = torch.randn((64, c), generator=g, device="cuda") + 2.0 ** 20
    y, rstd = torch.empty_like(x), torch.empty(64, device="cuda")
    binding.dion2_layernorm_forward(y, x, eps=1e-5, rstd=rstd)
    d = x.double() - x.double().mean(1, keepdim=True)
    want = 1.0 / torch.sqrt(d.square().mean(1) + 1e-5)
    bound = (c + 8) * 2.0 ** -24
    assert bool(((rstd.double() - want).abs() <= bound * want).all())
    assert bool(((y.double() - d * want[:, None]).abs() <= (bound + 2.0 ** -22) * (d * want[:, None]).abs() + 2.0 ** -27).all())
