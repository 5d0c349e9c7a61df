"""The layer passes (a linear layer's three products, an activation's gradient, layer norm forward and backward) against
plain 64-bit forms of their formulas, at the sizes, types, strides and values where they can go wrong.

Tolerances, entry by entry. An output is rounded once: at most half a step, 2^-8 (bf16) or 2^-24 (fp32) of its value.
A sum of n fp32 terms in any order is off by at most about n 2^-24 of the sum of their magnitudes; products of bf16 values
are exact in fp32, products of fp32 values and the matrix cores' own additions are allowed 2^-23 each instead:
(n + 16) 2^-23 sum |a b|. Activations: Phi within 1e-5 (bf16) or 4e-6 (fp32) relative, so act and act' within 3e-5 and
1e-5 of max(1, |z|), and slopes of at most 1.13 carry a pre-activation's error on."""
import math
import zlib

import pytest
import torch

from paper_2512_16928_amd import binding
from paper_2512_16928_amd.binding import ACTIVATIONS, DION2_ERR_WORKSPACE, Dion2Error

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}
ACT_ERR = {BF: 3e-5, F32: 1e-5}
EPS = 1e-5


def rnd(shape, dtype, gen, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def gen_of(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return g


class Framed:
    """A [rows, width] view inside a larger buffer of a marker value: `lead` elements before it, `pad` more per row.
    intact() says that nothing around the view was written."""

    def __init__(self, rows, width, dtype, lead=0, pad=0, fill=None):
        self.mark = 77.0
        self.buf = torch.full((lead + (rows + 1) * (width + pad) + 8,), self.mark, dtype=dtype, device="cuda")
        self.view = self.buf[lead:lead + rows * (width + pad)].view(rows, width + pad)[:, :width]
        if fill is not None:
            self.view.copy_(fill)
        self.used = torch.zeros_like(self.buf, dtype=torch.bool)
        self.used[lead:lead + rows * (width + pad)].view(rows, width + pad)[:, :width] = True

    def intact(self):
        return bool((self.buf[~self.used] == self.mark).all())


def near(got, want, bound, dtype, what):
    """|got - want| <= bound + the final rounding, entry by entry; the same entries finite."""
    got, ok = got.double(), torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), ok), f"{what}: finite entries differ"
    err = (got - want).abs()
    lim = bound * (1 + HALF[dtype]) + HALF[dtype] * want.abs() + 1e-37
    bad = ok & ~(err <= lim)
    if bad.any():
        i = int(torch.nonzero(bad.reshape(-1))[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off; entry {i}: {got.reshape(-1)[i]} for "
                             f"{want.reshape(-1)[i]}, limit {lim.reshape(-1)[i]}")


def act64(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(z, act):
    z = z.detach().clone().requires_grad_(True)
    return torch.autograd.grad(act64(z, act).sum(), z)[0] if act != "none" else torch.ones_like(z)


def product64(a, b):
    """a b^T in 64 bits, and the bound on what fp32 sums of it are off."""
    a, b = a.double(), b.double().t().contiguous()
    return a @ b, (a.shape[1] + 16) * 2.0 ** -23 * (a.abs() @ b.abs())


# (tokens, rows, cols): one entry, single tokens, below and above a vector, tile edges, odd and large, an
# output of 144 partly filled 256 x 256 tiles in each of the three products, and as many tokens as fill one or two of 16;
# then tiles of 128, and products whose K is cut into parts on tiles of 64, 128 and 256
SIZES = [(1, 1, 1), (1, 96, 64), (1, 257, 1000), (2, 33, 7), (3, 8, 130), (5, 1000, 264), (16, 300, 520), (17, 64, 64),
         (31, 7, 33), (64, 128, 128), (127, 129, 130), (128, 256, 512), (129, 100, 8), (300, 264, 257), (515, 130, 72),
         (1024, 520, 2048), (700, 1000, 517), (2900, 2824, 200), (2900, 72, 2824), (72, 2904, 2824),
         (16, 1000, 4104), (32, 520, 2048), (33, 264, 264),
         (2200, 2056, 136), (2200, 136, 2056), (136, 2200, 2056), (72, 520, 8200), (72, 8200, 520), (8200, 72, 520),
         (2048, 2048, 8192), (3000, 2048, 8192), (8192, 3000, 2048)]
ACTS = sorted(ACTIVATIONS)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_forward(hip_device, i, dtype):
    t, r, c = SIZES[i]
    act = ACTS[i % len(ACTS)]
    g = gen_of("fwd", i, dtype == BF)
    lead, pad = [(0, 0), (0, 8), (1, 3), (8, 64)][i % 4]
    X = Framed(t, c, dtype, lead, pad, rnd((t, c), dtype, g)).view
    W = rnd((r, c), dtype, g, 1.5 / math.sqrt(c))
    bias = rnd((r,), [dtype, F32, BF][i % 3], g, 0.5) if i % 3 != 1 or i == 1 else None
    R = Framed(t, r, dtype, lead, pad + 1, rnd((t, r), dtype, g)) if i % 2 else None
    Y, Z = Framed(t, r, dtype, lead, pad), Framed(t, r, dtype, 2 * lead, pad + 2)
    binding.dion2_linear_forward(Y.view, X, W, bias=bias, residual=R.view if R else None, Z=Z.view if i % 5 != 4 else None,
                                 act=ACTIVATIONS[act])
    z, zerr = product64(X, W)
    if bias is not None:
        z = z + bias.double()
        zerr = zerr + 2.0 ** -23 * z.abs()
    y = act64(z, act)
    yerr = 1.13 * zerr + (ACT_ERR[dtype] * z.abs().clamp(min=1.0) if act not in ("none", "relu") else 0.0)
    if R:
        y = y + R.view.double()
        yerr = yerr + 2.0 ** -23 * (y.abs() + R.view.double().abs())
    near(Y.view, y, yerr, dtype, "Y")
    assert Y.intact() and Z.intact()
    if i % 5 != 4:
        near(Z.view, z, zerr, dtype, "Z")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_backward_input(hip_device, i, dtype):
    t, r, c = SIZES[i]
    act = ACTS[(i + 1) % len(ACTS)]
    g = gen_of("input", i, dtype == BF)
    lead, pad = [(0, 0), (1, 3), (8, 64), (0, 8)][i % 4]
    dY = Framed(t, r, dtype, lead, pad, rnd((t, r), dtype, g, 1e-2)).view
    W = rnd((r, c), dtype, g, 0.1)
    Z = Framed(t, c, dtype, lead, pad, rnd((t, c), dtype, g, 2.0)).view if act != "none" else None
    dX = Framed(t, c, dtype, lead, pad)
    binding.dion2_linear_backward_input(dX.view, dY, W, Z=Z, act=ACTIVATIONS[act])
    p, err = product64(dY, W.t())
    if act != "none":
        s = slope64(Z.double(), act)
        err = err * s.abs() + p.abs() * (ACT_ERR[dtype] * Z.double().abs().clamp(min=1.0) if act != "relu" else 0.0) \
            + 2.0 ** -23 * (p * s).abs()
        p = p * s
    near(dX.view, p, err, dtype, "dX")
    assert dX.intact()


@pytest.mark.parametrize("g_dtype", [BF, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(SIZES)))
def test_backward_weight(hip_device, i, dtype, g_dtype):
    t, r, c = SIZES[i]
    g = gen_of("weight", i, dtype == BF)
    lead, pad = [(0, 0), (8, 64), (0, 8), (1, 3)][i % 4]
    dY = Framed(t, r, dtype, lead, pad, rnd((t, r), dtype, g, 1e-2)).view
    X = Framed(t, c, dtype, lead, pad, rnd((t, c), dtype, g)).view
    add = i % 2 == 1
    G0, b0 = rnd((r, c), g_dtype, g, 0.1), rnd((r,), g_dtype, g, 0.1)
    G, db = G0.clone(), Framed(1, r, g_dtype, 1, 0, b0[None])
    binding.dion2_linear_backward_weight(G, dY, X, dbias=db.view[0], accumulate=add)
    want, err = product64(dY.t(), X.t())
    sums, mag = dY.double().sum(0), dY.double().abs().sum(0)
    serr = (t + 16) * 2.0 ** -23 * mag
    if add:
        want, sums = want + G0.double(), sums + b0.double()
        err, serr = err + 2.0 ** -23 * want.abs(), serr + 2.0 ** -23 * sums.abs()
    near(G, want, err, g_dtype, "G")
    near(db.view[0], sums, serr, g_dtype, "dbias")
    assert db.intact()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_backward_weight_parts(hip_device, dtype):
    """G alone, dbias alone (X not needed), and no tokens: zeros, or what was there."""
    g = gen_of("parts", dtype == BF)
    dY, X = rnd((70, 40), dtype, g), rnd((70, 48), dtype, g)
    G, db = torch.full((40, 48), 3.0, dtype=F32, device="cuda"), torch.full((40,), 3.0, dtype=F32, device="cuda")
    binding.dion2_linear_backward_weight(G, dY, X)
    near(G, *product64(dY.t(), X.t()), F32, "G alone")
    binding.dion2_linear_backward_weight(None, dY, None, dbias=db)
    near(db, dY.double().sum(0), 86 * 2.0 ** -23 * dY.double().abs().sum(0), F32, "dbias alone")
    for add in (True, False):
        G.fill_(3.0)
        db.fill_(3.0)
        binding.dion2_linear_backward_weight(G, dY[:0], X[:0], dbias=db, accumulate=add)
        want = 3.0 if add else 0.0
        assert bool((G == want).all()) and bool((db == want).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", [a for a in ACTS])
def test_activation_backward(hip_device, act, dtype):
    for k, (t, w) in enumerate([(1, 1), (3, 7), (5, 129), (40, 1000), (333, 264)]):
        g = gen_of("act", act, k)
        lead, pad = [(0, 0), (1, 3), (8, 8)][k % 3]
        dY = rnd((t, w), dtype, g)
        z = rnd((t, w), F32, g, 3.0)
        z.view(-1)[:: 7] = 0.0
        z.view(-1)[3:: 11] *= 6.0        # far into the tails
        Z, dZ = Framed(t, w, dtype, lead, pad, z), Framed(t, w, dtype, 2 * lead, pad)
        binding.dion2_activation_backward(dZ.view, dY, Z.view, ACTIVATIONS[act])
        z, dy = Z.view.double(), dY.double()
        s = slope64(z, act)
        if act == "relu":
            s = torch.where(z > 0, 1.0, 0.0).double()      # 0 at 0
        err = dy.abs() * (ACT_ERR[dtype] * z.abs().clamp(min=1.0) if act not in ("none", "relu") else 0.0)
        near(dZ.view, dy * s, err + 2.0 ** -23 * (dy * s).abs(), dtype, "dZ")
        assert dZ.intact()
        binding.dion2_activation_backward(Z.view, dY, Z.view, ACTIVATIONS[act])      # in place of Z
        assert torch.equal(Z.view, dZ.view) and Z.intact()


@pytest.mark.parametrize("act", [a for a in ACTS if a != "none"])
def test_activation_slopes_are_differences(hip_device, act):
    """act' against central differences of act, both from the library, in fp32: an identity product's forward pass gives
    act. Step 2^-6: the difference's own error is at most h^2 / 6 max |act'''| (below 2.5 for these) plus 2 act errors
    over 2 h; ReLU away from its corner."""
    n, h = 64, 2.0 ** -6
    z = torch.linspace(-6.0, 6.0, 40 * n, device="cuda").view(40, n)
    if act == "relu":
        z = z[(z.abs() > 2 * h).all(1)]
    eye = torch.eye(n, device="cuda")
    up, down, slope = torch.empty_like(z), torch.empty_like(z), torch.empty_like(z)
    binding.dion2_linear_forward(up, z + h, eye, act=ACTIVATIONS[act])
    binding.dion2_linear_forward(down, z - h, eye, act=ACTIVATIONS[act])
    binding.dion2_activation_backward(slope, torch.ones_like(z), z, ACTIVATIONS[act])
    diff = (up.double() - down.double()) / (2 * h)
    assert float((diff - slope.double()).abs().max()) <= h * h * 2.5 / 6 + 2 * 1e-5 * 6 / (2 * h) * 0.5 + 1e-5


NORM_SIZES = [(1, 1), (1, 8), (1, 2048), (2, 7), (3, 64), (5, 130), (17, 512), (33, 1000), (64, 1001), (130, 2048),
              (300, 264), (9, 4096), (5, 4104), (7, 8200), (3, 16384), (2, 20001), (1030, 768)]


def norm_rows_in(t, c, dtype, g, lead, pad):
    """Rows of different size and offset, one constant row, one far from zero beside its spread."""
    x = torch.randn((t, c), generator=g, device="cuda") * torch.exp(torch.randn((t, 1), generator=g, device="cuda"))
    x += torch.randn((t, 1), generator=g, device="cuda")
    if t > 2:
        x[1] = 0.75
        x[2] += 100.0
    return Framed(t, c, dtype, lead, pad, x).view


def near_mean(c):
    """Bound on a mean's or mean square's relative error: each thread adds at most c / 64 + 8 terms, then eight levels."""
    return (c / 64 + 32) * 2.0 ** -24


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(NORM_SIZES)))
def test_layernorm_forward(hip_device, i, dtype):
    t, c = NORM_SIZES[i]
    g = gen_of("norm", i, dtype == BF)
    lead, pad = [(0, 0), (1, 3), (8, 64), (0, 8)][i % 4]
    X = norm_rows_in(t, c, dtype, g, lead, pad)
    pt = [dtype, F32, BF][i % 3]
    gamma = (1 + 0.2 * torch.randn(c, generator=g, device="cuda")).to(pt) if i % 4 != 3 else None
    beta = rnd((c,), pt, g, 0.3) if i % 5 != 4 else None
    Y, mean, rstd = Framed(t, c, dtype, lead, pad), Framed(1, t, F32), Framed(1, t, F32)
    binding.dion2_layernorm_forward(Y.view, X, gamma, beta, eps=EPS, mean=mean.view[0], rstd=rstd.view[0])
    x = X.double()
    mu = x.mean(1, keepdim=True)
    d = x - mu
    var = d.square().mean(1, keepdim=True)
    rs = 1.0 / torch.sqrt(var + EPS)
    xh, q = d * rs, near_mean(c)
    ga = 1.0 if gamma is None else gamma.double()
    be = 0.0 if beta is None else beta.double()
    y = xh * ga + be
    # the mean of the deviations is known to q of their magnitude (plus a rounding of x - mean, which q covers, and of the
    # mean that they are taken from, a factor 2^-24 of x: squared away), rstd to q and a few roundings
    spread = d.abs().mean(1, keepdim=True)
    err = ((2 * q + 2.0 ** -22) * xh.abs() + q * rs * spread + 2.0 ** -23 * rs * d.abs()) * (ga if gamma is None else ga.abs()) + 2.0 ** -22 * y.abs()
    near(Y.view, y, err, dtype, "Y")
    near(mean.view[0], mu[:, 0], (q * spread + 2.0 ** -23 * mu.abs())[:, 0], F32, "mean")
    near(rstd.view[0], rs[:, 0], ((2 * q + 2.0 ** -22) * rs)[:, 0], F32, "rstd")
    assert Y.intact() and mean.intact() and rstd.intact()
    y1 = Y.view.clone()
    binding.dion2_layernorm_forward(X, X, gamma, beta, eps=EPS)      # in place, without the statistics
    assert torch.equal(X, y1)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(NORM_SIZES)))
def test_layernorm_backward(hip_device, i, dtype):
    t, c = NORM_SIZES[i]
    g = gen_of("norm-grad", i, dtype == BF)
    lead, pad = [(0, 8), (0, 0), (1, 3), (8, 64)][i % 4]
    X = norm_rows_in(t, c, dtype, g, lead, pad)
    dY = Framed(t, c, dtype, lead, pad, rnd((t, c), F32, g, 1e-2)).view
    dR = Framed(t, c, dtype, lead, pad, rnd((t, c), F32, g, 1e-2)).view if i % 2 else None
    pt, gt, add = [F32, dtype, BF][i % 3], [BF, F32][(i + (dtype == BF)) % 2], i % 3 == 1
    gamma = (1 + 0.2 * torch.randn(c, generator=g, device="cuda")).to(pt) if i % 4 != 3 else None
    x = X.double()
    mean = x.mean(1).float()
    rstd = (1.0 / torch.sqrt((x - x.mean(1, keepdim=True)).square().mean(1) + EPS)).float()
    dg0, db0 = rnd((c,), gt, g, 0.1), rnd((c,), gt, g, 0.1)
    dX, dg, db = Framed(t, c, dtype, lead, pad), Framed(1, c, gt, 1, 0, dg0[None]), Framed(1, c, gt, 1, 0, db0[None])
    binding.dion2_layernorm_backward(dX.view, dY, X, mean, rstd, gamma=gamma, residual_grad=dR, dgamma=dg.view[0],
                                     dbeta=db.view[0], accumulate=add)
    rs, dy, q = rstd.double()[:, None], dY.double(), near_mean(c)
    xh = (x - mean.double()[:, None]) * rs
    h = dy if gamma is None else dy * gamma.double()
    m1, m2 = h.mean(1, keepdim=True), (h * xh).mean(1, keepdim=True)
    dx = rs * (h - m1 - xh * m2)
    err = rs * ((q + 2.0 ** -21) * (h.abs().mean(1, keepdim=True) + xh.abs() * (h * xh).abs().mean(1, keepdim=True))
                + 2.0 ** -21 * (h.abs() + m1.abs() + (xh * m2).abs()))
    if dR is not None:
        dx = dx + dR.double()
        err = err + 2.0 ** -23 * (dx.abs() + dR.double().abs())
    near(dX.view, dx, err, dtype, "dX")
    n = (t + 40) * 2.0 ** -23
    wg, wb = (dy * xh).sum(0), dy.sum(0)
    eg, eb = n * (dy * xh).abs().sum(0), n * dy.abs().sum(0)
    if add:
        wg, wb = wg + dg0.double(), wb + db0.double()
        eg, eb = eg + 2.0 ** -23 * wg.abs(), eb + 2.0 ** -23 * wb.abs()
    near(dg.view[0], wg, eg, gt, "dgamma")
    near(db.view[0], wb, eb, gt, "dbeta")
    assert dX.intact() and dg.intact() and db.intact()
    # each output by itself, and dX in place of dY: bitwise the same
    one = torch.empty_like(dX.view)
    binding.dion2_layernorm_backward(one, dY, X, mean, rstd, gamma=gamma, residual_grad=dR)
    assert torch.equal(one, dX.view)
    a, b = dg0.clone(), db0.clone()
    binding.dion2_layernorm_backward(None, dY, X, mean, rstd, gamma=gamma, dgamma=a, accumulate=add)
    binding.dion2_layernorm_backward(None, dY, X, mean, rstd, gamma=gamma, dbeta=b, accumulate=add)
    assert torch.equal(a, dg.view[0]) and torch.equal(b, db.view[0])
    if dR is not None:
        keep = dR.clone()
        binding.dion2_layernorm_backward(dR, dY, X, mean, rstd, gamma=gamma, residual_grad=dR, dgamma=a, dbeta=b)
        assert torch.equal(dR, dX.view)
        dR.copy_(keep)
    x0, a0, b0 = X.clone(), dg0.clone(), db0.clone()
    binding.dion2_layernorm_backward(X, dY, X, mean, rstd, gamma=gamma, residual_grad=dR, dgamma=a0, dbeta=b0, accumulate=add)
    assert torch.equal(X, dX.view) and torch.equal(a0, dg.view[0]) and torch.equal(b0, db.view[0])
    X.copy_(x0)
    binding.dion2_layernorm_backward(dY, dY, X, mean, rstd, gamma=gamma, residual_grad=dR, dgamma=a, dbeta=b)
    assert torch.equal(dY, dX.view)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("r,c", [(72, 40), (131, 77), (1032, 1040), (2056, 2056)])
def test_linear_calls_without_tokens(hip_device, r, c, dtype):
    """Gradients are sums of nothing, on every form of tile; the other calls write nothing."""
    X, dY = torch.empty((0, c), dtype=dtype, device="cuda"), torch.empty((0, r), dtype=dtype, device="cuda")
    W, Y, dX = torch.ones((r, c), dtype=dtype, device="cuda"), torch.empty_like(dY), torch.empty_like(X)
    binding.dion2_linear_forward(Y, X, W)
    binding.dion2_linear_backward_input(dX, dY, W)
    for g_dtype in (BF, F32):
        G, db = torch.full((r, c), 2.0, dtype=g_dtype, device="cuda"), torch.full((r,), 2.0, dtype=g_dtype, device="cuda")
        binding.dion2_linear_backward_weight(G, dY, X, dbias=db, accumulate=True)
        assert bool((G == 2).all()) and bool((db == 2).all())
        binding.dion2_linear_backward_weight(G, dY, X, dbias=db)
        assert bool((G == 0).all()) and bool((db == 0).all())
        db.fill_(2.0)
        binding.dion2_linear_backward_weight(None, dY, None, dbias=db)
        assert bool((db == 0).all())


def test_layernorm_backward_without_tokens(hip_device):
    z = torch.zeros((0, 40), device="cuda")
    s = torch.zeros(0, device="cuda")
    a, b = torch.full((40,), 2.0, device="cuda"), torch.full((40,), 2.0, device="cuda")
    binding.dion2_layernorm_backward(z, z, z, s, s, dgamma=a, dbeta=b, accumulate=True)
    assert bool((a == 2).all()) and bool((b == 2).all())
    binding.dion2_layernorm_backward(z, z, z, s, s, dgamma=a, dbeta=b)
    assert bool((a == 0).all()) and bool((b == 0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t,r,c", [(1, 64, 520), (40, 136, 136), (300, 272, 528), (300, 130, 77)])
def test_nan_and_inf_stay_where_they_belong(hip_device, t, r, c, dtype):
    """One NaN and one infinity in X (dY): the outputs of other tokens (rows of G of other units) are bitwise unchanged,
    also in tiles and slices that those share, at the last entry of a row among others."""
    g = gen_of("nan", t, r, c)
    X, W, dY = rnd((t, c), dtype, g), rnd((r, c), dtype, g, 0.1), rnd((t, r), dtype, g)
    Y, dX = torch.empty((t, r), dtype=dtype, device="cuda"), torch.empty((t, c), dtype=dtype, device="cuda")
    G, db = torch.empty((r, c), dtype=F32, device="cuda"), torch.empty(r, dtype=F32, device="cuda")

    def all_three():
        binding.dion2_linear_forward(Y, X, W, act=binding.ACT_GELU)
        binding.dion2_linear_backward_input(dX, dY, W)
        binding.dion2_linear_backward_weight(G, dY, X, dbias=db)
        return [v.clone() for v in (Y, dX, G, db)]

    y0, dx0, g0, b0 = all_three()
    tok = t // 2
    X[tok, c - 1] = float("nan")
    dY[tok, r - 1] = float("inf")
    y1, dx1, g1, b1 = all_three()
    other = torch.arange(t, device="cuda") != tok
    assert torch.equal(y1[other], y0[other]) and bool(y1[tok].isnan().all())
    assert torch.equal(dx1[other], dx0[other]) and not bool(dx1[tok].isfinite().any())
    assert torch.equal(g1[:-1, :-1], g0[:-1, :-1]) and bool(g1[:, -1].isnan().all()) and not bool(g1[-1].isfinite().any())
    assert torch.equal(b1[:-1], b0[:-1]) and bool(b1[-1].isinf())


def test_activations_of_infinities_and_nan(hip_device):
    inf, nan = float("inf"), float("nan")
    z = torch.tensor([[inf, nan, -inf, 0.0, -0.0, 1e30, -1e30, 3e38]] * 2, device="cuda")
    eye = torch.eye(8, device="cuda")
    for dt in (F32, BF):
        for act in ("relu", "gelu", "gelu_tanh", "silu"):
            x = torch.zeros((8, 8), dtype=dt, device="cuda")
            bias = z[0].to(dt)
            y = torch.empty_like(x)
            binding.dion2_linear_forward(y, x, eye.to(dt), bias=bias, act=ACTIVATIONS[act])
            v = y[0].float()
            assert v[0] == inf and v[1].isnan() and v[3] == 0 and v[4] == 0, act
            assert v[5] == bias[5].float() and v[6] == 0, act
            if act == "relu":
                assert v[2] == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_activations_of_large_values(hip_device, act, dtype):
    """From |z| = 200 on an activation is z or 0 and its slope 1 or 0, also where z^2 and z^3 are past fp32's range."""
    Z = torch.tensor([[200.0, 1e6, 1e13, 1e18, 3e19, 1e20, 1e30, 3e38]], device="cuda")
    Z = torch.cat([Z, -Z]).to(dtype)
    dZ, eye = torch.empty_like(Z), torch.eye(8, device="cuda").to(dtype)
    binding.dion2_activation_backward(dZ, torch.full_like(Z, 3.0), Z, ACTIVATIONS[act])
    assert torch.equal(dZ, 3.0 * (Z > 0).to(dtype))
    Y = torch.empty_like(Z)
    binding.dion2_linear_forward(Y, Z, eye, act=ACTIVATIONS[act])
    assert torch.equal(Y, Z.clamp(min=0))
    binding.dion2_linear_backward_input(dZ, torch.full_like(Z, 3.0), eye, Z=Z, act=ACTIVATIONS[act])
    assert torch.equal(dZ, 3.0 * (Z > 0).to(dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_layernorm_rows_of_nan_and_zero_variance(hip_device, dtype):
    X = torch.ones((6, 1000), dtype=dtype, device="cuda")
    X[2, 17] = float("nan")
    X[4, 999] = float("inf")
    Y = torch.empty_like(X)
    beta = torch.full((1000,), 0.5, device="cuda")
    binding.dion2_layernorm_forward(Y, X, None, beta, eps=EPS)
    assert bool((Y[[0, 1, 3, 5]] == 0.5).all())          # constant rows: no deviation, beta is left
    assert bool(Y[2].isnan().all()) and not bool(Y[4].isfinite().any())
    binding.dion2_layernorm_forward(Y, X, eps=0.0)       # 0 / 0, as the formula has it
    assert bool(Y[0].isnan().all())


def test_residual_in_place_and_slices_of_one_buffer(hip_device):
    """Y is the residual itself; X, Y, Z are column slices of one buffer."""
    g = gen_of("slices")
    for dt, t, r, c in ((BF, 200, 136, 264), (F32, 65, 40, 24), (BF, 4, 136, 264)):
        buf = rnd((t, c + 2 * r), dt, g)
        X, Y, Z = buf[:, :c], buf[:, c:c + r], buf[:, c + r:]
        W = rnd((r, c), dt, g, 0.1)
        want = torch.empty((t, r), dtype=dt, device="cuda")
        binding.dion2_linear_forward(want, X, W, residual=Y.clone(), act=binding.ACT_SILU)
        x0 = X.clone()
        binding.dion2_linear_forward(Y, X, W, residual=Y, Z=Z, act=binding.ACT_SILU)
        assert torch.equal(Y, want) and torch.equal(X, x0)
        dX, zc = torch.empty_like(X), X.clone()
        binding.dion2_linear_backward_input(dX, Y, W, Z=zc, act=binding.ACT_GELU)
        binding.dion2_linear_backward_input(zc, Y, W, Z=zc, act=binding.ACT_GELU)
        assert torch.equal(zc, dX)
        with pytest.raises(Dion2Error, match="overlaps"):
            binding.dion2_linear_forward(buf[:, c - 1:c - 1 + r], X, W)


CALLS = [(2, 520, 264), (300, 136, 264), (1100, 264, 520), (40, 130, 77)]


def every_call(t, r, c, dtype, seed, **kw):
    """One of each call on fresh inputs; returns (function that runs them, outputs)."""
    g = gen_of("every", t, r, c, seed)
    X, W, dY, R = rnd((t, c), dtype, g), rnd((r, c), dtype, g, 0.1), rnd((t, r), dtype, g), rnd((t, r), dtype, g)
    gamma, bias = rnd((c,), F32, g), rnd((r,), F32, g)
    new = lambda *s, d=dtype: torch.zeros(s, dtype=d, device="cuda")  # noqa: E731
    o = dict(Y=new(t, r), Z=new(t, r), dX=new(t, c), G=new(r, c, d=F32), db=new(r, d=F32), N=new(t, c), mean=new(t, d=F32),
             rstd=new(t, d=F32), dN=new(t, c), dg=new(c, d=F32), dbeta=new(c, d=F32), dZ=new(t, r))

    def run(stream=None):
        s = dict(stream=stream)
        binding.dion2_layernorm_forward(o["N"], X, gamma, eps=EPS, mean=o["mean"], rstd=o["rstd"], **s)
        binding.dion2_linear_forward(o["Y"], o["N"], W, bias=bias, residual=R, Z=o["Z"], act=binding.ACT_GELU, **s, **kw)
        binding.dion2_activation_backward(o["dZ"], dY, o["Z"], binding.ACT_GELU, **s)
        binding.dion2_linear_backward_input(o["dX"], o["dZ"], W, Z=X, act=binding.ACT_SILU, **s, **kw)
        binding.dion2_linear_backward_weight(o["G"], o["dZ"], o["N"], dbias=o["db"], **s, **kw)
        binding.dion2_layernorm_backward(o["dN"], o["dX"], X, o["mean"], o["rstd"], gamma=gamma, dgamma=o["dg"],
                                         dbeta=o["dbeta"], **s, **kw)
    return run, o


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t,r,c", CALLS)
def test_runs_repeat_bitwise_with_any_workspace_and_stream(hip_device, t, r, c, dtype):
    run, o = every_call(t, r, c, dtype, 0)
    run()
    first = {k: v.clone() for k, v in o.items()}
    need = max(binding.dion2_linear_workspace_size(t, r, c, dtype), binding.dion2_layernorm_workspace_size(t, c, dtype))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN bits
    for v in o.values():
        v.zero_()
    run2, o2 = every_call(t, r, c, dtype, 0, workspace=ws)
    run2()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for k in first:
        assert torch.equal(first[k], o2[k]), f"{k} with the caller's workspace"
        assert torch.equal(first[k], o[k]), f"{k} on another stream"


@pytest.mark.parametrize("t,r,c", [(2, 520, 264), (1100, 264, 520)])
def test_captured_calls(hip_device, t, r, c):
    """Captured with the caller's workspace and replayed with other inputs and eager work in between, while eager calls of
    the same kind use the library's workspace; without one a captured call that needs it is refused, and one that needs
    none is captured."""
    need = max(binding.dion2_linear_workspace_size(t, r, c), binding.dion2_layernorm_workspace_size(t, c))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    run, o = every_call(t, r, c, BF, 1, workspace=ws)
    run()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in o.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    other, oo = every_call(t, r, c, BF, 2)
    for i in range(4):
        for v in o.values():
            v.zero_()
        other()
        graph.replay()
        other()
        torch.cuda.synchronize()
        for k in o:
            assert torch.equal(o[k], want[k]), f"replay {i}: {k}"
    dY = torch.ones((64, 64), dtype=BF, device="cuda")
    db = torch.zeros(64, dtype=F32, device="cuda")
    dZ = torch.empty_like(dY)
    refused = torch.cuda.CUDAGraph()
    with torch.cuda.graph(refused):
        binding.dion2_activation_backward(dZ, dY, dY, binding.ACT_RELU)
        with pytest.raises(Dion2Error, match="captured") as e:
            binding.dion2_linear_backward_weight(None, dY, None, dbias=db)
    assert e.value.status == DION2_ERR_WORKSPACE
    refused.replay()
    torch.cuda.synchronize()
    assert torch.equal(dZ, dY)


def test_rows_past_2_31_entries(hip_device):
    """Activations of more than 2^31 entries: the last rows against a call on them alone."""
    t, c = 270_000, 8192
    X = torch.empty((t, c), dtype=BF, device="cuda")
    X[:1024] = rnd((1024, c), BF, gen_of("big"))
    for i in range(1024, t, 1024):
        n = min(1024, t - i)
        X[i:i + n] = X[:n] * 0.5
    tail = X[-300:].clone()
    W = rnd((64, c), BF, gen_of("bigw"), 0.02)
    Y, y1 = torch.empty((t, 64), dtype=BF, device="cuda"), torch.empty((300, 64), dtype=BF, device="cuda")
    binding.dion2_linear_forward(Y, X, W)
    z, err = product64(tail, W)
    near(Y[-300:], z, err, BF, "Y's last rows")
    dX = torch.empty_like(X)
    binding.dion2_linear_backward_input(dX, Y, W)
    z, err = product64(Y[-300:], W.t())
    near(dX[-300:], z, err, BF, "dX's last rows")
    binding.dion2_layernorm_forward(X, X, eps=EPS)
    n1 = torch.empty_like(tail)
    binding.dion2_layernorm_forward(n1, tail, eps=EPS)
    assert torch.equal(X[-300:], n1)
    dY = torch.zeros((t, 1), dtype=BF, device="cuda").expand(t, 1)
    del dX
    # only the last 300 tokens have a gradient: G is theirs
    dY = torch.zeros((t, 16), dtype=BF, device="cuda")
    dY[-300:] = rnd((300, 16), BF, gen_of("bigg"))
    G = torch.empty((16, c), dtype=F32, device="cuda")
    binding.dion2_linear_backward_weight(G, dY, X)
    want, _ = product64(dY[-300:].t(), X[-300:].t())
    near(G, want, (t + 16) * 2.0 ** -23 * (dY[-300:].double().abs().t() @ X[-300:].double().abs()), F32, "G")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_pitches(hip_device, dtype):
    """Rows 2^21 + 8 entries apart: more than the directly fed tiles address."""
    g = gen_of("pitch", dtype == BF)
    t, r, c, pitch = 70, 72, 136, (1 << 21) + 8
    buf = torch.zeros((t, pitch), dtype=dtype, device="cuda")
    X, dY = buf[:, :c], buf[:, c:c + r]
    X.copy_(rnd((t, c), dtype, g))
    dY.copy_(rnd((t, r), dtype, g))
    W, Y, G = rnd((r, c), dtype, g, 0.1), buf[:, 1024:1024 + r], torch.empty((r, c), dtype=F32, device="cuda")
    binding.dion2_linear_forward(Y, X, W)
    near(Y, *product64(X, W), dtype, "Y")
    binding.dion2_linear_backward_weight(G, dY, X)
    near(G, *product64(dY.t(), X.t()), F32, "G")
    dX = buf[:, 2048:2048 + c]
    binding.dion2_linear_backward_input(dX, dY, W)
    near(dX, *product64(dY, W.t()), dtype, "dX")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t,r,c", [(40, 72, 136), (300, 264, 1032), (2200, 2056, 136), (2200, 136, 2056)])
def test_pointers_between_vectors(hip_device, t, r, c, dtype):
    """Whole widths and pitches, but activations that start one entry past a 16-byte boundary."""
    g = gen_of("between", t, r, c, dtype == BF)
    X = Framed(t, c, dtype, 1, 8, rnd((t, c), dtype, g)).view
    dY = Framed(t, r, dtype, 1, 8, rnd((t, r), dtype, g, 1e-2)).view
    W, Y, dX = rnd((r, c), dtype, g, 0.1), Framed(t, r, dtype, 1, 8), Framed(t, c, dtype, 1, 8)
    G, db = torch.empty((r, c), dtype=F32, device="cuda"), torch.empty(r, dtype=F32, device="cuda")
    binding.dion2_linear_forward(Y.view, X, W)
    near(Y.view, *product64(X, W), dtype, "Y")
    binding.dion2_linear_backward_input(dX.view, dY, W)
    near(dX.view, *product64(dY, W.t()), dtype, "dX")
    binding.dion2_linear_backward_weight(G, dY, X, dbias=db)
    near(G, *product64(dY.t(), X.t()), F32, "G")
    near(db, dY.double().sum(0), (t + 16) * 2.0 ** -23 * dY.double().abs().sum(0), F32, "dbias")
    assert Y.intact() and dX.intact()


@pytest.mark.parametrize("t,r,c", [(300, 131, 517), (1100, 519, 263), (2500, 2051, 77), (3000, 131, 2055), (5, 1003, 2051)])
def test_odd_widths_with_the_callers_workspace(hip_device, t, r, c):
    """Widths that are no multiple of 8: operands are copied into the workspace, whose stated size is enough and whose
    content does not matter; without it the results are the same."""
    run, o = every_call(t, r, c, BF, 3)
    run()
    first = {k: v.clone() for k, v in o.items()}
    need = max(binding.dion2_linear_workspace_size(t, r, c), binding.dion2_layernorm_workspace_size(t, c))
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    run2, o2 = every_call(t, r, c, BF, 3, workspace=ws[:need])
    run2()
    torch.cuda.synchronize()
    for k in first:
        assert torch.equal(first[k], o2[k]), k
    assert bool((ws[need:] == 0xFF).all())


@pytest.mark.parametrize("t,r,c", [(300, 131, 517), (2500, 2051, 77), (3000, 131, 2055), (130, 1027, 1029), (1500, 1001, 1003)])
def test_odd_fp32_widths_with_the_callers_workspace(hip_device, t, r, c):
    """The same in fp32, where whole rows are multiples of four, against 64 bits; the workspace ends where it is said to."""
    g = gen_of("oddf", t, r, c)
    X, dY = Framed(t, c, F32, 4, 2, rnd((t, c), F32, g)).view, Framed(t, r, F32, 1, 1, rnd((t, r), F32, g, 1e-2)).view
    W, Y, dX = rnd((r, c), F32, g, 0.1), Framed(t, r, F32, 4, 3), Framed(t, c, F32, 2, 1)
    G, db = torch.empty((r, c), device="cuda"), torch.empty(r, device="cuda")
    need = binding.dion2_linear_workspace_size(t, r, c, F32, ld_x=c + 2, ld_dy=r + 1)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN wherever it is read unwritten
    for _ in range(2):
        binding.dion2_linear_forward(Y.view, X, W, workspace=ws[:need])
        near(Y.view, *product64(X, W), F32, "Y")
        binding.dion2_linear_backward_input(dX.view, dY, W, workspace=ws[:need])
        near(dX.view, *product64(dY, W.t()), F32, "dX")
        binding.dion2_linear_backward_weight(G, dY, X, dbias=db, workspace=ws[:need])
        near(G, *product64(dY.t(), X.t()), F32, "G")
        near(db, dY.double().sum(0), (t + 16) * 2.0 ** -23 * dY.double().abs().sum(0), F32, "dbias")
        ws[:need] = 0xFF
    assert Y.intact() and dX.intact() and bool((ws[need:] == 0xFF).all())


@pytest.mark.parametrize("cols", [5, 264, 2041, 5123])
@pytest.mark.parametrize("t", [1, 7, 16, 17, 32])
def test_few_tokens_of_any_width(hip_device, t, cols):
    """Up to 32 tokens take one form, whatever the width, the pitch and the alignment; no entry beside a row is read
    into it."""
    g = gen_of("few", t, cols)
    rows = 203
    W, bias = rnd((rows, cols), BF, g, 1.0 / math.sqrt(cols)), rnd((rows,), BF, g)
    for lead, pad in ((0, 0), (1, 3), (0, (1 << 21) + 8)):
        X, Y = Framed(t, cols, BF, lead, pad, rnd((t, cols), BF, g)), Framed(t, rows, BF, lead, pad % 64)
        X.buf[~X.used] = float("nan")
        binding.dion2_linear_forward(Y.view, X.view, W, bias=bias)
        want, bound = product64(X.view, W)
        near(Y.view, want + bias.double(), bound + 2.0 ** -22 * (want.abs() + bias.double().abs()), BF, (lead, pad))
        assert Y.intact()


@pytest.mark.parametrize("cols", [9, 1000, 2041, 5000, 20000])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_layernorm_of_large_constant_rows(hip_device, dtype, cols):
    """The variance of a constant row is 0 and what rounding makes of it is not below. The mean is off by at most
    (cols + 2) 2^-24 of it, the correction by as much of that, and rstd is at most 1 / sqrt(eps)."""
    value = torch.tensor([1.0, 1e6 / 3, -1e8 / 3, 1e9 / 7, 3.3e12], device="cuda").to(dtype)
    X = value[:, None].repeat(1, cols)
    Y, rstd = torch.empty_like(X), torch.empty(5, device="cuda")
    binding.dion2_layernorm_forward(Y, X, eps=EPS, rstd=rstd)
    assert bool(torch.isfinite(rstd).all()) and bool((rstd > 0).all()) and bool((rstd <= EPS ** -0.5 * (1 + 2.0 ** -20)).all())
    lim = ((cols + 2) * 2.0 ** -24) ** 2 * value.double().abs() * EPS ** -0.5 * (1 + 2.0 ** -6)
    assert bool((Y.double().abs() <= lim[:, None]).all())


def test_threads_share_a_stream(hip_device):
    """Two host threads, two calls each in turn, on one stream and the library's workspace: the calls take turns."""
    import threading
    jobs = [every_call(300, 136, 264, BF, s) for s in (5, 6)]
    for run, _ in jobs:
        run()
    torch.cuda.synchronize()
    want = [{k: v.clone() for k, v in o.items()} for _, o in jobs]
    fails = []

    def work(run, o, w):
        try:
            for _ in range(20):
                run()
        except Exception as e:   # noqa: BLE001 - reported by the test
            fails.append(e)

    threads = [threading.Thread(target=work, args=(run, o, w)) for (run, o), w in zip(jobs, want)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    torch.cuda.synchronize()
    assert not fails
    for (_, o), w in zip(jobs, want):
        for k in o:
            assert torch.equal(o[k], w[k]), k


def test_more_rows_than_a_launch_has_blocks(hip_device):
    """2^26 + 5 short rows: as many waves as would pass a launch's 2^32 threads."""
    t, c = (1 << 26) + 5, 8
    X = torch.zeros((t, c), dtype=BF, device="cuda")
    ends = torch.randn((64, c), generator=gen_of("rows"), device="cuda").to(BF)
    X[:64], X[-64:] = ends, ends
    binding.dion2_layernorm_forward(X, X, eps=EPS)
    want = torch.empty_like(ends)
    binding.dion2_layernorm_forward(want, ends, eps=EPS)
    assert torch.equal(X[:64], want) and torch.equal(X[-64:], want)
    assert bool((X[64:-64] == 0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_block_trains_with_the_step(hip_device, dtype):
    """x + W2 gelu(W1 norm(x) + b1) + b2, forward and backward by these calls and then the step on both matrices: the
    gradients against differentiating the same block in 64 bits, and the step from these G bitwise the step from copies."""
    t, d, h = 192, 264, 520
    g = gen_of("block", dtype == BF)
    x, dy = rnd((t, d), dtype, g), rnd((t, d), dtype, g, 1e-2)
    W1, W2 = rnd((h, d), dtype, g, 0.06), rnd((d, h), dtype, g, 0.04)
    b1, b2 = rnd((h,), dtype, g, 0.1), rnd((d,), dtype, g, 0.1)
    gamma, beta = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dtype), rnd((d,), dtype, g, 0.1)
    new = lambda *s, k=dtype: torch.empty(s, dtype=k, device="cuda")  # noqa: E731
    n, mean, rstd, z, a, y = new(t, d), new(t, k=F32), new(t, k=F32), new(t, h), new(t, h), new(t, d)
    binding.dion2_layernorm_forward(n, x, gamma, beta, eps=EPS, mean=mean, rstd=rstd)
    binding.dion2_linear_forward(a, n, W1, bias=b1, Z=z, act=binding.ACT_GELU)
    binding.dion2_linear_forward(y, a, W2, bias=b2, residual=x)
    dz, dn, dx = new(t, h), new(t, d), new(t, d)
    G1, G2, db1, db2, dg, db = new(h, d), new(d, h), new(h), new(d), new(d), new(d)
    binding.dion2_linear_backward_weight(G2, dy, a, dbias=db2)
    binding.dion2_linear_backward_input(dz, dy, W2, Z=z, act=binding.ACT_GELU)
    binding.dion2_linear_backward_weight(G1, dz, n, dbias=db1)
    binding.dion2_linear_backward_input(dn, dz, W1)
    binding.dion2_layernorm_backward(dx, dn, x, mean, rstd, gamma=gamma, residual_grad=dy, dgamma=dg, dbeta=db)
    leaves = [v.double().requires_grad_(True) for v in (x, W1, b1, W2, b2, gamma, beta)]
    X, V1, c1, V2, c2, ga, be = leaves
    nn = torch.nn.functional.layer_norm(X, (d,), ga, be, EPS)
    out = X + act64(nn @ V1.t() + c1, "gelu") @ V2.t() + c2
    want = torch.autograd.grad(out, leaves, dy.double())
    # Three intermediate tensors are stored in the activations' type, each rounded by half a step per entry: random, so
    # relative to an output's norm four half steps are far more than they add up to; fp32 sums of at most 520 terms.
    tol = 4 * HALF[dtype] + (0 if dtype == BF else 520 * 2.0 ** -24)
    for name, got, ref in (("y", y, out.detach()), *zip(("dx", "G1", "db1", "G2", "db2", "dgamma", "dbeta"),
                                                        (dx, G1, db1, G2, db2, dg, db), want)):
        assert float((got.double() - ref).norm() / ref.norm()) <= tol, name
    M1, M2 = torch.zeros(h, d, device="cuda"), torch.zeros(d, h, device="cuda")
    kept = [v.clone() for v in (W1, M1, G1, W2, M2, G2)]
    binding.dion2_step_groups([(W1[None], M1[None], G1[None], binding.AXIS_AUTO), (W2[None], M2[None], G2[None], binding.AXIS_AUTO)], 0.25)
    for i, (W, M, G) in enumerate(((W1, M1, G1), (W2, M2, G2))):
        w, m, gg = kept[3 * i:3 * i + 3]
        assert not torch.equal(W, w)
        binding.dion2_step_ex(w, m, gg, 0.25)
        assert torch.equal(W, w) and torch.equal(M, m)
