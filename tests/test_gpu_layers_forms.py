"""Forms of the products that particular sizes, pitches and alignments take, against 64 bits. The tolerances are those of
the sums: n exact (bf16) or 2^-23 (fp32) products added in fp32 in any order, (n + 16) 2^-23 sum |a b|, and half a step of
the output's type."""
import zlib

import pytest
import torch

from paper_2512_16928_amd import binding

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def normal(key, shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(zlib.crc32(repr(key).encode()))
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def rows_of(x, pad, lead=0):
    """x as part of a wider buffer of NaN: `pad` entries behind each row, `lead` before the first."""
    t, w = x.shape
    buf = torch.full((lead + t * (w + pad) + 8,), float("nan"), dtype=x.dtype, device="cuda")
    view = buf[lead:lead + t * (w + pad)].view(t, w + pad)[:, :w]
    return view.copy_(x)


def product64(a, b):
    """a b^T in 64 bits and the bound of fp32 sums of it."""
    a, b = a.double(), b.double().t().contiguous()
    return a @ b, (a.shape[1] + 16) * 2.0 ** -23 * (a.abs() @ b.abs())


def near(got, want, off, dtype, what):
    err = (got.double() - want).abs()
    lim = off + HALF[dtype] * (want.abs() + off) + 1e-37
    assert bool((err <= lim).all()), f"{what}: {float((err / lim).max())} of the limit"


# these make bf16 copies, as the tests of the workspace's size say
@pytest.mark.parametrize("t,r,c,px,py", [(1500, 1001, 1003, 0, 0), (2500, 2051, 1027, 0, 0), (8191, 2047, 2041, 0, 0),
                                         (3000, 2048, 8192, 3, 5), (2047, 1001, 4099, 1, 2)])
def test_bf16_copies_in_the_callers_workspace(hip_device, t, r, c, px, py):
    """Operands copied in whole chunks into a workspace of NaN that is as long as it is said to need: no entry is read that
    was not written, none written behind the end, and the library's own workspace gives the same bits."""
    X, dY = rows_of(normal(("X", t, c), (t, c), BF), px), rows_of(normal(("dY", t, r), (t, r), BF, 1e-2), py)
    W = normal(("W", r, c), (r, c), BF, 0.05)
    need = binding.dion2_linear_workspace_size(t, r, c, BF, ld_x=c + px, ld_dy=r + py)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN in bf16 and in fp32

    def calls(**kw):
        Y, dX = torch.empty((t, r), dtype=BF, device="cuda"), torch.empty((t, c), dtype=BF, device="cuda")
        G, db = torch.empty((r, c), device="cuda"), torch.empty(r, device="cuda")
        for f in (lambda: binding.dion2_linear_forward(Y, X, W, **kw),
                  lambda: binding.dion2_linear_backward_input(dX, dY, W, **kw),
                  lambda: binding.dion2_linear_backward_weight(G, dY, X, dbias=db, **kw)):
            ws.fill_(0xFF)
            f()
            assert bool((ws[need:] == 0xFF).all())
        return Y, dX, G, db

    Y, dX, G, db = out = calls(workspace=ws[:need])
    near(Y, *product64(X, W), BF, "Y")
    near(dX, *product64(dY, W.t()), BF, "dX")
    near(G, *product64(dY.t(), X.t()), F32, "G")
    near(db, dY.double().sum(0), (t + 16) * 2.0 ** -23 * dY.double().abs().sum(0), F32, "dbias")
    for a, b in zip(out, calls()):
        assert torch.equal(a, b)


# fp32 activations one entry past a 16-byte boundary: many tiles of 128 through registers, some of them partial, whole and
# (weight of the first, input gradient of the second, forward pass of the third) in parts
@pytest.mark.parametrize("t,r,c", [(4050, 2028, 2044), (2010, 8100, 2044), (1020, 1020, 8196)])
def test_large_fp32_products_between_vectors(hip_device, t, r, c):
    X, dY = rows_of(normal(("X", t, c), (t, c), F32), 8, 1), rows_of(normal(("dY", t, r), (t, r), F32, 1e-2), 8, 1)
    W = normal(("W", r, c), (r, c), F32, 0.05)
    Y, dX, G, db = (torch.empty(s, device="cuda") for s in ((t, r), (t, c), (r, c), (r,)))
    binding.dion2_linear_forward(Y, X, W)
    near(Y, *product64(X, W), F32, "Y")
    binding.dion2_linear_backward_input(dX, dY, W)
    near(dX, *product64(dY, W.t()), F32, "dX")
    binding.dion2_linear_backward_weight(G, dY, X, dbias=db)
    near(G, *product64(dY.t(), X.t()), F32, "G")
    near(db, dY.double().sum(0), (t + 16) * 2.0 ** -23 * dY.double().abs().sum(0), F32, "dbias")


def act64(z, act):
    if act == "relu":
        return torch.relu(z)      # its gradient at 0 is 0, as defined (that of a clamp is 1)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -(0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh((2.0 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


@pytest.mark.parametrize("t,r,c", [(2900, 2824, 1032), (2817, 2816, 1096)])
@pytest.mark.parametrize("act", sorted(binding.ACTIVATIONS))
def test_forward_epilogue_on_large_tiles(hip_device, act, t, r, c):
    """Tiles of 256 (the first size) and 128, whole ones and partial ones at both edges, K uncut: bias in the sums' start, Z, the activation and the
    residual (apart and in place) in one epilogue. Evaluating an activation is off by less than 2e-6 max(1, |z|), and its slope
    of at most 1.13 carries z's error on."""
    X, W = rows_of(normal(("X", t, c), (t, c), BF), 8), normal(("W", r, c), (r, c), BF, 1.5 / c ** 0.5)
    R = rows_of(normal(("R", t, r), (t, r), BF), 16)
    for bias_type in (BF, F32):
        bias = normal(("b", r), (r,), bias_type, 0.5)
        Y, Z = torch.empty((t, r), dtype=BF, device="cuda"), torch.empty((t, r), dtype=BF, device="cuda")
        binding.dion2_linear_forward(Y, X, W, bias=bias, residual=R, Z=Z, act=binding.ACTIVATIONS[act])
        z, off = product64(X, W)
        z = z + bias.double()
        off = off + 2.0 ** -23 * (z.abs() + bias.double().abs())
        near(Z, z, off, BF, "Z")
        y = act64(z, act)
        yoff = 1.13 * off + (2e-6 * z.abs().clamp(min=1.0) if act not in ("none", "relu") else 0.0)
        near(Y, y + R.double(), yoff + 2.0 ** -24 * (y + R.double()).abs(), BF, "Y")
        again = R.clone()
        binding.dion2_linear_forward(again, X, W, bias=bias, residual=again, act=binding.ACTIVATIONS[act])
        assert torch.equal(again, Y)
        alone = torch.empty_like(Y)
        binding.dion2_linear_forward(alone, X, W, act=binding.ACTIVATIONS[act])
        z = z - bias.double()
        near(alone, act64(z, act), 1.13 * off + 2e-6 * z.abs().clamp(min=1.0), BF, "without bias and residual")


@pytest.mark.parametrize("t,r,c", [(2900, 1032, 2824), (1030, 2904, 2824)])
@pytest.mark.parametrize("act", sorted(binding.ACTIVATIONS))
def test_input_gradient_epilogue_on_large_tiles(hip_device, act, t, r, c):
    """dX = (dY W) act'(Z) on tiles of 256 (the first size) and 64, apart and in place of Z. A slope is evaluated to less than
    2e-6 max(1, |z|)."""
    dY, W = rows_of(normal(("dY", t, r), (t, r), BF, 1e-2), 8), normal(("W", r, c), (r, c), BF, 0.1)
    Z = rows_of(normal(("Z", t, c), (t, c), BF, 2.0), 24)
    dX = torch.empty((t, c), dtype=BF, device="cuda")
    given = Z if act != "none" else None
    binding.dion2_linear_backward_input(dX, dY, W, Z=given, act=binding.ACTIVATIONS[act])
    p, off = product64(dY, W.t())
    if act != "none":
        z = Z.double().requires_grad_(True)
        s = torch.autograd.grad(act64(z, act).sum(), z)[0]
        off = off * s.abs() + p.abs() * (2e-6 * Z.double().abs().clamp(min=1.0)) + 2.0 ** -24 * (p * s).abs()
        p = p * s
    near(dX, p, off, BF, "dX")
    if act != "none":
        binding.dion2_linear_backward_input(Z, dY, W, Z=Z, act=binding.ACTIVATIONS[act])
        assert torch.equal(Z, dX)
