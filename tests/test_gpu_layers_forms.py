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
