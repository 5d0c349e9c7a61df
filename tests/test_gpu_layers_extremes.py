"""Layer calls at the ends of their ranges: the largest matrices, the most tokens, parameters that start between vectors, and
the library's workspaces released between calls."""
import pytest
import torch

from paper_2512_16928_amd import binding

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: 2.0 ** -24}


def normal(seed, shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for i in range(0, shape[0], 1 << 18):
        n = min(1 << 18, shape[0] - i)
        out[i:i + n] = torch.randn((n, *shape[1:]), generator=g, device="cuda") * scale
    return out


def product64(a, b):
    a, b = a.double(), b.double().t().contiguous()
    return a @ b, (a.shape[1] + 16) * 2.0 ** -23 * (a.abs() @ b.abs())


def near(got, want, off, dtype, what):
    err, lim = (got.double() - want).abs(), off + HALF[dtype] * (want.abs() + off) + 1e-37
    assert bool((err <= lim).all()), f"{what}: {float((err / lim).max())} of the limit"


@pytest.mark.parametrize("t,r,c", [(40, 1 << 20, 2040), (3, 1 << 20, 2047), (70, 2041, (1 << 20) - 3)])
def test_the_longest_weights(hip_device, t, r, c):
    """Sides of 2^20 and close to 2^31 entries: the first and the last rows and columns against 64 bits. Of odd width their
    copies would pass what is copied."""
    X, dY, W = normal(1, (t, c), BF), normal(2, (t, r), BF, 1e-2), normal(3, (r, c), BF, 0.02)
    Y, dX = torch.empty((t, r), dtype=BF, device="cuda"), torch.empty((t, c), dtype=BF, device="cuda")
    G, db = torch.empty((r, c), dtype=BF, device="cuda"), torch.empty(r, dtype=BF, device="cuda")
    binding.dion2_linear_forward(Y, X, W)
    binding.dion2_linear_backward_weight(G, dY, X, dbias=db)
    binding.dion2_linear_backward_input(dX, dY, W)
    for rows in (slice(0, 130), slice(r - 130, r)):
        near(Y[:, rows], *product64(X, W[rows]), BF, "Y")
        near(db[rows], dY[:, rows].double().sum(0), (t + 16) * 2.0 ** -23 * dY[:, rows].double().abs().sum(0), BF, "dbias")
        for cols in (slice(0, 130), slice(c - 130, c)):
            near(G[rows, cols], *product64(dY[:, rows].t(), X[:, cols].t()), BF, "G")
    for cols in (slice(0, 130), slice(c - 130, c)):
        near(dX[:, cols], *product64(dY, W[:, cols].t()), BF, "dX")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_most_tokens(hip_device, dtype):
    """2^26 + 5 tokens of eight entries: the first and the last against 64 bits, and a gradient that all but those leave at 0."""
    t, r, c = (1 << 26) + 5, 8, 8
    ends = [slice(0, 300), slice(t - 300, t)]
    X, dY = torch.ones((t, c), dtype=dtype, device="cuda"), torch.zeros((t, r), dtype=dtype, device="cuda")
    for i, rows in enumerate(ends):
        X[rows], dY[rows] = normal(10 + i, (300, c), dtype), normal(20 + i, (300, r), dtype)
    W, Y, dX = normal(3, (r, c), dtype), torch.empty_like(dY), torch.empty_like(X)
    G, db = torch.empty((r, c), device="cuda"), torch.empty(r, device="cuda")
    binding.dion2_linear_forward(Y, X, W)
    binding.dion2_linear_backward_input(dX, dY, W)
    binding.dion2_linear_backward_weight(G, dY, X, dbias=db)
    for rows in ends:
        near(Y[rows], *product64(X[rows], W), dtype, "Y")
        near(dX[rows], *product64(dY[rows], W.t()), dtype, "dX")
    assert bool((dX[300:-300] == 0).all()) and bool((Y[300:-300] == Y[300]).all())
    x, dy = (torch.cat([v[rows] for rows in ends]) for v in (X, dY))     # zeros change no sum
    near(G, *product64(dy.t(), x.t()), F32, "G")
    near(db, dy.double().sum(0), 616 * 2.0 ** -23 * dy.double().abs().sum(0), F32, "dbias")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("t,r,c", [(5, 264, 136), (300, 264, 520), (40, 203, 1001), (2900, 2824, 264)])
def test_parameters_between_vectors(hip_device, t, r, c, dtype):
    """bias, gamma, beta and the gradients of parameters as slices of one flat buffer, one entry past a 16-byte boundary:
    bitwise the same as tensors of their own, and nothing beside them written."""
    X, W, dY = normal(1, (t, c), dtype), normal(2, (r, c), dtype, 0.05), normal(3, (t, r), dtype)
    flat = normal(4, (1 + r + 2 * c + 3,), dtype)
    grad = torch.full_like(flat, 7.0)

    def parts(v):
        return v[1:1 + r], v[1 + r:1 + r + c], v[1 + r + c:1 + r + 2 * c]

    def calls(bias, gamma, beta, db, dg, dbeta):
        N, Y, dX, dN = torch.empty_like(X), torch.empty_like(dY), torch.empty_like(X), torch.empty_like(X)
        mean, rstd = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
        binding.dion2_layernorm_forward(N, X, gamma, beta, mean=mean, rstd=rstd)
        binding.dion2_linear_forward(Y, N, W, bias=bias, act=binding.ACT_SILU)
        binding.dion2_linear_backward_weight(None, dY, None, dbias=db)
        binding.dion2_linear_backward_input(dX, dY, W)
        binding.dion2_layernorm_backward(dN, dX, X, mean, rstd, gamma=gamma, dgamma=dg, dbeta=dbeta)
        return N, Y, dX, dN, db, dg, dbeta

    own = calls(*(p.clone() for p in parts(flat)), *(p.clone() for p in parts(grad)))
    for a, b in zip(own, calls(*parts(flat), *parts(grad))):
        assert torch.equal(a, b)
    assert bool((grad[0] == 7) and (grad[1 + r + 2 * c:] == 7).all())


def test_released_workspaces_come_back(hip_device):
    """dion2_release_workspaces between layer calls and steps: the next call takes new ones and gives the same."""
    X, dY = normal(1, (300, 517), BF), normal(2, (300, 131), BF)
    G, db = torch.empty((131, 517), device="cuda"), torch.empty(131, device="cuda")
    W, M = normal(3, (131, 517), F32, 0.02).contiguous(), torch.zeros((131, 517), device="cuda")
    seen = []
    for _ in range(3):
        w, m = W.clone(), M.clone()
        binding.dion2_linear_backward_weight(G, dY, X, dbias=db)
        binding.dion2_step_ex(w, m, G, 0.25)
        seen.append((G.clone(), db.clone(), w, m))
        torch.cuda.synchronize()
        binding.dion2_release_workspaces()
    for later in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], later))
