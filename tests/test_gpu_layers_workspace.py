"""Layer calls and steps on one stream keep apart what the library holds for each."""
import pytest
import torch

from paper_2512_16928_amd import binding

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def test_layer_calls_leave_a_captured_step_its_workspace(hip_device):
    """A step captured on the library's workspace, layer calls of growing sizes on the same stream between its replays: the
    step's block stays where it is and keeps its order, so every replay is the eager step."""
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    side = torch.cuda.Stream()
    W, M, G = (torch.randn((256, 384), generator=g, device="cuda") * s for s in (0.02, 1e-3, 1e-3))
    W0, M0 = W.clone(), M.clone()
    sizes = [(300, 131, 517), (1500, 1001, 1003), (2500, 2051, 1027)]
    held = binding.dion2_workspace_size(1, 256, 384, 0.25)
    assert binding.dion2_linear_workspace_size(*sizes[-1]) > 4 * held
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.dion2_step_ex(W, M, G, 0.25)         # the workspace is there before the capture
        side.synchronize()
        W.copy_(W0)
        M.copy_(M0)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.dion2_step_ex(W, M, G, 0.25)
    wants = []
    w, m = W0.clone(), M0.clone()
    for _ in sizes:
        binding.dion2_step_ex(w, m, G, 0.25)
        wants.append((w.clone(), m.clone()))
    torch.cuda.synchronize()
    for (t, r, c), (w1, m1) in zip(sizes, wants):
        dY, X = (torch.randn((t, n), generator=g, device="cuda").to(BF) for n in (r, c))
        out, db = torch.empty((r, c), dtype=F32, device="cuda"), torch.empty(r, dtype=F32, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            binding.dion2_linear_backward_weight(out, dY, X, dbias=db)
            graph.replay()
            binding.dion2_linear_backward_weight(out, dY, X, dbias=db)
        torch.cuda.synchronize()
        assert torch.equal(W, w1) and torch.equal(M, m1), (t, r, c)
        a, b = dY.double().t().contiguous(), X.double()
        want, off = a @ b, (t + 16) * 2.0 ** -23 * (a.abs() @ b.abs())     # fp32 sums of t exact products, then one rounding
        assert bool(((out.double() - want).abs() <= off + 2.0 ** -24 * (want.abs() + off)).all())


def test_layer_calls_are_not_in_the_steps_measured_phases(hip_device):
    """The measurement hooks time steps: layer calls leave their totals at nothing."""
    X, W = torch.ones((40, 64), dtype=BF, device="cuda"), torch.ones((96, 64), dtype=BF, device="cuda")
    Y = torch.empty((40, 96), dtype=BF, device="cuda")
    before = binding.dion2_profile_enable(True)
    try:
        binding.dion2_profile_reset()
        binding.dion2_linear_forward(Y, X, W)
        binding.dion2_layernorm_forward(X, X)
        totals = binding.dion2_profile_read()
    finally:
        binding.dion2_profile_enable(before)
        binding.dion2_profile_reset()
    assert all(v["calls"] == 0 and v["launches"] == 0 and v["ms"] == 0 for v in totals.values())
