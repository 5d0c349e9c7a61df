"""The layer calls refuse bad arguments before touching HIP (no GPU needed): the C entry points with made-up pointers
that are never read, and the binding's own checks of tensors."""
import ctypes

import pytest
import torch

from paper_2512_16928_amd import binding
from paper_2512_16928_amd.binding import (DION2_ERR_INVALID_ARG, DION2_ERR_UNSUPPORTED, DION2_ERR_WORKSPACE,
                                          DTYPE_F32, LayerOptions)

BASE = 1 << 40


def at(i):
    """Made-up device pointers, 64 GB apart: no two matrices below overlap."""
    return BASE + i * (1 << 36)


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(binding.LIB_PATH):
        from paper_2512_16928_amd import build
        build.build()
    return binding.load()


def options(**kw):
    opt = LayerOptions()
    binding.load().dion2_layer_options_init(ctypes.byref(opt))
    for k, v in kw.items():
        setattr(opt, k, v)
    return opt


def test_option_defaults_and_layout(lib):
    opt = options()
    assert (opt.dtype, opt.p_dtype, opt.g_dtype) == (1, 1, 1)
    assert opt.act == binding.ACT_NONE and opt.accumulate == 0 and not opt.workspace
    assert abs(opt.eps - 1e-5) < 1e-11
    assert all(getattr(opt, "ld_" + n) == 0 for n in ("x", "y", "z", "r", "dx", "dy", "dz", "dr"))


def test_option_layout_matches_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = "\n".join(f'printf("%zu\\n", offsetof(dion2_layer_options, {n}));' for n, _ in LayerOptions._fields_)
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "dion2.h"\nint main(void) {\n' + lines +
                   '\nprintf("%zu\\n", sizeof(dion2_layer_options));\nreturn 0;\n}\n')
    subprocess.run([cc, "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "layout")],
                   check=True, capture_output=True, timeout=120)
    out = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True, timeout=60).stdout.split()
    assert [int(v) for v in out] == [getattr(LayerOptions, n).offset for n, _ in LayerOptions._fields_] + \
        [ctypes.sizeof(LayerOptions)]


FORWARD = dict(Y=at(0), X=at(1), W=at(2), bias=at(3), R=at(4), Z=at(5), tokens=64, rows=96, cols=80)
INPUT = dict(dX=at(0), dY=at(1), W=at(2), Z=None, tokens=64, rows=96, cols=80)
WEIGHT = dict(G=at(0), dbias=at(1), dY=at(2), X=at(3), tokens=64, rows=96, cols=80)
ACT = dict(dZ=at(0), dY=at(1), Z=at(2), tokens=64, width=80)
NORM = dict(Y=at(0), mean=at(1), rstd=at(2), X=at(3), gamma=at(4), beta=at(5), tokens=64, cols=80)
NORM_GRAD = dict(dX=at(0), dgamma=at(1), dbeta=at(2), dY=at(3), X=at(4), mean=at(5), rstd=at(6), gamma=at(7), dR=at(8),
                 tokens=64, cols=80)
CALLS = {"dion2_linear_forward": FORWARD, "dion2_linear_backward_input": INPUT,
         "dion2_linear_backward_weight": WEIGHT, "dion2_activation_backward": ACT,
         "dion2_layernorm_forward": NORM, "dion2_layernorm_backward": NORM_GRAD}


@pytest.mark.parametrize("call,kw,opt,status,msg", [
    ("dion2_linear_forward", dict(Y=None), {}, DION2_ERR_INVALID_ARG, "Y must not be NULL"),
    ("dion2_linear_forward", dict(X=None), {}, DION2_ERR_INVALID_ARG, "X must not be NULL"),
    ("dion2_linear_forward", dict(W=None), {}, DION2_ERR_INVALID_ARG, "W must not be NULL"),
    ("dion2_linear_forward", dict(W=None, tokens=0), {}, DION2_ERR_INVALID_ARG, "W must not be NULL"),
    ("dion2_linear_forward", dict(W=at(2) + 8), {}, DION2_ERR_INVALID_ARG, "16-byte aligned"),
    ("dion2_linear_forward", dict(X=at(1) + 1), {}, DION2_ERR_INVALID_ARG, "X must be 2-byte aligned"),
    ("dion2_linear_forward", dict(X=at(1) + 2), dict(dtype=DTYPE_F32), DION2_ERR_INVALID_ARG, "4-byte aligned"),
    ("dion2_linear_forward", dict(bias=at(3) + 2), dict(p_dtype=DTYPE_F32), DION2_ERR_INVALID_ARG, "bias must be 4-byte"),
    ("dion2_linear_forward", dict(tokens=-1), {}, DION2_ERR_INVALID_ARG, "tokens"),
    ("dion2_linear_forward", dict(rows=0), {}, DION2_ERR_INVALID_ARG, "rows"),
    ("dion2_linear_forward", dict(cols=-4), {}, DION2_ERR_INVALID_ARG, "rows"),
    ("dion2_linear_forward", dict(tokens=1 << 31), {}, DION2_ERR_UNSUPPORTED, "tokens"),
    ("dion2_linear_forward", dict(rows=1 << 21, cols=8), {}, DION2_ERR_UNSUPPORTED, "sides"),
    ("dion2_linear_forward", dict(rows=1 << 16, cols=1 << 16), {}, DION2_ERR_UNSUPPORTED, "entries"),
    ("dion2_linear_forward", dict(tokens=(1 << 31) - 1, rows=1, cols=1), {}, DION2_ERR_UNSUPPORTED, "one launch"),
    ("dion2_linear_forward", dict(tokens=1 << 30, rows=64, cols=8), {}, DION2_ERR_UNSUPPORTED, "one launch"),
    ("dion2_layernorm_forward", dict(tokens=1 << 30), {}, DION2_ERR_UNSUPPORTED, "one launch"),
    ("dion2_linear_forward", {}, dict(ld_x=79), DION2_ERR_INVALID_ARG, "pitch of X"),
    ("dion2_linear_forward", {}, dict(ld_y=95), DION2_ERR_INVALID_ARG, "pitch of Y"),
    ("dion2_linear_forward", {}, dict(ld_z=-1), DION2_ERR_INVALID_ARG, "pitch of Z"),
    ("dion2_linear_forward", {}, dict(ld_r=1 << 28), DION2_ERR_INVALID_ARG, "pitch of R"),
    ("dion2_linear_forward", {}, dict(act=5), DION2_ERR_INVALID_ARG, "activation"),
    ("dion2_linear_forward", {}, dict(act=-1), DION2_ERR_INVALID_ARG, "activation"),
    ("dion2_linear_forward", {}, dict(dtype=2), DION2_ERR_INVALID_ARG, "dtype"),
    ("dion2_linear_forward", dict(Y=at(1)), {}, DION2_ERR_INVALID_ARG, "Y overlaps X"),
    ("dion2_linear_forward", dict(Y=at(2)), {}, DION2_ERR_INVALID_ARG, "Y overlaps W"),
    ("dion2_linear_forward", dict(Z=at(0) + 2), {}, DION2_ERR_INVALID_ARG, "Y overlaps Z"),
    ("dion2_linear_forward", dict(Z=at(4)), {}, DION2_ERR_INVALID_ARG, "Z overlaps R"),
    ("dion2_linear_forward", dict(R=at(0) + 16), {}, DION2_ERR_INVALID_ARG, "Y overlaps R"),
    ("dion2_linear_forward", dict(R=at(0)), dict(ld_r=128), DION2_ERR_INVALID_ARG, "Y overlaps R"),
    # column slices of one buffer of 170 that share a column
    ("dion2_linear_forward", dict(X=at(0) + 2 * 95), dict(ld_x=175, ld_y=175), DION2_ERR_INVALID_ARG, "Y overlaps X"),
    # slices of it that share none, but at another pitch
    ("dion2_linear_forward", dict(X=at(0) + 2 * 96), dict(ld_x=177, ld_y=176), DION2_ERR_INVALID_ARG, "Y overlaps X"),
    ("dion2_linear_forward", {}, dict(workspace=at(9) + 16, workspace_bytes=1 << 30), DION2_ERR_INVALID_ARG, "256-byte"),
    ("dion2_linear_backward_input", dict(dX=None), {}, DION2_ERR_INVALID_ARG, "dX must not be NULL"),
    ("dion2_linear_backward_input", dict(dY=None), {}, DION2_ERR_INVALID_ARG, "dY must not be NULL"),
    ("dion2_linear_backward_input", {}, dict(act=2), DION2_ERR_INVALID_ARG, "Z must not be NULL"),
    ("dion2_linear_backward_input", dict(Z=at(3)), {}, DION2_ERR_INVALID_ARG, "without an activation"),
    ("dion2_linear_backward_input", dict(dX=at(1)), {}, DION2_ERR_INVALID_ARG, "dX overlaps dY"),
    ("dion2_linear_backward_input", dict(Z=at(0) + 2), dict(act=1), DION2_ERR_INVALID_ARG, "dX overlaps Z"),
    ("dion2_linear_backward_weight", dict(G=None, dbias=None), {}, DION2_ERR_INVALID_ARG, "both be NULL"),
    ("dion2_linear_backward_weight", dict(X=None), {}, DION2_ERR_INVALID_ARG, "X must not be NULL"),
    ("dion2_linear_backward_weight", dict(G=at(0) + 8), {}, DION2_ERR_INVALID_ARG, "G must be 16-byte aligned"),
    ("dion2_linear_backward_weight", dict(G=at(2)), {}, DION2_ERR_INVALID_ARG, "G overlaps dY"),
    ("dion2_linear_backward_weight", dict(dbias=at(0) + 16), {}, DION2_ERR_INVALID_ARG, "G overlaps dbias"),
    ("dion2_linear_backward_weight", {}, dict(g_dtype=7), DION2_ERR_INVALID_ARG, "dtype"),
    ("dion2_linear_backward_weight", {}, dict(workspace=at(9), workspace_bytes=1), DION2_ERR_WORKSPACE, "below"),
    ("dion2_activation_backward", dict(dZ=None), {}, DION2_ERR_INVALID_ARG, "dZ must not be NULL"),
    ("dion2_activation_backward", dict(width=0), {}, DION2_ERR_INVALID_ARG, "rows, cols"),
    ("dion2_activation_backward", dict(dZ=at(1) + 2), {}, DION2_ERR_INVALID_ARG, "dZ overlaps dY"),
    ("dion2_layernorm_forward", dict(X=None), {}, DION2_ERR_INVALID_ARG, "X must not be NULL"),
    ("dion2_layernorm_forward", dict(mean=at(2) + 4), {}, DION2_ERR_INVALID_ARG, "mean overlaps rstd"),
    ("dion2_layernorm_forward", dict(gamma=at(0)), {}, DION2_ERR_INVALID_ARG, "Y overlaps gamma"),
    ("dion2_layernorm_forward", {}, dict(eps=-1.0), DION2_ERR_INVALID_ARG, "eps"),
    ("dion2_layernorm_forward", {}, dict(eps=float("nan")), DION2_ERR_INVALID_ARG, "eps"),
    ("dion2_layernorm_forward", dict(cols=(1 << 20) + 1), {}, DION2_ERR_UNSUPPORTED, "sides"),
    ("dion2_layernorm_backward", dict(mean=None), {}, DION2_ERR_INVALID_ARG, "mean must not be NULL"),
    ("dion2_layernorm_backward", dict(rstd=None), {}, DION2_ERR_INVALID_ARG, "rstd must not be NULL"),
    ("dion2_layernorm_backward", dict(dX=None, dgamma=None, dbeta=None, dR=None), {}, DION2_ERR_INVALID_ARG, "all be NULL"),
    ("dion2_layernorm_backward", dict(dX=None), {}, DION2_ERR_INVALID_ARG, "dR is given without dX"),
    ("dion2_layernorm_backward", dict(dX=at(3) + 2), {}, DION2_ERR_INVALID_ARG, "dX overlaps dY"),
    ("dion2_layernorm_backward", dict(dgamma=at(2)), {}, DION2_ERR_INVALID_ARG, "dgamma overlaps dbeta"),
    ("dion2_layernorm_backward", dict(dgamma=at(7)), {}, DION2_ERR_INVALID_ARG, "dgamma overlaps gamma"),
    ("dion2_layernorm_backward", {}, dict(workspace=at(9), workspace_bytes=64), DION2_ERR_WORKSPACE, "below"),
])
def test_refused(lib, call, kw, opt, status, msg):
    args = {**CALLS[call], **kw}
    o = options(**opt)
    assert getattr(lib, call)(*args.values(), ctypes.byref(o), None) == status
    assert msg in binding.dion2_last_error()


@pytest.mark.parametrize("call", sorted(set(CALLS) - {"dion2_linear_backward_weight", "dion2_layernorm_backward"}))
def test_no_tokens_is_no_work(lib, call):
    """Nothing is launched, so no GPU is needed; empty matrices may be NULL."""
    args = {**CALLS[call], "tokens": 0}
    assert getattr(lib, call)(*args.values(), None, None) == 0
    for name in ("X", "dX", "dY", "dZ", "Y", "Z", "R"):
        if name in args:
            args[name] = None
    assert getattr(lib, call)(*args.values(), None, None) == 0


def test_workspace_sizes(lib):
    assert binding.dion2_linear_workspace_size(-1, 64, 64) == 0
    assert binding.dion2_linear_workspace_size(64, 0, 64) == 0
    assert binding.dion2_layernorm_workspace_size(64, 0) == 0
    for t in (0, 1, 5, 300, 2048):
        for dt in (torch.bfloat16, torch.float32):
            assert binding.dion2_linear_workspace_size(t, 96, 80, dt) >= 96 * 4    # the bias gradient's partial sums
            assert binding.dion2_linear_workspace_size(t, 96, 80, dt) % 256 == 0
            assert binding.dion2_layernorm_workspace_size(t, 80, dt) >= 2 * 80 * 4
    bad = options(dtype=9)
    assert lib.dion2_linear_workspace_size(64, 64, 64, ctypes.byref(bad)) == 0




def test_binding_takes_device_tensors_only():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="HIP device tensor"):
        binding.dion2_linear_forward(x, x, x)
    with pytest.raises(ValueError, match="HIP device tensor"):
        binding.dion2_layernorm_forward(x, x)
    with pytest.raises(TypeError, match="torch tensor"):
        binding.dion2_linear_backward_weight(x, [1.0], x)


def test_binding_checks_shapes_types_and_strides():
    dev, bf, f32 = torch.device("cpu"), torch.bfloat16, torch.float32
    x = torch.zeros(6, 8, dtype=bf)
    assert binding._rows("X", None, torch.Size((6, 8)), bf, dev) == (None, 0)
    assert binding._rows("X", x, torch.Size((6, 8)), bf, dev) == (x.data_ptr(), 8)
    assert binding._rows("X", x[:, 2:5], torch.Size((6, 3)), bf, dev) == (x.data_ptr() + 4, 8)
    assert binding._rows("X", x[::2], torch.Size((3, 8)), bf, dev) == (x.data_ptr(), 16)
    assert binding._rows("X", x[:1].expand(1, 8), torch.Size((1, 8)), bf, dev) == (x.data_ptr(), 0)
    for t, shape, dt, msg in ((x, (6, 9), bf, "shape"), (x, (6, 8), f32, "float32"), (x.t(), (8, 6), bf, "unit stride"),
                              (x[:1].expand(6, 8), (6, 8), bf, "must not overlap"), (x[:, ::2], (6, 4), bf, "unit stride")):
        with pytest.raises(ValueError, match=msg):
            binding._rows("X", t, torch.Size(shape), dt, dev)
    with pytest.raises(ValueError, match="contiguous"):
        binding._whole("W", x.t(), torch.Size((8, 6)), (bf,), dev)
    with pytest.raises(ValueError, match="shape"):
        binding._whole("W", x, torch.Size((8, 6)), (bf,), dev)
    with pytest.raises(ValueError, match="one of"):
        binding._whole("G", x.to(torch.float16), x.shape, (bf, f32), dev)
    with pytest.raises(ValueError, match="one dtype"):
        binding._one_type("gamma and beta", x, x.float())


def test_copies_of_operands_are_bounded(lib):
    need = [binding.dion2_linear_workspace_size(t, 2047, 2048) for t in (1 << 18, 1 << 21)]
    assert need[0] >= 1 << 30 and need[1] <= (2 << 30) + (1 << 28)
    # a single row's pitch and up to 32 tokens' forward pass ask for nothing
    assert binding.dion2_linear_workspace_size(1, 64, 64, ld_x=1001) == binding.dion2_linear_workspace_size(1, 64, 64)
