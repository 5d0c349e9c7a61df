"""What the linear calls ask for in workspace: host arithmetic, no GPU needed."""
import ctypes
import os
import random
import re

import pytest
import torch

from paper_2512_16928_amd import binding

BF, F32 = torch.bfloat16, torch.float32
MIB = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2512_16928_amd import build
        build.build()
    return binding.load()


@pytest.mark.parametrize("t,r,c", [(1 << 18, 32000, 8192), (1 << 20, 50304, 4096), (1 << 18, 20000, 30000)])
def test_many_tiles_take_no_parts(t, r, c):
    """Thousands of output tiles: cutting K would gain next to nothing and a single part, 4 bytes an entry of G, is more
    than a gigabyte. What is left are the bias gradient's sums, a byte for eight entries at most."""
    assert binding.dion2_linear_workspace_size(t, r, c, BF) <= r * c // 8 + MIB


def test_parts_are_bounded():
    """2 GiB of copies, 512 MiB of parts and the bias gradient's sums (below 300 MiB, as rows * cols < 2^31), over all sizes."""
    rng = random.Random(5)
    size = lambda lo, hi: round(2.0 ** rng.uniform(lo, hi))  # noqa: E731
    checked = 0
    while checked < 4000:
        t, r, c = size(0, 20), size(3, 20), size(3, 20)
        if r * c >= 1 << 31 or -(-t // 64) * -(-max(r, c) // 64) >= 1 << 24:
            continue
        pad = rng.choice((0, 0, 3, 8))
        need = binding.dion2_linear_workspace_size(t, r, c, rng.choice((BF, F32)), ld_x=c + pad, ld_dy=r + pad)
        assert need <= 2048 * MIB + 512 * MIB + 300 * MIB, (t, r, c)
        checked += 1


def test_few_tiles_keep_their_parts():
    """Products of few tiles and a long sum are still cut."""
    for t, r, c in ((72, 520, 8200), (2048, 2048, 8192), (64, 2048, 8192)):
        assert binding.dion2_linear_workspace_size(t, r, c, BF) >= 2 * t * r * 4
    assert binding.dion2_linear_workspace_size(1 << 18, 128, 128, F32) >= 2 * 128 * 128 * 4


def bytes_asked(call, t, r, c, px=0, py=0, dtype=binding.DTYPE_BF16):
    """What one linear call asks for, from its refusal of a workspace of one byte. The pointers are made up: only where
    nothing can be launched."""
    if torch.cuda.is_available():
        pytest.skip("made-up pointers")
    at = lambda i: (1 << 40) + i * (1 << 36)  # noqa: E731
    opt = binding.LayerOptions()
    binding.load().dion2_layer_options_init(ctypes.byref(opt))
    opt.dtype, opt.ld_x, opt.ld_dy, opt.workspace, opt.workspace_bytes = dtype, c + px, r + py, at(9), 1
    lib = binding.load()
    args = {"forward": (lib.dion2_linear_forward, (at(0), at(1), at(2), None, None, None)),
            "input": (lib.dion2_linear_backward_input, (at(0), at(1), at(2), None)),
            "weight": (lib.dion2_linear_backward_weight, (at(0), None, at(1), at(2)))}[call]
    status = args[0](*args[1], t, r, c, ctypes.byref(opt), None)
    assert status == binding.DION2_ERR_WORKSPACE, (status, binding.dion2_last_error())
    return int(re.search(r"below the (\d+) needed", binding.dion2_last_error()).group(1))


def copy_of(rows, width, e=2):
    return -(-rows * -(-width * e // 16) * 16 // 256) * 256


# (tokens, rows, cols, how much longer than its width a row of X and of dY is, call, what is copied, parts): calls of
# test_gpu_layers_forms.py that run on copies in bf16, on tiles of 64, 128 and 256, whole and in parts
COPIED = [(1500, 1001, 1003, 0, 0, "forward", "XW", 0), (1500, 1001, 1003, 0, 0, "input", "YW", 0),
          (1500, 1001, 1003, 0, 0, "weight", "YX", 0), (2500, 2051, 1027, 0, 0, "forward", "XW", 0),
          (8191, 2047, 2041, 0, 0, "forward", "XW", 0), (8191, 2047, 2041, 0, 0, "input", "YW", 0),
          (8191, 2047, 2041, 0, 0, "weight", "YX", 2), (3000, 2048, 8192, 3, 5, "forward", "X", 2)]


@pytest.mark.parametrize("t,r,c,px,py,call,copied,parts", COPIED)
def test_bf16_copies_are_made_and_counted(t, r, c, px, py, call, copied, parts):
    """The bytes asked for are the copies' and the parts' to the byte, and within what is said to suffice."""
    want = sum({"X": copy_of(t, c), "Y": copy_of(t, r), "W": copy_of(r, c)}[k] for k in copied)
    m, n = {"forward": (t, r), "input": (t, c), "weight": (r, c)}[call]
    want += parts * -(-m // 32) * -(-n // 32) * 4096
    got = bytes_asked(call, t, r, c, px, py)
    assert got <= want + 255 and got >= want
    assert got <= binding.dion2_linear_workspace_size(t, r, c, BF, ld_x=c + px, ld_dy=r + py)
