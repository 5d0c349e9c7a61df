"""What the linear calls ask for in workspace: host arithmetic, no GPU needed."""
import os
import random

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
