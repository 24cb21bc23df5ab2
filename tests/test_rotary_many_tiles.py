"""rotary_kernel's way through its tiles at the largest numbers that the interface takes: B * N below 2^31, a tile for each sequence of one token."""
import os
import re

import numpy as np
import pytest
import torch

from paper_2509_22323_b200 import binding, build

TYPES = {"int": np.int32, "uint32_t": np.uint32, "long long": np.int64}


@pytest.mark.parametrize("tiles", [1, 1 << 30, (1 << 30) + 5, (1 << 31) - 1])
@pytest.mark.parametrize("most", [(1 << 31) - 1, 592])
def test_a_thread_block_leaves_after_its_tiles(tiles, most):
    """The loop as the source has it, in the source's type: the last thread block's tiles, of a grid of `most` thread blocks at most."""
    with open(os.path.join(build.CSRC, "k7_rotary.cu")) as f:
        (kind,) = re.findall(r"for \((\S[\w ]*) tile = blockIdx\.x; tile < (?:\(\w+\))?p\.n_tiles; tile \+= gridDim\.x\)", f.read())
    grid = min(tiles, most)
    at = tiles - 1 - (tiles - 1) % grid                              # the block's last tile is among these
    with np.errstate(over="ignore"):
        for block in {0, grid - 1, (tiles - 1) % grid}:
            tile = TYPES[kind](at + block if at + block < tiles else at + block - grid)
            assert 0 <= tile < tiles
            tile = np.add(tile, TYPES[kind](grid), dtype=TYPES[kind])
            assert not tile < tiles, "reads and writes rows that are not there"


@pytest.mark.gpu
def test_more_than_2_to_the_30_sequences():
    """One head of 16 channels, one token, in place: 34 GB, with rows in front and behind that stay as they were."""
    B, D, edge = (1 << 30) + 5, 16, 64
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB")
    freq = binding.rapid3_rotary_freqs(D)[0].cuda()
    rotary = binding.Rotary("pairs", freq, torch.full((1, 1, 1), 3, dtype=torch.int32, device="cuda"))
    row = torch.linspace(-2, 2, D, device="cuda").to(torch.bfloat16)
    want = binding.rapid3_rotary(row.view(1, 1, 1, D), None, rotary)[0].view(D)
    assert not torch.equal(row, want)
    buffer = torch.empty((B + 2 * edge, D), dtype=torch.bfloat16, device="cuda")
    buffer.copy_(row.expand_as(buffer))
    x = buffer[edge:edge + B].view(B, 1, 1, D)
    binding.rapid3_rotary(x, None, rotary, x)
    for at in range(0, B, 1 << 26):
        assert (buffer[edge + at:edge + min(B, at + (1 << 26))] == want).all()
    assert (buffer[:edge] == row).all() and (buffer[edge + B:] == row).all()
    del buffer, x
    torch.cuda.empty_cache()
