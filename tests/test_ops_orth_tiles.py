"""Every product kernel of the orthogonalised updates against the iteration in
64 bits: stacks that take each of the five tiles for each of the three products,
with sides that are no multiples of the tiles, lying and standing, in every
type. Tolerances as in test_ops_orth.py."""
import pytest
import torch

from test_ops_orth import TYPES, check

# (batch, rows, cols): the tiles of X X^T, A A and B X
STACKS = {(1, 130, 129): "64 64 64", (1, 66, 965): "64k 64 64", (1, 961, 970): "64k 64k 64k",
          (60, 66, 390): "64 64 128", (59, 193, 202): "128 128 128", (29, 130, 1091): "64k 64 192",
          (28, 65, 2179): "64k 64 256", (42, 386, 427): "192 192 256", (38, 645, 836): "256 256 256",
          (1, 2500, 2600): "128 128 128"}
LARGE = {(1, 4096, 4096): "192 192 256", (1, 3903, 4041): "192 192 256"}


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("batch,rows,cols", STACKS)
def test_stacks_of_every_tile(batch, rows, cols, kind):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    g = 0.01 * torch.randn((batch, rows, cols), generator=gen, device="cuda")
    check(g.to(kind))
    check(g.to(kind).mT.contiguous())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("batch,rows,cols", LARGE)
def test_large_ones(batch, rows, cols, kind):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    check((0.01 * torch.randn((rows, cols), generator=gen, device="cuda")).to(kind))
