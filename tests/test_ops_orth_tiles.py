"""Every product kernel of the orthogonalised updates against the iteration in
64 bits: stacks that take each of the five tiles for each of the three products
(which is checked on the CPU), with sides that are no multiples of the tiles,
lying and standing, in every type. Tolerances as in test_ops_orth.py."""
import os
import shutil
import subprocess

import pytest
import torch

from test_ops_orth import TYPES, check

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2504_01506_amd", "csrc")

# (batch, rows, cols): the tiles of X X^T, A A and B X
STACKS = {(1, 130, 129): "64 64 64", (1, 66, 965): "64k 64 64", (1, 961, 970): "64k 64k 64k",
          (60, 66, 390): "64 64 128", (59, 193, 202): "128 128 128", (29, 130, 1091): "64k 64 192",
          (28, 65, 2179): "64k 64 256", (42, 386, 427): "192 192 256", (38, 645, 836): "256 256 256",
          (1, 2500, 2600): "128 128 128"}
LARGE = {(1, 4096, 4096): "192 192 256", (1, 3903, 4041): "192 192 256"}


def test_the_stacks_take_every_tile(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path / "tiles_check")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-I", CSRC, os.path.join(HERE, "tiles_check.cpp"), "-o", exe],
                   check=True)
    stacks = {**STACKS, **LARGE}
    for turn in (1, -1):
        sizes = [str(v) for b, *sides in stacks for v in (b, *sides[::turn])]
        out = subprocess.run([exe, *sizes], capture_output=True, text=True, check=True).stdout.splitlines()
        assert out == list(stacks.values())
    for product in zip(*(t.split() for t in out)):
        assert set(product) == {"64k", "64", "128", "192", "256"}


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
