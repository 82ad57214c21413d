"""Layer norm's gradient: how its sums over rows are joined."""
import pytest
import torch


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim", [1, 2, 3, 7, 8, 10, 16, 33, 64, 200, 256, 1000])
def test_a_block_joins_its_threads_in_64_bits(dim, kind):
    """Ones but for 2^25 and -2^25, which lie in different threads of a block: its sum over n rows, n - 2, is exact
    if the threads' sums (whole numbers below 2^26, of few rows each) are added in 64 bits. In 32 bits the
    ones beside 2^25 are lost."""
    from paper_2504_01506_amd import ops
    short = dim * torch.finfo(kind).bits < 128
    n = 256 if short else 4          # one block: a row a thread, or a row a group of lanes
    x = torch.randn((n, dim), device="cuda").to(kind)
    dy = torch.ones((n, dim), device="cuda", dtype=kind)
    dy[0], dy[n // 2] = 2.0 ** 25, -2.0 ** 25
    db = ops.layer_norm_grad(x, torch.ones(dim, device="cuda"), dy)[2]
    assert (db == n - 2).all(), db


@pytest.mark.gpu
@pytest.mark.parametrize("n,dim,kind", [
    (n, dim, kind) for n, dim in ((9, 2), (2, 2), (54_754, 1), (54_754, 2), (30_000, 3), (1, 3), (70_001, 5))
    for kind in (torch.float32, torch.bfloat16, torch.float16) if dim * torch.finfo(kind).bits < 128])
def test_rows_shorter_than_16_bytes_lose_nothing_where_terms_cancel(n, dim, kind):
    """Two elements leave a gradient of eps' size alone, a column of many a sum near zero: held in 64 bits, both are
    off by the output's rounding. (What 64 bits themselves lose, 2^-50 of the terms' sizes, is allowed beside.)"""
    from paper_2504_01506_amd import ops
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n + dim)
    x = torch.randn((n, dim), generator=gen, device="cuda").to(kind)
    dy = (0.01 * torch.randn((n, dim), generator=gen, device="cuda")).to(kind)
    w = (1 + 0.2 * torch.randn(dim, generator=gen, device="cuda")).to(kind)
    got = ops.layer_norm_grad(x, w, dy, 1e-5)
    eps = float(torch.tensor(1e-5, dtype=torch.float32))
    xd, g = x.double(), dy.double() * w.double()
    d = xd - xd.sum(1, keepdim=True) / dim
    r = 1 / ((d * d).sum(1, keepdim=True) / dim + eps).sqrt()
    h = d * r
    gm, ghm = g.sum(1, keepdim=True) / dim, (g * h).sum(1, keepdim=True) / dim
    size = r * (g.abs() + gm.abs() + (h * ghm).abs() + g.abs().amax(1, keepdim=True))
    for have, want, terms in ((got[0], r * (g - gm - h * ghm), size), (got[1], (dy.double() * h).sum(0), (dy.double() * h).abs().sum(0)),
                              (got[2], dy.double().sum(0), dy.double().abs().sum(0))):
        # (rounded to fp32 and then to 16 bits: half a step of each)
        tol = want.abs() * (torch.finfo(kind).eps / 2 + 2.0 ** -23) + 2.0 ** -48 * terms + torch.finfo(kind).smallest_normal
        assert ((have.double() - want).abs() <= tol).all(), ((have.double() - want).abs() / tol).max().item()
