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
