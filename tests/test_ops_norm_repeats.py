"""Layer norm and its gradient give equal bits on equal calls, also where the
last elements of a row are written by two lanes (rows that are no whole number
of vectors): both must round them alike."""
import pytest
import torch


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,dim", [(200_000, 9), (200_000, 13), (100_000, 45), (30_000, 515), (20_000, 1021), (4000, 7170),
                                   (1069, 7170), (2000, 12_909)])
def test_equal_calls_give_equal_bits(n, dim, kind):
    from paper_2504_01506_amd import ops
    gen = torch.Generator(device="cuda")
    gen.manual_seed(dim)
    x, dy = torch.randn((2, n, dim), generator=gen, device="cuda").to(kind)
    w, b = torch.randn((2, dim), generator=gen, device="cuda").to(kind)
    first = (ops.layer_norm(x, w, b), *ops.layer_norm_grad(x, w, dy))
    for _ in range(8):
        for p, q in zip((ops.layer_norm(x, w, b), *ops.layer_norm_grad(x, w, dy)), first):
            assert torch.equal(p, q), (p != q).sum().item()


@pytest.mark.gpu
def test_rounding_does_not_depend_on_the_place():
    """The same numbers at every place of a vector, rows of ones and twos in turn: a row's equal elements are equal."""
    from paper_2504_01506_amd import ops
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    values = torch.randn((100_000, 2), generator=gen, device="cuda")
    for dim in (16, 30, 64, 1026):
        x = values.repeat_interleave(dim // 2, 1).half()            # first half one value, second half another
        y = ops.layer_norm(x, torch.full((dim,), 1.37, device="cuda"), torch.full((dim,), 0.61, device="cuda"))
        assert (y[:, :dim // 2] == y[:, :1]).all() and (y[:, dim // 2:] == y[:, -1:]).all()
