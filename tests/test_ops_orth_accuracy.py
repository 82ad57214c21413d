"""Orthogonalised updates of every type are as exact as the same steps in fp32.

A step rounds each element of X, A and B to 22 bits, 2^-23 of it where fp32
rounds to 2^-24, and leaves out products of 2^-24: at most four times fp32's
roundings, which go through the same steps. The error of the iteration in fp32
on the same update is one sample of its own; twice as much for that. With y the
result before its rounding to bf16, w the exact one and |y - w| = e, an element
that rounds otherwise than w's has a border between y and w, so that its
rounded value is off by at most |round(w) - w| + 2 |y - w|: in norms, the
rounding of the exact result and 2 e."""
import pytest
import torch

A, B, C = 3.4445, -4.7750, 2.0315


def iterate(g, steps, kind, eps=1e-7):
    x = g.to(kind)
    if x.shape[0] > x.shape[1]:
        return iterate(g.t(), steps, kind, eps).t()
    x = x / (x.norm() + eps)
    for _ in range(steps):
        q = torch.mm(x, x.t().contiguous())
        x = A * x + torch.mm(B * q + C * torch.mm(q, q), x)
    return x


def updates():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)

    def r(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def basis(n, k):
        return torch.linalg.qr(r(n, k).double())[0].float()

    low = r(256, 64) @ r(64, 1024) / 8
    twins = r(80, 4000)
    return {"noise": r(160, 1000), "tall noise": r(1000, 160), "rank 64": r(160, 64) @ r(64, 4000),
            "square of rank 64": r(256, 64) @ r(64, 256), "rank 64 and noise of 1e-2": low + 1e-2 * r(256, 1024),
            "rank 64 and noise of 1e-3": low + 1e-3 * r(256, 1024),
            "rows nearly alike": torch.cat([twins, twins + r(80, 4000) / 64]),
            "near the identity": torch.eye(512, device="cuda") + 0.01 * r(512, 512),
            "singular values down to 1e-4": basis(130, 130) * torch.logspace(0, -4, 130, device="cuda") @
            basis(1000, 130).t().contiguous()}


NAMES = ["noise", "tall noise", "rank 64", "square of rank 64", "rank 64 and noise of 1e-2",
         "rank 64 and noise of 1e-3", "rows nearly alike", "near the identity", "singular values down to 1e-4"]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("name", NAMES)
def test_as_exact_as_steps_in_fp32(name, kind):
    from paper_2504_01506_amd import ops
    g = (0.01 * updates()[name]).to(kind)
    for steps in (1, 5, 6, 8, 30):
        want = iterate(g, steps, torch.float64)
        own = (iterate(g, steps, torch.float32).double() - want).norm()
        e = 8 * own + 2.0 ** -22 * want.norm()
        tol = (want.to(kind).double() - want).norm() + 2 * e
        off = (ops.orthogonalize(g, steps).double() - want).norm()
        print(f"{name} {kind} {steps}: off {off / want.norm():.2e}, allowed {tol / want.norm():.2e}", flush=True)
        assert off <= tol


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(128, 900), (129, 900), (300, 300), (1024, 1200)])
def test_a_bf16_update_is_the_same_update_in_fp32_rounded(rows, cols):
    """Same numbers, same steps: but for the last bit of the norm, whose sum is taken in another order, and so for
    elements at a border, of which bf16 has one in 2^16 fp32 steps."""
    from paper_2504_01506_amd import ops
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows)
    g = (0.01 * torch.randn((rows, cols), generator=gen, device="cuda")).bfloat16()
    got, want = ops.orthogonalize(g), ops.orthogonalize(g.float()).bfloat16()
    assert (got != want).float().mean() <= 1e-3
