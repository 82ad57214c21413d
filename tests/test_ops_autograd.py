"""The dense operators beside torch's autograd, which does not record them: no
result without the history that its inputs ask for, and no change of a saved
tensor that autograd does not learn of."""
import pytest
import torch


def calls(x, w, t):
    """The calls on rows x, a weight w and tokens t: each with the arguments that may ask for a gradient."""
    from paper_2504_01506_amd import ops
    s, e = torch.zeros((*x.shape[:1], 2), device=x.device), torch.zeros(x.shape[0], device=x.device)
    return [(lambda a, b, c, **out: ops.layer_norm(a, b, c, **out), (x, w, w.clone())),
            (lambda a, b, c, **out: ops.layer_norm_grad(a, b, c, **out), (x, w, x.clone())),
            (lambda a, b, c, d, f, **out: ops.log_probs_grad(a, t, b, c, d, f, **out),
             (x, s, e, e.clone(), e.clone())),
            (ops.orthogonalize, (x,)),
            (lambda a: ops.log_probs(a, t), (x,))]


def test_tensors_that_require_a_gradient_are_refused():
    x, w = torch.ones((6, 8)), torch.ones(8)
    every = calls(x, w, torch.zeros(6, dtype=torch.int64))
    for call, args in every:
        for k in range(len(args)):
            with pytest.raises(ValueError, match="autograd"):
                call(*(a.clone().requires_grad_(i == k) for i, a in enumerate(args)))
    for call, args in every[:-1]:
        with pytest.raises(ValueError, match="autograd"):
            call(*args, out=x.clone().requires_grad_(True))


@pytest.mark.gpu
def test_without_recording_they_are_taken():
    from paper_2504_01506_amd import ops
    x = torch.randn((6, 8), device="cuda")
    leaf, w = x.clone().requires_grad_(True), torch.ones(8, device="cuda", requires_grad=True)
    with pytest.raises(ValueError, match="autograd"):
        ops.layer_norm(leaf, w)
    want = ops.layer_norm(x, w.detach())
    assert torch.equal(ops.layer_norm(leaf.detach(), w.detach()), want)
    with torch.no_grad():
        assert torch.equal(ops.layer_norm(leaf, w), want)
        leaf.sub_(ops.orthogonalize(leaf))
    with torch.inference_mode():
        out = torch.empty((6, 8), device="cuda")
        assert torch.equal(ops.layer_norm(leaf, w, out=out), ops.layer_norm(leaf.detach(), w.detach()))


@pytest.mark.gpu
def test_from_a_function_of_autograds_own():
    from paper_2504_01506_amd import ops

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            ctx.save_for_backward(x, w)
            return ops.layer_norm(x, w, b)

        @staticmethod
        def backward(ctx, grad):
            return ops.layer_norm_grad(*ctx.saved_tensors, grad)

    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    x, w, b, dy = (torch.randn(s, generator=gen, device="cuda") for s in ((9, 70), 70, 70, (9, 70)))
    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    got = torch.autograd.grad(Norm.apply(*leaves), leaves, dy)
    for have, want in zip(got, ops.layer_norm_grad(x, w, dy)):
        assert torch.equal(have, want)


@pytest.mark.gpu
def test_a_given_output_counts_as_changed():
    from paper_2504_01506_amd import ops
    x, w = torch.randn((6, 8), device="cuda"), torch.ones(8, device="cuda")
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    for call, args in calls(x, w, t)[:-1]:
        leaf = torch.zeros((6, 8), device="cuda", requires_grad=True)
        saved = leaf.exp()                       # its gradient needs the result
        before = saved._version
        call(*args, out=saved.detach())
        assert saved._version > before
        with pytest.raises(RuntimeError, match="modified"):
            saved.sum().backward()
    square = torch.randn((7, 5), device="cuda")
    before = square._version
    ops.orthogonalize(square.t(), out=square.t())
    assert square._version > before
