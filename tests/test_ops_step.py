"""The dense operators together with a table, as a training step of a token
model uses them: get the tokens' rows, normalise them, two products, the log
probabilities of the next tokens, and all of it backwards into put_grad and an
orthogonalised update. Against the same step in 64 bits, the table's part by
the CPU oracle on the gradients that the step gave it."""
import numpy as np
import pytest
import torch

from oracle import oracle as O
from paper_2504_01506_amd import mlkv

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def reference(rows, w, b, dense, head, targets, coef):
    """loss and its gradients in 64 bits; targets < 0 do not count."""
    rows, w, b, dense, head = (t.double().detach().requires_grad_(True) for t in (rows, w, b, dense, head))
    mu = rows.mean(1, keepdim=True)
    h = (rows - mu) / ((rows - mu).square().mean(1, keepdim=True) + 1e-5).sqrt() * w + b
    lp = torch.log_softmax(torch.relu(h @ dense) @ head, 1)
    ent = -(lp.exp() * lp).sum(1)
    logp = torch.where(targets < 0, 0.0, lp.gather(1, targets.clamp(min=0)[:, None])[:, 0])
    loss = -(logp.sum() + coef * ent.sum()) / targets.numel()
    return loss, torch.autograd.grad(loss, (rows, w, b, dense, head))


@pytest.mark.parametrize("n,dim,vocab,ids", [(1, 16, 40, 50), (700, 64, 1000, 900), (1333, 100, 5003, 300)])
def test_training_steps_of_a_token_model(n, dim, vocab, ids):
    from paper_2504_01506_amd import ops
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    rng = np.random.default_rng(n)
    t, o = mlkv.Table(dim, 4096), O.OracleTable(dim, 4096)
    w, b = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
    dense = torch.randn((dim, dim), generator=gen, device="cuda") / dim ** 0.5
    head = torch.randn((dim, vocab), generator=gen, device="cuda") / dim ** 0.5
    coef = 0.01
    for step in range(3):
        keys = rng.integers(0, ids, size=n).astype(np.uint64)     # tokens repeat
        targets = torch.from_numpy(rng.integers(0, vocab, size=n)).cuda()
        targets[::7] = -1
        k = torch.from_numpy(keys.view(np.int64)).cuda()
        rows = t.get(k, torch.empty((n, dim), device="cuda"))
        x = ops.layer_norm(rows, w, b)
        mid = x @ dense
        act = torch.relu(mid)
        logits = act @ head
        r = ops.log_probs(logits, targets, top=3)
        assert torch.equal(r.top_ids[:, 0], logits.argmax(1))
        scale = torch.full((n,), -1.0 / n, device="cuda")
        g = ops.log_probs_grad(logits, targets, r.stats, r.entropy, scale, scale * coef, out=logits)
        g_head, g_act = act.t() @ g, g @ head.t()
        g_mid = g_act * (mid > 0)
        g_dense = x.t() @ g_mid
        g_rows, g_w, g_b = ops.layer_norm_grad(rows, w, g_mid @ dense.t())

        loss, want = reference(rows, w, b, dense, head, targets, coef)
        got = -(r.logp.sum() + coef * r.entropy.sum()) / n
        # fp32 products of dim and vocab terms on both ways: their sums' roundings, 2 u a term at most
        assert abs(got.item() - loss.item()) <= 2 * U * (dim + 200) * (1 + abs(loss.item()))
        for name, have, ref in zip(("rows", "w", "b", "dense", "head"), (g_rows, g_w, g_b, g_dense, g_head), want):
            off = (have.double() - ref).norm() / ref.norm().clamp(min=1e-30)
            assert off <= 2 * U * (dim + vocab + n + 200), (name, off.item())

        t.put_grad(k, g_rows, 0.05, 1e-8)
        assert t.sync() == mlkv.MLKV_OK
        rc, want_rows = o.get(keys)
        assert rc == O.OK
        assert np.abs(rows.cpu().numpy() - want_rows).max() <= 1e-5 * np.abs(want_rows).max()
        assert o.put_grad(keys, g_rows.cpu().numpy(), 0.05, 1e-8) == O.OK
        dense -= 0.02 * ops.orthogonalize(g_dense)
        w -= 0.05 * g_w
        b -= 0.05 * g_b
    have, state, _, _ = t.export()
    want_rows, want_state = o.read_rows(np.arange(o.size))
    assert t.size == o.size
    assert np.abs(have.cpu().numpy() - want_rows).max() <= 1e-5 * np.abs(want_rows).max()
    assert np.allclose(state.cpu().numpy(), want_state, rtol=1e-5, atol=0)
    t.close()


def test_a_step_recorded_once_and_replayed():
    """The dense part of a step in one HIP graph, replayed on new inputs beside
    eager steps, the table's calls between the replays."""
    from paper_2504_01506_amd import ops
    n, dim, vocab = 257, 64, 3001
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    t = mlkv.Table(dim, 4096)
    t.reserve(n)
    head = torch.randn((dim, vocab), generator=gen, device="cuda") / 8
    w, b = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
    rows = torch.empty((n, dim), device="cuda")
    targets = torch.empty(n, dtype=torch.int64, device="cuda")
    scale = torch.full((n,), -1.0 / n, device="cuda")

    def step():
        x = ops.layer_norm(rows, w, b)
        logits = x @ head
        r = ops.log_probs(logits, targets, top=2)
        g = ops.log_probs_grad(logits, targets, r.stats, r.entropy, scale)
        return (r.logp, r.top_ids, ops.orthogonalize(x.t() @ g), *ops.layer_norm_grad(rows, w, g @ head.t()))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):   # the library products' own set-up before the capture
        t.get(torch.arange(n, device="cuda"), rows)
        targets.fill_(5)
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(4):
        keys = torch.randint(0, 3000, (n,), generator=gen, device="cuda")
        t.get(keys, rows)
        targets.copy_(torch.randint(0, vocab, (n,), generator=gen, device="cuda"))
        graph.replay()
        eager = step()
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
        for p, q in zip(got[2:], eager[2:]):
            assert torch.allclose(p, q, rtol=1e-4, atol=1e-6 * q.abs().max().item())
        t.put_grad(keys, got[3], 0.05, 1e-8)
        assert t.sync() == mlkv.MLKV_OK
    t.close()
