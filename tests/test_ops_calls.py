"""Calls of the dense operators that their documentation allows or forbids, by
how buffers lie: stacks of matrices whose rows come in turn, and outputs that
overlap inputs."""
import random

import pytest
import torch

from paper_2504_01506_amd import mlkv


@pytest.fixture
def gen():
    g = torch.Generator(device="cuda")
    g.manual_seed(23)
    return g


# ---- stacks of matrices whose rows come in turn ----
def orth(**change):
    """A stack of 4 matrices of 66 x 100 without a workspace: refused for that, and for what is wrong before it."""
    a = dict(g=4096, gb=6600, gr=100, out=2 ** 20, ob=6600, orow=100, batch=4, rows=66, cols=100)
    a.update(change)
    assert mlkv.mlkv_orthogonalize(a["g"], a["gb"], a["gr"], a["batch"], a["rows"], a["cols"], 5, 1e-7, mlkv.MLKV_F32,
                                   a["out"], a["ob"], a["orow"], None, 0, 0) == mlkv.MLKV_EINVAL
    return mlkv.last_error()


@pytest.mark.parametrize("ob,orow,says", [
    (6600, 100, "work"), (100, 400, "work"), (103, 409, "work"), (103, 408, "overlap"), (99, 400, "overlap"),
    (100, 399, "overlap"), (100, 100, "overlap"), (0, 400, "overlap"), (-100, 400, "overlap"), (1 << 61, 100, "overlap")])
def test_strides_of_stacks(ob, orow, says):
    assert says in orth(ob=ob, orow=orow)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,heads,dim", [(250, 4, 64), (130, 6, 70), (40, 3, 90), (1, 5, 9), (300, 2, 1)])
def test_heads_side_by_side(gen, rows, heads, dim, kind):
    from paper_2504_01506_amd import ops
    buf = torch.full((rows, heads * dim + 3), 7.0, dtype=kind, device="cuda")
    w = buf[:, :heads * dim]
    w.copy_(torch.randn((rows, heads * dim), generator=gen, device="cuda"))
    by_head = w.unflatten(1, (heads, dim)).transpose(0, 1)       # [heads, rows, dim]
    want = ops.orthogonalize(by_head.contiguous())
    assert torch.equal(ops.orthogonalize(by_head), want)
    assert ops.orthogonalize(by_head, out=by_head) is by_head
    assert torch.equal(by_head, want) and (buf[:, heads * dim:] == 7).all()


# ---- outputs that overlap inputs ----
def rows_call(x, xs, out, os, n=3, dim=64, g=1 << 30, w=1 << 31):
    """A layer norm gradient without a workspace (fp32), strides and addresses in elements of 4 bytes."""
    assert mlkv.mlkv_layer_norm_grad(4 * x, xs, 4 * w, 4 * g, dim, n, dim, 1e-5, mlkv.MLKV_F32, mlkv.MLKV_F32, 4 * out,
                                     os, 1 << 34, 1 << 35, None, 0, 0) == mlkv.MLKV_EINVAL
    return "overlaps" in mlkv.last_error()


def meets(x, xs, out, os, n, dim):
    taken = {x + i * xs + c for i in range(n) for c in range(dim)}
    return any(out + i * os + c in taken for i in range(n) for c in range(dim))


def test_rows_of_output_over_rows_of_input_are_refused():
    assert rows_call(1000, 64, 1001, 64) and rows_call(1001, 64, 1000, 64)
    assert not rows_call(1000, 64, 1000, 64) and not rows_call(1000, 64, 1192, 64)
    assert rows_call(1000, 64, 1191, 64) and not rows_call(1000, 64, 808, 64) and rows_call(1000, 64, 809, 64)
    assert not rows_call(1000, 128, 1064, 128) and rows_call(1000, 128, 1063, 128)   # side by side
    assert not rows_call(1000, 128, 1064, 256) and rows_call(1000, 128, 1000 + 128 * 2, 256)
    assert not rows_call(1000, 0, 1064, 64) and rows_call(1000, 0, 1063, 64)
    assert not rows_call(1000, 0, 1000 - 192, 64) and rows_call(1000, 0, 1000 - 191, 64)
    assert rows_call(5000, 64, 1000, 64, w=1000 + 191) and not rows_call(5000, 64, 1000, 64, w=1000 + 192)
    assert rows_call(5000, 64, 1000, 64, g=1191) and not rows_call(5000, 64, 1000, 64, g=1000)
    big = 2 ** 31 - 1                                                                # at once, however many rows
    assert not rows_call(1 << 40, 16384, (1 << 40) + 8192, 16384, big, 8192, g=1 << 50)
    assert rows_call(1 << 40, 16384, (1 << 40) + 8191, 16384, big, 8192, g=1 << 50)


def test_overlaps_against_every_element():
    for n in (1, 2, 5):
        for dim in (1, 3):
            for xs in (0, dim, dim + 1, 6, 7):
                for os in (dim, dim + 2, 7, 12):
                    for out in range(-40, 90):
                        if out == 0:       # equal pointers are in place, or refused for their strides
                            continue
                        want = meets(0, xs, out, os, n, dim)
                        assert rows_call(1000, xs, 1000 + out, os, n, dim) == want, (n, dim, xs, os, out)


def test_logits_grad_over_its_inputs_is_refused():
    a = dict(x=1 << 20, t=1 << 24, st=2 << 24, e=3 << 24, gl=4 << 24, ge=5 << 24)
    n, vocab, at = 3, 64, 6 << 24
    for name, size in (("x", 4 * vocab), ("t", 8), ("st", 8), ("e", 4), ("gl", 4), ("ge", 4)):
        for off in (-n * size + 8, 8, n * vocab * 4 - 8):
            b = {**a, name: at + off}
            assert mlkv.mlkv_log_probs_grad(b["x"], vocab, b["t"], b["st"], b["e"], b["gl"], b["ge"], n, vocab,
                                            mlkv.MLKV_F32, at, vocab, 0) == mlkv.MLKV_EINVAL
            assert "overlaps" in mlkv.last_error()


def test_norm_over_its_inputs_is_refused():
    a = dict(x=1 << 20, w=1 << 24, b=2 << 24)
    for name, off in (("x", 4), ("w", 0), ("w", 700), ("b", -200)):
        v = {**a, name: (3 << 24) + off}
        assert mlkv.mlkv_layer_norm(v["x"], 64, v["w"], v["b"], 3, 64, 1e-5, mlkv.MLKV_F32, mlkv.MLKV_F32, 3 << 24, 64,
                                    0) == mlkv.MLKV_EINVAL
        assert "overlaps" in mlkv.last_error()


def places(at, batch, rows, cols, bs, rs):
    return {at + b * bs + r * rs + c for b in range(batch) for r in range(rows) for c in range(cols)}


def test_stacks_over_each_other_are_refused():
    assert "work" in orth(g=2 ** 20 + 4 * 6600, gb=13200, ob=13200)                  # every second matrix
    assert "overlaps" in orth(g=2 ** 20 + 4 * 6599, gb=13200, ob=13200)
    assert "work" in orth(g=2 ** 20 + 400, gr=200, gb=13200, orow=200, ob=13200)     # side by side
    rng = random.Random(1)
    w = 257                                          # (wide enough to need a workspace: each call ends there at the latest)
    for batch, rows in ((1, 2), (2, 1), (3, 2), (2, 3)):
        for gb, gr in ((0, w), (w * rows, w), (w, w * batch), (1300, 300), (300, 1300), (500, 0), (20, 290)):
            for ob, orow in ((w * rows, w), (w, w * batch), (1500, 270), (260, 1200)):
                out = places(0, batch, rows, w, ob, orow)
                if len(out) < batch * rows * w:
                    continue
                edges = [i * gr + j * gb + d * w + e for i in (-2, -1, 0, 1) for j in (-1, 0, 1) for d in (-1, 0, 1)
                         for e in (-1, 0, 1)]
                for g in rng.sample(edges, 20) + [rng.randrange(-4000, 4000) for _ in range(10)]:
                    if g != 0:
                        said = orth(g=2 ** 20 + 4 * g, gb=gb, gr=gr, ob=ob, orow=orow, batch=batch, rows=rows, cols=w)
                        want = bool(places(g, batch, rows, w, gb, gr) & out)
                        assert ("out overlaps g" in said) == want, (batch, rows, gb, gr, ob, orow, g)


@pytest.mark.gpu
def test_rows_side_by_side_in_one_buffer(gen):
    from paper_2504_01506_amd import ops
    buf = torch.randn((50, 3, 96), generator=gen, device="cuda")
    x, dy, out = buf[:, 0], buf[:, 1], buf[:, 2]
    keep = buf.clone()
    assert torch.equal(ops.layer_norm(x, out=out), ops.layer_norm(x.contiguous()))
    assert torch.equal(ops.layer_norm_grad(x, None, dy, out=out)[0],
                       ops.layer_norm_grad(x.contiguous(), None, dy.contiguous())[0])
    assert torch.equal(buf[:, :2], keep[:, :2])
    t = torch.zeros(50, dtype=torch.int64, device="cuda")
    r = ops.log_probs(x, t)
    one = torch.ones(50, device="cuda")
    assert torch.equal(ops.log_probs_grad(x, t, r.stats, None, one, out=out),
                       ops.log_probs_grad(x.contiguous(), t, r.stats, None, one))
    stack = torch.randn((6, 70, 80), generator=gen, device="cuda")
    want = ops.orthogonalize(stack[::2].contiguous())
    assert torch.equal(ops.orthogonalize(stack[::2], out=stack[1::2]), want)
    flat = buf.flatten()
    for bad in (lambda: ops.layer_norm(flat[:4800].view(50, 96), out=flat[1:4801].view(50, 96)),
                lambda: ops.orthogonalize(stack[:4], out=stack[2:])):
        with pytest.raises(mlkv.MlkvError, match="overlaps"):
            bad()


# ---- transposed views ----
@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(70, 200), (200, 70), (3, 40, 90), (50, 50), (1, 9), (9, 1), (2, 1, 30)])
def test_transposed_views_on_either_side(gen, shape):
    from paper_2504_01506_amd import ops
    lying = torch.randn(shape, generator=gen, device="cuda")
    standing = lying.mT.contiguous().mT
    side = torch.cuda.Stream()
    for g in (lying, standing):
        want = ops.orthogonalize(g)     # (a square's transpose takes other sums)
        for like in (lying, standing):
            for stream in (None, side):
                out = torch.empty_like(like)     # (keeps the strides)
                torch.cuda.synchronize()
                assert ops.orthogonalize(g, out=out, stream=stream) is out
                torch.cuda.synchronize()
                assert torch.equal(out, want)
    assert torch.equal(ops.orthogonalize(standing, out=standing), want)


@pytest.mark.gpu
def test_a_square_into_its_transpose(gen):
    from paper_2504_01506_amd import ops
    w = torch.randn((90, 90), generator=gen, device="cuda")
    want = ops.orthogonalize(w.t())
    assert torch.equal(ops.orthogonalize(w.t(), out=w), want) and torch.equal(w, want)


@pytest.mark.gpu
def test_outputs_that_lie_neither_way_are_refused(gen):
    from paper_2504_01506_amd import ops
    g = torch.randn((40, 60), generator=gen, device="cuda")
    hold = torch.zeros((40, 120), device="cuda")
    for bad in (g, g.t().contiguous().t()):
        with pytest.raises((ValueError, RuntimeError)):
            ops.orthogonalize(bad, out=hold[:, ::2])
        with pytest.raises((ValueError, RuntimeError)):
            ops.orthogonalize(bad, out=hold[:1, :60].expand(40, 60))
    assert (hold == 0).all()


# ---- views whose memory holds their negative ----
@pytest.mark.gpu
def test_views_that_stand_for_their_negative_are_refused(gen):
    from paper_2504_01506_amd import ops
    x, w = torch.randn((6, 8), generator=gen, device="cuda"), torch.randn(8, generator=gen, device="cuda")
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    r = ops.log_probs(x, t)
    neg = torch._neg_view
    for bad in (lambda: ops.layer_norm(neg(x)), lambda: ops.layer_norm(x, neg(w)), lambda: ops.layer_norm(x, w, neg(w)),
                lambda: ops.layer_norm(x, out=neg(x)), lambda: ops.layer_norm_grad(x, None, neg(x)),
                lambda: ops.layer_norm_grad(x, None, x, out=neg(x)), lambda: ops.log_probs(neg(x), t),
                lambda: ops.log_probs_grad(x, t, neg(r.stats), None, r.logp),
                lambda: ops.log_probs_grad(x, t, r.stats, None, neg(r.logp)),
                lambda: ops.log_probs_grad(x, t, r.stats, neg(r.entropy), r.logp, r.logp),
                lambda: ops.log_probs_grad(x, t, r.stats, None, r.logp, out=neg(x)),
                lambda: ops.orthogonalize(neg(x)), lambda: ops.orthogonalize(x, out=neg(x))):
        with pytest.raises(ValueError, match="resolved"):
            bad()
    # (rows of one element from the imaginary part of a conjugate)
    grad = torch.complex(x[:, :1], x[:, 1:2]).conj().imag
    with pytest.raises(ValueError, match="resolved"):
        ops.layer_norm_grad(x[:, :1], None, grad)


def test_a_view_that_stands_for_its_negative_is_no_argument():
    from paper_2504_01506_amd import ops
    x = torch.ones(4)
    with pytest.raises(ValueError, match="resolved"):
        ops._check(torch._neg_view(x), "weight", x)


def test_one_rows_stride_may_be_anything():
    """... and is not multiplied (2^62 elements of 4 bytes would wrap to an overlap of itself)."""
    far = 2 ** 62
    assert not rows_call(1000, far, 5000, far, 1) and not rows_call(1000, -far, 1000, far, 1)
    assert rows_call(1000, far, 1063, -far, 1) and not rows_call(1000, far, 1064, -far, 1)
    assert "work" in orth(batch=1, gb=far, ob=-far, rows=70) and "overlaps" in orth(batch=1, gb=far, ob=-far, out=4096 + 400)
    assert "work" in orth(rows=1, gr=far, orow=-far, cols=257, gb=257, ob=257)
