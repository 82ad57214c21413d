"""Calls of the dense operators that their documentation allows or forbids, by
how buffers lie: stacks of matrices whose rows come in turn."""
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
