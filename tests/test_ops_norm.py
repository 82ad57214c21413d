"""Layer norm and its gradient against the formulas in 64 bits.

Tolerances, with u = 2^-24 and h the normalised row: a row's sums take at most
~30 roundings (16 elements a lane, 6 joins in a wave, 16 waves), the mean is
corrected by the sum of what it left, and h is a product of three rounded
numbers: its error is below 64 u (1 + |h|). An output adds its own half step,
finfo(type).eps / 2 of its value."""
import pytest
import torch

from paper_2504_01506_amd import mlkv

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def half_step(t, kind):
    return t.abs() * (torch.finfo(kind).eps / 2) + torch.finfo(kind).smallest_normal * torch.finfo(kind).eps


def reference(x, w, b, eps):
    x = x.double()
    mu = x.mean(-1, keepdim=True)
    r = 1 / ((x - mu).square().mean(-1, keepdim=True) + eps).sqrt()
    h = (x - mu) * r
    return h, r, h * w + b


def check_forward(out, x, w, b, eps):
    w64 = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    b64 = torch.zeros(x.shape[-1], dtype=torch.float64, device=x.device) if b is None else b.double()
    h, _, want = reference(x, w64, b64, eps)
    tol = 64 * U * (w64.abs() * (1 + h.abs()) + b64.abs()) + half_step(want, x.dtype)
    assert out.dtype == x.dtype and out.shape == x.shape
    bad = (out.double() - want).abs() > tol * (1 + 1e-3)
    assert not bad.any(), (bad.sum().item(), (out.double() - want).abs().max().item())


def check_grad(got, x, w, dy, eps):
    dx, dw, db = got
    kind = x.dtype if w is None else w.dtype
    w64 = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    h, r, _ = reference(x, w64, 0.0, eps)
    g = dy.double() * w64

    def mean(t):
        return t.mean(-1, keepdim=True)

    want = r * (g - mean(g) - h * mean(g * h))
    size = g.abs() + mean(g.abs()) + (1 + h.abs()) * (mean((g * h).abs()) + mean(g.abs()))
    tol = 128 * U * r * size + half_step(want, x.dtype)
    assert ((dx.double() - want).abs() <= tol * (1 + 1e-3)).all(), (dx.double() - want).abs().max().item()
    # a thread's sum over its rows is as long as the call has rows a thread: at most 128 here
    flat = dy.double().reshape(-1, x.shape[-1])
    hf = h.reshape(-1, x.shape[-1])
    for t, term, bulk in ((dw, flat * hf, flat.abs() * (1 + hf.abs())), (db, flat, flat.abs())):
        want = term.sum(0)
        tol = (64 + 128) * U * bulk.sum(0) + half_step(want, kind)
        assert t.dtype == kind
        assert ((t.double() - want).abs() <= tol * (1 + 1e-3)).all(), (t.double() - want).abs().max().item()


def rows(gen, n, dim, kind, pad=0, mean=0.3, scale=1.0):
    buf = torch.full((n, dim + pad), 77.0, dtype=kind, device="cuda")
    buf[:, :dim] = (torch.randn((n, dim), generator=gen, device="cuda") * scale +
                    mean * torch.randn((n, 1), generator=gen, device="cuda")).to(kind)
    return buf[:, :dim]


@pytest.fixture
def gen():
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    return g


DIMS = [1, 2, 3, 4, 5, 8, 10, 16, 17, 63, 64, 65, 127, 128, 250, 400, 512, 513, 1000, 1021, 1024, 1025, 1026, 1028,
        2047, 2048, 4096, 5000, 8192, 8193, 12288, 16383, 16384]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_widths(gen, dim, kind):
    from paper_2504_01506_amd import ops
    for n, pad in ((1, 0), (3, 1), (65, 8)):
        x, dy = rows(gen, n, dim, kind, pad), rows(gen, n, dim, kind, 0, 0.1)
        w = (1 + 0.3 * torch.randn(dim, generator=gen, device="cuda")).to(kind)
        b = torch.randn(dim, generator=gen, device="cuda").to(kind)
        check_forward(ops.layer_norm(x, w, b, 1e-5), x, w, b, 1e-5)
        check_grad(ops.layer_norm_grad(x, w, dy, 1e-5), x, w, dy, 1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,dim", [(20_000, 16), (70_001, 10), (5000, 1024), (3001, 2000), (1300, 4096)])
def test_many_rows(gen, n, dim, kind):
    from paper_2504_01506_amd import ops
    x, dy = rows(gen, n, dim, kind), rows(gen, n, dim, kind, 0, 0.1)
    w, b = torch.randn((2, dim), generator=gen, device="cuda")
    check_forward(ops.layer_norm(x, w, b, 1e-5), x, w, b, 1e-5)
    check_grad(ops.layer_norm_grad(x, w, dy, 1e-5), x, w, dy, 1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
def test_params_of_either_type_or_none(gen, kind):
    from paper_2504_01506_amd import ops
    x, dy = rows(gen, 40, 200, kind), rows(gen, 40, 200, kind)
    for wk in {torch.float32, kind}:
        w = torch.randn(200, generator=gen, device="cuda").to(wk)
        check_forward(ops.layer_norm(x, w, None, 1e-5), x, w, None, 1e-5)
        check_forward(ops.layer_norm(x, None, w, 1e-5), x, None, w, 1e-5)
        check_grad(ops.layer_norm_grad(x, w, dy, 1e-5), x, w, dy, 1e-5)
    check_forward(ops.layer_norm(x), x, None, None, 1e-5)
    check_grad(ops.layer_norm_grad(x, None, dy), x, None, dy, 1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("mean,scale", [(1e4, 1.0), (0.0, 1e-3), (-3e3, 1e-2), (0.0, 1e4)])
def test_far_means_and_scales(gen, mean, scale):
    # the rows' own rounding about a far mean is an input: the reference sees the same numbers
    from paper_2504_01506_amd import ops
    for dim in (64, 1000, 4096):
        x, dy = rows(gen, 33, dim, torch.float32, 0, mean, scale), rows(gen, 33, dim, torch.float32)
        w = torch.randn(dim, generator=gen, device="cuda")
        check_forward(ops.layer_norm(x, w, None, 1e-5), x, w, None, 1e-5)
        check_grad(ops.layer_norm_grad(x, w, dy, 1e-5), x, w, dy, 1e-5)


@pytest.mark.gpu
def test_leading_dims_strides_offsets_and_broadcast_rows(gen):
    from paper_2504_01506_amd import ops
    w = torch.randn(130, generator=gen, device="cuda")
    for kind in TYPES:
        wide = torch.randn((4, 5, 6, 140), generator=gen, device="cuda").to(kind)
        for x in (wide[..., 3:133], wide[:, :, 1, :130], wide[2, 3, :, 8:138]):
            check_forward(ops.layer_norm(x, w, None), x, w, None, 1e-5)
        one = wide[0, 0, 0, :130]
        check_forward(ops.layer_norm(one, w, None), one, w, None, 1e-5)
        same = one.expand(70, 130)     # every row the same: stride 0
        dy = rows(gen, 70, 130, kind)
        check_forward(ops.layer_norm(same, w, None), same, w, None, 1e-5)
        check_grad(ops.layer_norm_grad(same, w, dy), same, w, dy, 1e-5)
        check_grad(ops.layer_norm_grad(dy, w, same), dy, w, same, 1e-5)
    with pytest.raises(ValueError, match="evenly"):
        ops.layer_norm(wide[:, :4, :, :130], w.to(kind))


@pytest.mark.gpu
def test_in_place_and_rows_behind_the_last(gen):
    from paper_2504_01506_amd import ops
    for dim in (64, 1000, 5000):
        x = rows(gen, 50, dim, torch.float32, 4)
        dy = rows(gen, 50, dim, torch.float32, 4)
        w = torch.randn(dim, generator=gen, device="cuda")
        want, gwant = ops.layer_norm(x, w), ops.layer_norm_grad(x, w, dy)
        buf = torch.full((60, dim + 4), -5.0, device="cuda")
        out = buf[:50, :dim]
        assert ops.layer_norm(x, w, out=out) is out
        assert torch.equal(out, want)
        assert (buf[50:] == -5).all() and (buf[:, dim:] == -5).all()
        for target in ("dy", "x"):
            x2, dy2 = rows(gen, 50, dim, torch.float32, 4), rows(gen, 50, dim, torch.float32, 4)
            x2.copy_(x), dy2.copy_(dy)
            got = ops.layer_norm_grad(x2, w, dy2, out=dy2 if target == "dy" else x2)
            assert all(torch.equal(p, q) for p, q in zip(got, gwant))
        x2 = rows(gen, 50, dim, torch.float32, 4)
        x2.copy_(x)
        assert torch.equal(ops.layer_norm(x2, w, out=x2), want)


@pytest.mark.gpu
def test_no_rows_equal_rows_and_values_out_of_range(gen):
    from paper_2504_01506_amd import ops
    w = torch.randn(96, generator=gen, device="cuda")
    none = torch.empty((0, 96), device="cuda")
    assert ops.layer_norm(none, w).shape == (0, 96)
    dx, dw, db = ops.layer_norm_grad(none, w, none)
    assert dx.shape == (0, 96) and (dw == 0).all() and (db == 0).all()
    x = torch.full((3, 96), 4.5, device="cuda")
    assert (ops.layer_norm(x, w) == 0).all()            # variance 0 under eps
    assert torch.isnan(ops.layer_norm(x, None, None, 0.0)).all()
    x = torch.randn((5, 96), generator=gen, device="cuda")
    x[1, 7], x[3, 0] = float("nan"), float("inf")
    out = ops.layer_norm(x, w)
    assert torch.isnan(out[[1, 3]]).all() and torch.isfinite(out[[0, 2, 4]]).all()
    check_forward(out[[0, 2, 4]], x[[0, 2, 4]], w, None, 1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("n,pad", [(64, 0), (192, 3), (561_728, 25)])
def test_rows_of_one_element(gen, n, pad):
    """Such rows are their mean: nothing passes to x or weight. The gradients of 64 rows cancel here but for their
    60 ones, as exactly as their sums (fp64 over a wave's rows) are whole numbers in fp32."""
    from paper_2504_01506_amd import ops
    x = rows(gen, n, 1, torch.float32, pad)
    w = torch.randn(1, generator=gen, device="cuda")
    dy = torch.ones(n // 64, 64, device="cuda")
    dy[:, 0], dy[:, 63], dy[:, 5], dy[:, 60] = 2.0 ** 25, -2.0 ** 25, -2.0 ** 40, 2.0 ** 40
    dx, dw, db = ops.layer_norm_grad(x, w, dy.view(n, 1))
    assert (dx == 0).all() and dw.item() == 0 and db.item() == 60 * (n // 64)
    dy = 0.01 * torch.randn(n, 1, generator=gen, device="cuda")
    dx, dw, db = ops.layer_norm_grad(x, w, dy)
    assert (dx == 0).all() and dw.item() == 0
    # five roundings on the way, each of at most the sum of the parts' sizes
    assert abs(db.item() - dy.double().sum().item()) <= 5 * 2.0 ** -24 * dy.double().abs().sum().item()


@pytest.mark.gpu
def test_gradient_against_differences(gen):
    from paper_2504_01506_amd import ops
    for dim in (7, 64, 1500):
        x, dy = rows(gen, 6, dim, torch.float32), rows(gen, 6, dim, torch.float32)
        w, b = torch.randn((2, dim), generator=gen, device="cuda")
        got = ops.layer_norm_grad(x, w, dy)

        def value(x, w, b):
            return (reference(x, w, b, 1e-5)[2] * dy.double()).sum()

        at = [x.double(), w.double(), b.double()]
        for k in range(3):
            way = torch.randn(at[k].shape, generator=gen, device="cuda").double()
            step = 1e-5
            up, down = [list(at), list(at)]
            up[k], down[k] = at[k] + step * way, at[k] - step * way
            want = (value(*up) - value(*down)) / (2 * step)
            have = (got[k].double() * way).sum()
            # second-order error of the difference 1e-10, rounding 1e-16 / step, both times the sums' size
            assert (have - want).abs() <= 1e-5 * (got[k].double().abs() * way.abs()).sum()


@pytest.mark.gpu
def test_offsets_past_32_bits(gen):
    from paper_2504_01506_amd import ops
    few, dy = rows(gen, 512, 4097, torch.float16), rows(gen, 512, 4097, torch.float16)
    w = torch.randn(4097, generator=gen, device="cuda")
    x, g = few.repeat(2100, 1), dy.repeat(2100, 1)      # 4.4e9 elements
    want, want_g = ops.layer_norm(few, w), ops.layer_norm_grad(few, w, dy)[0]
    check_forward(want, few, w, None, 1e-5)
    out = ops.layer_norm(x, w)
    assert torch.equal(out[-512:], want) and torch.equal(out[1050 * 512:1051 * 512], want)
    got = ops.layer_norm_grad(x, w, g, out=out)[0]
    assert torch.equal(got[-512:], want_g) and torch.equal(got[1050 * 512:1051 * 512], want_g)


@pytest.mark.gpu
def test_streams_and_graph_replays(gen):
    from paper_2504_01506_amd import ops
    x, dy = rows(gen, 3000, 256, torch.bfloat16), rows(gen, 3000, 256, torch.bfloat16)
    x2, dy2 = rows(gen, 900, 3000, torch.bfloat16), rows(gen, 900, 3000, torch.bfloat16)
    w, w2 = torch.randn(256, generator=gen, device="cuda"), torch.randn(3000, generator=gen, device="cuda")
    want, want2 = ops.layer_norm_grad(x, w, dy), ops.layer_norm_grad(x2, w2, dy2)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):      # two calls at once, one by its raw handle
        got, got2 = ops.layer_norm_grad(x, w, dy, stream=a), ops.layer_norm_grad(x2, w2, dy2, stream=b.cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got + got2, want + want2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ops.layer_norm(x, w)
        got = ops.layer_norm_grad(x, w, dy)
    for k in range(3):
        x.add_(0.25 * k)
        graph.replay()
        eager = ops.layer_norm_grad(x, w, dy)
        assert torch.equal(y, ops.layer_norm(x, w))
        assert all(torch.equal(p, q) for p, q in zip(got, eager))
        torch.cuda.synchronize()


@pytest.mark.gpu
def test_the_default_stream_by_its_handle(gen):
    from paper_2504_01506_amd import ops
    x = rows(gen, 50, 64, torch.float32)
    want = ops.layer_norm(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        default = torch.cuda.default_stream()
        got = [ops.layer_norm(x, stream=s) for s in (0, default, default.cuda_stream)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


# ---- refusals (no GPU needed: nothing is launched) ----
def call(**change):
    a = dict(x=4096, xs=64, w=8192, b=8192, n=3, dim=64, eps=1e-5, dtype=mlkv.MLKV_F32, wdtype=mlkv.MLKV_F32,
             out=16384, os=64)
    a.update(change)
    return mlkv.mlkv_layer_norm(a["x"], a["xs"], a["w"], a["b"], a["n"], a["dim"], a["eps"], a["dtype"], a["wdtype"],
                                a["out"], a["os"], 0)


@pytest.mark.parametrize("change,says", [
    (dict(n=-1), "n must"), (dict(n=2 ** 31), "n must"), (dict(dim=0), "dim"), (dict(dim=16385), "dim"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(wdtype=mlkv.MLKV_BF16), "weight_dtype"),
    (dict(x=None), "x is NULL"), (dict(out=None), "out is NULL"), (dict(xs=63), "x_stride"), (dict(xs=-64), "x_stride"),
    (dict(os=0), "out_stride"), (dict(os=2 ** 62), "out_stride"), (dict(x=4098), "aligned"), (dict(w=8194), "aligned"),
    (dict(out=4096, os=128), "same stride")])
def test_refusals(change, says):
    assert call(**change) == mlkv.MLKV_EINVAL
    assert says in mlkv.last_error()


def grad_call(**change):
    a = dict(x=4096, xs=64, w=8192, g=32768, gs=64, n=3, dim=64, eps=1e-5, dtype=mlkv.MLKV_F32, wdtype=mlkv.MLKV_F32,
             dx=16384, dxs=64, dw=65536, db=131072, work=262144, bytes=mlkv.mlkv_layer_norm_grad_workspace(3, 64))
    a.update(change)
    return mlkv.mlkv_layer_norm_grad(a["x"], a["xs"], a["w"], a["g"], a["gs"], a["n"], a["dim"], a["eps"], a["dtype"],
                                     a["wdtype"], a["dx"], a["dxs"], a["dw"], a["db"], a["work"], a["bytes"], 0)


@pytest.mark.parametrize("change,says", [
    (dict(g=None), "grad is NULL"), (dict(gs=1), "grad_stride"), (dict(dxs=1), "x_grad_stride"),
    (dict(work=None), "work"), (dict(bytes=511), "work"), (dict(work=262152), "work"),
    (dict(dx=32768, dxs=65), "same stride"), (dict(dx=4096, dxs=65), "same stride"), (dict(dw=65538), "aligned"),
    (dict(dim=0), "dim"), (dict(n=-5), "n must"), (dict(dtype=7), "dtype")])
def test_gradient_refusals(change, says):
    assert grad_call(**change) == mlkv.MLKV_EINVAL
    assert says in mlkv.last_error()


def test_workspace_sizes():
    size = mlkv.mlkv_layer_norm_grad_workspace
    assert size(0, 64) == 0 and 64 * 8 <= size(3, 64) <= 3 * 64 * 8
    assert size(2 ** 31 - 1, 16384) <= 2 ** 28
    assert size(-1, 64) == mlkv.MLKV_EINVAL and size(1, 0) == mlkv.MLKV_EINVAL and size(1, 16385) == mlkv.MLKV_EINVAL


def test_tensors_are_checked():
    from paper_2504_01506_amd import ops
    x = torch.zeros((2, 8))
    with pytest.raises(ValueError, match="GPU"):
        ops.layer_norm(x)
    with pytest.raises(ValueError, match="GPU"):
        ops.layer_norm_grad(x, None, x)


@pytest.mark.gpu
def test_tensors_are_checked_on_the_gpu():
    from paper_2504_01506_amd import ops
    x = torch.zeros((4, 8), device="cuda")
    for bad in (lambda: ops.layer_norm(x.double()), lambda: ops.layer_norm(x.t()), lambda: ops.layer_norm(x[:, :0]),
                lambda: ops.layer_norm(x, torch.ones(8)), lambda: ops.layer_norm(x, torch.ones(7, device="cuda")),
                lambda: ops.layer_norm(x, torch.ones(8, device="cuda").half()),
                lambda: ops.layer_norm(x, torch.ones(16, device="cuda")[::2]),
                lambda: ops.layer_norm(x, out=x[:3]), lambda: ops.layer_norm(x, out=x.bfloat16()),
                lambda: ops.layer_norm(x.bfloat16(), torch.ones(8, device="cuda"),
                                       torch.ones(8, device="cuda").bfloat16()),
                lambda: ops.layer_norm_grad(x, None, x.bfloat16()), lambda: ops.layer_norm_grad(x, None, x[:3])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(mlkv.MlkvError, match="eps"):
        ops.layer_norm(x, eps=-1.0)
    with pytest.raises(mlkv.MlkvError, match="x_stride|out_stride"):
        ops.layer_norm(x, out=torch.zeros(8, device="cuda").expand(4, 8))
