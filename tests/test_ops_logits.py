"""Log probabilities of tokens, entropies and top alternatives, and their
gradient, against the definitions in 64 bits.

Tolerances, u = 2^-24: an exponential carries 2 u and twice u |x - m| from its
argument, a sum of a row at most ~90 roundings (64 logits a thread, 6 + 2 joins,
chunks): the relative error of s is below 160 u, so log s is off by 160 u +
u |log s| and a log probability by that and the roundings of x - m and of the
difference. The entropy adds the same for sum e z / s, which is at most log s + H."""
import math

import pytest
import torch

from paper_2504_01506_amd import mlkv

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def close(got, want, tol):
    want = want.float().double()    # (differences of the types' extremes leave fp32's range)
    same = (got.double() == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got.double() - want).abs() <= tol))
    assert not bad.any(), (bad.sum().item(), got[bad][:4], want[bad][:4])


def order(x, k):
    """Indices of the k largest of each row, ties to the lowest index."""
    return torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :k]


def reference(x, tokens, k):
    x = x.double()
    m = x.max(-1).values
    none = m == -math.inf
    d = x - torch.where(none, 0.0, m)[..., None]
    e = d.exp()
    s = e.sum(-1)
    logs = torch.where(none, 0.0, s.log())
    ent = torch.where(none, 0.0, s.log() - (e * d.clamp(min=-1e300)).sum(-1) / s)
    lp = torch.where(none[..., None], -math.inf, d - logs[..., None])
    at = lp.gather(-1, tokens.clamp(0, x.shape[-1] - 1)[..., None])[..., 0]
    logp = torch.where(tokens < 0, 0.0, torch.where(tokens >= x.shape[-1], math.nan, at))
    ids = order(x, k)
    return logp, ent, m, logs, ids, lp.gather(-1, ids), d


def check(x, tokens, top):
    from paper_2504_01506_amd import ops
    r = ops.log_probs(x, tokens, top=top)
    logp, ent, m, logs, ids, tops, d = reference(x, tokens, top)
    tol = 160 * U + 2 * U * logs.abs()
    at = d.gather(-1, tokens.clamp(0, x.shape[-1] - 1)[..., None])[..., 0].abs()
    close(r.stats[..., 0], m, 0.0 * m)
    close(r.stats[..., 1], logs, tol)
    close(r.logp, logp, tol + 2 * U * at + 2 * U * logp.abs())
    close(r.entropy, ent, 2 * tol + 320 * U * (logs + ent))
    if top:
        assert r.top_ids.dtype == torch.int64 and torch.equal(r.top_ids, ids)
        far = d.gather(-1, ids).abs()
        close(r.top_logp, tops, (tol + 2 * U * tops.abs().amax(-1))[..., None] + 2 * U * far)
    else:
        assert r.top_ids is None and r.top_logp is None
    return r


@pytest.fixture
def gen():
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    return g


def logits(gen, n, vocab, kind, pad=0, scale=2.5):
    buf = torch.full((n, vocab + pad), 99.0, dtype=kind, device="cuda")
    buf[:, :vocab] = (torch.randn((n, vocab), generator=gen, device="cuda") * scale).to(kind)
    return buf[:, :vocab]


def some_tokens(gen, n, vocab):
    t = torch.randint(vocab, (n,), generator=gen, device="cuda")
    if n > 2:
        t[1] = -1
        t[n // 2] = vocab - 1
    return t


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 8, 9, 31, 64, 65, 200, 1000, 2047, 2048, 2049, 2056, 4097, 8192, 9000,
                                   16384, 16391, 16400, 16433, 32768, 50_003, 128_000])
def test_vocabularies(gen, vocab, kind):
    for n, pad, top in ((1, 0, 20), (5, 1, 1), (37, 3, 64), (4, 8, 5), (6, 0, 0)):
        check(logits(gen, n, vocab, kind, pad), some_tokens(gen, n, vocab), min(top, vocab))


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [40, 900, 6000, 40_000])
@pytest.mark.parametrize("far", [300.0, -3e4, 6e4, 1e8, -1e30, 3e37, 2e38])
def test_far_logits(gen, vocab, far):
    # a row's own offset is no part of its distribution, as far as its digits go
    for kind in (torch.float32, torch.bfloat16):
        x = logits(gen, 5, vocab, torch.float32)
        x = (far + x * max(1.0, abs(far) * 2.0 ** -20)).to(kind)
        check(x, some_tokens(gen, 5, vocab), 9)


@pytest.mark.gpu
@pytest.mark.parametrize("n,vocab,top", [(2000, 300, 3), (700, 33_000, 10), (129, 20_000, 64), (3, 600_000, 50), (1100, 20_000, 10), (1025, 5001, 64),
                                         (1, 2_000_001, 64), (40, 262_144, 33)])
def test_many_rows_and_long_rows(gen, n, vocab, top):
    for kind in (torch.float32, torch.bfloat16):
        check(logits(gen, n, vocab, kind), some_tokens(gen, n, vocab), top)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [100, 5000, 40_000])
def test_ties(gen, vocab, kind):
    t = some_tokens(gen, 6, vocab)
    x = torch.zeros((6, vocab), dtype=kind, device="cuda")
    x[1] = 3.0
    x[2] = torch.randint(3, (vocab,), generator=gen, device="cuda").to(kind)
    x[3, ::2] = -0.0                                        # zeros of both signs are equal
    x[4] = torch.arange(vocab, device="cuda").to(kind) * 1e-3   # rising: the largest last
    x[5] = -x[4]
    y = x.clone()
    y[:, vocab // 2:vocab // 2 + 5] = 4.0
    check(y, t, min(64, vocab))
    for top in (1, 17, 64):
        check(x, t, top)
        check(x[:, 1:], t.clamp(max=vocab - 2), top)        # rows off their 16-byte boundaries


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [3000, 40_000])
def test_ties_and_masks_in_many_rows(gen, vocab, kind):
    # rows enough for each to be a block's
    x = torch.zeros((8, vocab), dtype=kind, device="cuda")
    x[1] = torch.randint(3, (vocab,), generator=gen, device="cuda").to(kind)
    x[2] = torch.arange(vocab, device="cuda").to(kind) * 1e-3
    x[3], x[3, 77:90] = -math.inf, 1.0
    x[4] = -math.inf
    x[5], x[5, ::50] = torch.finfo(kind).min, 2.0
    x[6:] = logits(gen, 2, vocab, kind)
    x, t = x.repeat(160, 1), some_tokens(gen, 1280, vocab)
    for top in (1, 20, 64):
        check(x, t, top)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [90, 3000, 70_000])
def test_masks(gen, vocab, kind):
    n = 9
    x, t = logits(gen, n, vocab, kind), some_tokens(gen, n, vocab)
    low = torch.finfo(kind).min
    x[0, 5:] = -math.inf
    x[1, :] = -math.inf                     # nothing left
    x[2, :-1] = -math.inf                   # one left, the last
    x[3, 4:] = low                          # masked by the type's lowest value
    x[4, :] = low                           # nothing but that: a uniform row
    x[5, ::2], x[5, 1::2] = -math.inf, low
    x[6, 0], x[6, 1:] = torch.finfo(kind).max, low
    x[7, :] = torch.finfo(kind).max
    x[8, vocab // 3] = -math.inf
    t[1], t[0] = 3, vocab - 1
    for top in (0, 2, 40):
        r = check(x, t, top)
        assert r.logp[1] == -math.inf and r.entropy[1] == 0 and r.logp[0] == -math.inf


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [50, 3000, 70_000])
def test_nan_and_infinity_stay_in_their_rows(gen, vocab, kind):
    from paper_2504_01506_amd import ops
    x = logits(gen, 8, vocab, kind)
    t = torch.full((8,), 4, device="cuda")
    x[1, vocab - 1] = math.nan
    x[2, 0] = math.inf
    x[3, :] = math.nan
    x[4, :], x[4, 9] = -math.inf, math.nan
    x[5, 7:] = math.inf
    t[3] = -1
    r = ops.log_probs(x, t, top=12)
    bad = [1, 2, 3, 4, 5]
    for f in (r.entropy, r.stats, r.top_logp):
        assert torch.isnan(f[bad]).all()
    assert torch.isnan(r.logp[[1, 2, 4, 5]]).all() and r.logp[3] == 0
    assert (r.top_ids[bad] == -1).all()
    good = [0, 6, 7]
    check(x[good], t[good], 12)
    g = ops.log_probs_grad(x, t, r.stats, r.entropy, torch.ones(8, device="cuda"))
    assert torch.isnan(g[[1, 2, 4, 5]].float()).all() and torch.isfinite(g[good].float()).all()


@pytest.mark.gpu
def test_tokens_outside_the_vocabulary(gen):
    from paper_2504_01506_amd import ops
    x = logits(gen, 6, 700, torch.float32)
    t = torch.tensor([-1, -100, 700, 2 ** 40, -2 ** 62, 5], device="cuda")
    r = check(x, t, 4)
    assert (r.logp[[0, 1, 4]] == 0).all() and torch.isnan(r.logp[[2, 3]]).all()
    g = ops.log_probs_grad(x, t, r.stats, r.entropy, torch.ones(6, device="cuda"))
    assert (g[[0, 1, 4]] == 0).all() and torch.isnan(g[[2, 3]]).all() and torch.isfinite(g[5]).all()


@pytest.mark.gpu
def test_shapes_strides_and_rows_that_repeat(gen):
    from paper_2504_01506_amd import ops
    wide = torch.randn((3, 4, 5100), generator=gen, device="cuda").bfloat16()
    x, t = wide[..., 7:5007], torch.randint(5000, (3, 4), generator=gen, device="cuda")
    r = check(x, t, 6)
    assert r.logp.shape == (3, 4) and r.stats.shape == (3, 4, 2) and r.top_ids.shape == (3, 4, 6)
    one = wide[0, 0, :5000]
    check(one, torch.tensor(17, device="cuda"), 3)
    check(one.expand(9, 5000), some_tokens(gen, 9, 5000), 3)
    none = ops.log_probs(wide[:0, 0], torch.empty(0, dtype=torch.int64, device="cuda"), top=2)
    assert none.logp.shape == (0,) and none.top_ids.shape == (0, 2)
    assert ops.log_probs_grad(wide[:0, 0], None, none.stats, None, None).shape == (0, 5100)


def check_grad(x, t, a, b, out=None):
    from paper_2504_01506_amd import ops
    r = ops.log_probs(x, t)
    keep = x.clone()
    got = ops.log_probs_grad(x, t if a is not None else None, r.stats, r.entropy if b is not None else None, a, b,
                             out=out)
    x64, m, logs = keep.double(), r.stats[..., :1].double(), r.stats[..., 1:].double()
    none = m == -math.inf
    d = torch.where(none, -math.inf, x64 - m)
    lp = d - logs
    p = torch.exp(lp)
    zero = torch.zeros(x.shape[:-1], dtype=torch.float64, device=x.device)
    a64 = (zero if a is None else torch.where(t < 0, 0.0, a.double()))[..., None]
    b64 = (zero if b is None else b.double())[..., None]
    ent = r.entropy.double()[..., None]
    hot = torch.zeros_like(x64)
    hot.scatter_(-1, t.clamp(min=0)[..., None], 1.0)
    lpc = lp.clamp(min=-1e4)
    want = torch.where(none, 0.0, a64 * (hot - p) - b64 * p * (lpc + ent))
    lost = p * (a64.abs() + b64.abs() * ((lpc + ent).abs() + 1))
    tol = U * (8 + 4 * (d.clamp(min=-1e4).abs() + lpc.abs())) * lost + 4 * U * (a64 * hot).abs()
    kind = x.dtype
    tol = tol + want.abs() * (torch.finfo(kind).eps / 2) + torch.finfo(kind).smallest_normal * torch.finfo(kind).eps
    tol = tol + 2.0 ** -126 * (a64.abs() + b64.abs())       # probabilities below fp32's normal numbers
    close(got, want, tol * (1 + 1e-3))
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,vocab,pad", [(1, 1, 0), (3, 2, 0), (5, 7, 1), (4, 8, 0), (9, 1000, 3), (6, 4096, 0),
                                         (3, 8200, 5), (2, 50_003, 0), (300, 77, 0), (2, 128_000, 8)])
def test_gradient(gen, n, vocab, pad, kind):
    x, t = logits(gen, n, vocab, kind, pad), some_tokens(gen, n, vocab)
    a, b = torch.randn((2, n), generator=gen, device="cuda")
    check_grad(x, t, a, None)
    check_grad(x, t, a, b)
    check_grad(x, t, None, b)
    buf = torch.full((n + 2, vocab + 3), 4.0, dtype=kind, device="cuda")   # rows at other offsets than the logits'
    check_grad(x, t, a, b, out=buf[:n, 1:vocab + 1])
    assert (buf[n:] == 4).all() and (buf[:, 0] == 4).all() and (buf[:, vocab + 1:] == 4).all()
    check_grad(x, t, a, b, out=x)     # in place


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
def test_gradient_under_masks(gen, kind):
    x, t = logits(gen, 6, 3000, kind), some_tokens(gen, 6, 3000)
    low = torch.finfo(kind).min
    x[0, 5:], x[1], x[2, :-1], x[3, 4:], x[4] = -math.inf, -math.inf, -math.inf, low, low
    t[0], t[1] = 2999, 3        # a token that the mask rules out
    a, b = torch.randn((2, 6), generator=gen, device="cuda")
    assert (check_grad(x, t, a, None)[1] == 0).all()
    assert (check_grad(x, t, a, b)[1] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [300, 9000])
def test_padded_positions_get_zeros(gen, vocab, kind):
    """A position without a token passes no gradient, also where its logits are no numbers."""
    from paper_2504_01506_amd import ops
    x = logits(gen, 6, vocab, kind)
    t = some_tokens(gen, 6, vocab)
    t[:4] = -1
    t[4:] = 7
    x[0], x[1, 3], x[2, vocab - 1] = math.nan, math.inf, math.nan
    r = ops.log_probs(x, t)
    a = torch.ones(6, device="cuda")
    b = torch.zeros(6, device="cuda")
    a[:3] = math.nan  # (no use is made of it there)
    for more in ((), (b,)):
        g = ops.log_probs_grad(x, t, r.stats, r.entropy, a, *more)
        assert (g[:4] == 0).all() and (g[4:] != 0).any(-1).all()
    check_grad(x[3:].contiguous(), t[3:].contiguous(), a[3:].contiguous(), b[3:].contiguous())
    b[2] = b[3] = 1.0
    g = ops.log_probs_grad(x, t, r.stats, r.entropy, a, b)
    assert (g[:2] == 0).all() and torch.isnan(g[2]).all() and (g[3] != 0).any()


@pytest.mark.gpu
def test_gradient_against_differences(gen):
    from paper_2504_01506_amd import ops
    x, t = logits(gen, 5, 300, torch.float32), some_tokens(gen, 5, 300)
    a, b = torch.randn((2, 5), generator=gen, device="cuda")
    r = ops.log_probs(x, t)
    got = ops.log_probs_grad(x, t, r.stats, r.entropy, a, b).double()

    def value(x):
        logp, ent = reference(x, t, 0)[:2]
        return (a.double() * logp + b.double() * ent).sum()

    way, step = torch.randn(x.shape, generator=gen, device="cuda").double(), 1e-5
    want = (value(x.double() + step * way) - value(x.double() - step * way)) / (2 * step)
    assert ((got * way).sum() - want).abs() <= 1e-5 * (got.abs() * way.abs()).sum()


@pytest.mark.gpu
def test_offsets_past_32_bits(gen):
    from paper_2504_01506_amd import ops
    n, vocab = 40_000, 120_001          # 4.8e9 logits
    few = logits(gen, 100, vocab, torch.bfloat16)
    x = few.repeat(n // 100, 1)
    t = some_tokens(gen, 100, vocab).repeat(n // 100)
    r = ops.log_probs(x, t, top=4)
    check(x[-3:], t[-3:], 4)
    want = reference(few, t[:100], 4)
    assert torch.equal(r.top_ids, want[4].repeat(n // 100, 1))
    assert (r.logp.double() - want[0].repeat(n // 100)).abs().max() <= 1e-4
    one = torch.ones(n, device="cuda")
    first = ops.log_probs_grad(x[:100], t[:100], r.stats[:100], None, one[:100])
    ops.log_probs_grad(x, t, r.stats, None, one, out=x)
    for at in (n - 200, n // 200 * 100):
        # rows at one place modulo 16 bytes are cut alike: 100 rows are 24,000,200 bytes, 8 modulo 16, 200 of them 0
        assert torch.equal(x[at:at + 100], first)


@pytest.mark.gpu
def test_streams_and_graph_replays(gen):
    from paper_2504_01506_amd import ops
    x, x2 = logits(gen, 3, 60_000, torch.bfloat16), logits(gen, 500, 40_000, torch.bfloat16)
    t, t2 = some_tokens(gen, 3, 60_000), some_tokens(gen, 500, 40_000)
    want, want2 = ops.log_probs(x, t, 9), ops.log_probs(x2, t2, 9)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        got, got2 = ops.log_probs(x, t, 9, stream=a), ops.log_probs(x2, t2, 9, stream=b.cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got + got2, want + want2))
    one = torch.ones(500, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ops.log_probs(x, t, 9)
        got2 = ops.log_probs(x2, t2, 9)
        g2 = ops.log_probs_grad(x2, t2, got2.stats, got2.entropy, one, one)
    for k in range(3):
        x.mul_(1 - 0.1 * k), x2.mul_(1 + 0.1 * k)
        graph.replay()
        e, e2 = ops.log_probs(x, t, 9), ops.log_probs(x2, t2, 9)
        assert all(torch.equal(p, q) for p, q in zip(got + got2, e + e2))
        assert torch.equal(g2, ops.log_probs_grad(x2, t2, e2.stats, e2.entropy, one, one))
        torch.cuda.synchronize()


# ---- refusals (no GPU needed: nothing is launched) ----
def call(**change):
    a = dict(x=4096, s=64, t=8192, n=3, v=64, top=4, dtype=mlkv.MLKV_F32, logp=16384, ent=32768, st=65536,
             ids=131072, tl=262144, work=None, bytes=0)
    a.update(change)
    return mlkv.mlkv_log_probs(a["x"], a["s"], a["t"], a["n"], a["v"], a["top"], a["dtype"], a["logp"], a["ent"],
                               a["st"], a["ids"], a["tl"], a["work"], a["bytes"], 0)


@pytest.mark.parametrize("change,says", [
    (dict(n=-1), "n must"), (dict(n=2 ** 31), "n must"), (dict(v=0), "vocab"), (dict(v=2 ** 24 + 1), "vocab"),
    (dict(top=-1), "top must"), (dict(top=65), "top must"), (dict(v=3, s=3), "top must"), (dict(dtype=9), "dtype"),
    (dict(x=None), "logits is NULL"), (dict(t=None), "tokens is NULL"), (dict(s=63), "stride"), (dict(s=-1), "stride"),
    (dict(top=0), "must be NULL"), (dict(x=4097), "aligned"), (dict(t=8196), "aligned"), (dict(ids=131076), "aligned"),
    (dict(st=65537), "aligned"), (dict(v=100_000, s=100_000), "work"),
    (dict(v=100_000, s=100_000, work=2 ** 20, bytes=100), "work"),
    (dict(v=100_000, s=100_000, work=2 ** 20 + 8, bytes=2 ** 20), "work")])
def test_refusals(change, says):
    assert call(**change) == mlkv.MLKV_EINVAL
    assert says in mlkv.last_error()


def grad_call(**change):
    a = dict(x=4096, s=64, t=8192, st=16384, ent=32768, ga=65536, gb=131072, n=3, v=64, dtype=mlkv.MLKV_F32,
             out=262144, os=64)
    a.update(change)
    return mlkv.mlkv_log_probs_grad(a["x"], a["s"], a["t"], a["st"], a["ent"], a["ga"], a["gb"], a["n"], a["v"],
                                    a["dtype"], a["out"], a["os"], 0)


@pytest.mark.parametrize("change,says", [
    (dict(st=None), "stats"), (dict(out=None), "logits_grad"), (dict(t=None), "tokens"), (dict(ent=None), "entropy"),
    (dict(os=0), "grad_stride"), (dict(s=5), "stride"), (dict(out=262145), "aligned"), (dict(gb=131073), "aligned"),
    (dict(out=4096, os=65), "same stride"), (dict(v=0), "vocab"), (dict(n=-1), "n must"), (dict(dtype=-2), "dtype")])
def test_gradient_refusals(change, says):
    assert grad_call(**change) == mlkv.MLKV_EINVAL
    assert says in mlkv.last_error()


def test_workspace_sizes():
    size = mlkv.mlkv_log_probs_workspace
    assert size(5, 64, 4, mlkv.MLKV_F32) == 0 and size(0, 10 ** 6, 4, mlkv.MLKV_F32) == 0
    assert size(40, 128_000, 5, mlkv.MLKV_BF16) > 0
    for bad in ((-1, 64, 4, 0), (1, 0, 0, 0), (1, 64, 65, 0), (1, 64, 4, 5), (1, 2 ** 24 + 1, 1, 0)):
        assert size(*bad) == mlkv.MLKV_EINVAL


@pytest.mark.gpu
def test_tensors_are_checked():
    from paper_2504_01506_amd import ops
    x, t = torch.zeros((4, 8), device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    r = ops.log_probs(x, t)
    one = torch.ones(4, device="cuda")
    for bad in (lambda: ops.log_probs(x.cpu(), t), lambda: ops.log_probs(x, t.cpu()), lambda: ops.log_probs(x, t.int()),
                lambda: ops.log_probs(x, t[:3]), lambda: ops.log_probs(x.double(), t), lambda: ops.log_probs(x.t(), t),
                lambda: ops.log_probs_grad(x, None, r.stats, None, one),
                lambda: ops.log_probs_grad(x, t, r.stats, None, one, one),
                lambda: ops.log_probs_grad(x, t, r.stats[:, :1], None, one),
                lambda: ops.log_probs_grad(x, t, r.stats, None, one.double()),
                lambda: ops.log_probs_grad(x, t, r.stats, None, one, out=x.half())):
        with pytest.raises(ValueError):
            bad()
    for top in (-1, 9, 65):
        with pytest.raises(mlkv.MlkvError, match="top"):
            ops.log_probs(x, t, top=top)
