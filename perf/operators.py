"""The dense operators of a training step around a table, as cases to time.

A case is a dict of plain values. `op` names the operator:

  norm       layer norm of n rows of dim elements
  norm_grad  its gradient: of the rows, of the weight and of the bias
  logp       log probabilities of given tokens, with entropy and the `top` most likely alternatives, from n rows of
             vocab logits
  logp_grad  the gradient of those log probabilities (and, with `entropy`, of the entropies) in the logits
  orth       the update of a dense weight made orthogonal by Newton-Schulz steps, `batch` matrices of rows x cols

`type` is the rows', logits' or matrices' type. `pad` elements lie between the rows of the inputs (a slice of a wider
buffer). `masked` is the share of logits that a grammar or a padded vocabulary leaves at -inf.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5           # layer norm
NS_EPS, NS_STEPS = 1e-7, 5
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315   # the quintic's published coefficients


def listed():
    return [
        # one ranking request: the rows of 26 sparse features, normalised before the model (latency counts)
        {"name": "norm-request", "op": "norm", "type": "f32", "n": 26, "dim": 64, "pad": 0},
        # hidden states of a training batch
        {"name": "norm-hidden", "op": "norm", "type": "bf16", "n": 16_384, "dim": 4096, "pad": 0},
        # node rows of a graph batch, on their way to a put_grad: the repository's gnn workload
        {"name": "norm-grad-nodes", "op": "norm_grad", "type": "f32", "n": 1_000_000, "dim": 128, "pad": 0},
        # an odd width inside a wider buffer
        {"name": "norm-grad-odd", "op": "norm_grad", "type": "f16", "n": 4999, "dim": 1021, "pad": 6},
        # serving: one token's distribution, with the alternatives that an interface shows
        {"name": "logp-token", "op": "logp", "type": "bf16", "n": 1, "vocab": 128_000, "top": 20, "masked": 0.0,
         "pad": 0},
        # scoring a batch of prompts
        {"name": "logp-prompt", "op": "logp", "type": "bf16", "n": 4096, "vocab": 128_000, "top": 5, "masked": 0.0,
         "pad": 0},
        # an odd vocabulary under a grammar's mask, logits in 32 bits
        {"name": "logp-masked", "op": "logp", "type": "f32", "n": 333, "vocab": 50_003, "top": 8, "masked": 0.9,
         "pad": 0},
        # the loss of a training batch
        {"name": "logp-grad-batch", "op": "logp_grad", "type": "bf16", "n": 8192, "vocab": 32_000, "entropy": False,
         "masked": 0.0, "pad": 0},
        # policy training with an entropy term, odd vocabulary
        {"name": "logp-grad-entropy", "op": "logp_grad", "type": "f16", "n": 257, "vocab": 50_003, "entropy": True,
         "masked": 0.1, "pad": 5},
        # the projections of many small heads as one stack (latency counts)
        {"name": "orth-heads", "op": "orth", "type": "f32", "batch": 16, "rows": 64, "cols": 250},
        # a feed-forward weight, its momentum in 16 bits
        {"name": "orth-wide", "op": "orth", "type": "bf16", "batch": 1, "rows": 1024, "cols": 4096},
        # a large square weight
        {"name": "orth-square", "op": "orth", "type": "f32", "batch": 1, "rows": 4096, "cols": 4096},
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]; one in three a multiple of 64 where there is room."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v >= 128 and rng.random() < 1 / 3:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "logp", "logp_grad", "orth"])
    kind = rng.choice(list(TYPES))
    if op in ("norm", "norm_grad"):
        dim = _log(rng, 1, 16_384)
        n = _log(rng, 1, max(1, min(1_000_000, 100_000_000 // dim)))
        return {"op": op, "type": kind, "n": n, "dim": dim, "pad": rng.choice([0, 0, rng.randrange(1, 33)])}
    if op in ("logp", "logp_grad"):
        vocab = _log(rng, 64, 262_144)
        n = _log(rng, 1, max(1, min(16_384, 200_000_000 // vocab)))
        c = {"op": op, "type": kind, "n": n, "vocab": vocab, "masked": rng.choice([0.0, 0.0, rng.uniform(0.01, 0.95)]),
             "pad": rng.choice([0, 0, rng.randrange(1, 33)])}
        if op == "logp":
            c["top"] = rng.choice([0, 1, rng.randrange(2, 21), 64])
        else:
            c["entropy"] = rng.random() < 0.5
        return c
    rows, cols = _log(rng, 8, 4096), _log(rng, 8, 4096)
    batch = _log(rng, 1, max(1, min(32, 16_777_216 // (rows * cols))))
    return {"op": op, "type": kind, "batch": batch, "rows": rows, "cols": cols}


def _padded(n, width, pad, kind, fill):
    """n rows of `width` elements made by `fill`, in a buffer with `pad` more elements a row."""
    buf = torch.zeros((n, width + pad), dtype=kind, device="cuda")
    x = buf[:, :width]
    x.copy_(fill(torch.empty((n, width), dtype=torch.float32, device="cuda")))
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = TYPES[case["type"]]
    s = dict(case)
    if case["op"] in ("norm", "norm_grad"):
        n, dim, pad = case["n"], case["dim"], case["pad"]
        # rows about a mean of their own, as trained rows and hidden states are
        shift = torch.randn((n, 1), generator=g, device="cuda") * 0.3
        s["x"] = _padded(n, dim, pad, kind, lambda t: t.normal_(generator=g).add_(shift))
        s["weight"] = (1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(kind)
        s["bias"] = (0.1 * torch.randn(dim, generator=g, device="cuda")).to(kind)
        if case["op"] == "norm_grad":
            s["grad"] = _padded(n, dim, pad, kind, lambda t: t.normal_(0, 0.01, generator=g))
    elif case["op"] in ("logp", "logp_grad"):
        n, vocab = case["n"], case["vocab"]
        s["logits"] = _padded(n, vocab, case["pad"], kind, lambda t: t.normal_(0, 2.5, generator=g))
        if case["masked"]:
            off = torch.rand(vocab, generator=g, device="cuda") < case["masked"]
            off[torch.randint(vocab, (1,), generator=g, device="cuda")] = False
            s["logits"][:, off] = -math.inf
        # tokens that the model finds likely, some it does not, and padding; none that the mask rules out
        few = torch.randint(vocab, (n, 32), generator=g, device="cuda")
        likely = few.gather(1, s["logits"].gather(1, few).float().argmax(1, keepdim=True))[:, 0]
        u = torch.rand(n, generator=g, device="cuda")
        t = torch.where(u < 0.2, few[:, 0], likely)
        if case["masked"]:
            out = s["logits"].gather(1, t[:, None])[:, 0] == -math.inf
            t = torch.where(out, s["logits"].argmax(1), t)
        s["tokens"] = torch.where(u > 0.95, -1, t)
        if case["op"] == "logp_grad":
            m, logs, ent = _softmax(s["logits"])[1:]
            s["stats"], s["ent"] = torch.stack([m, logs], 1), ent
            scale = (4096 if kind == torch.float16 else 1) / n   # a mean's gradient; fp16 trains under a loss scale
            s["g_logp"] = torch.randn(n, generator=g, device="cuda") * scale
            s["g_ent"] = torch.full((n,), 0.01 * scale, device="cuda") if case["entropy"] else None
    else:
        b, r, c = case["batch"], case["rows"], case["cols"]
        # a momentum: a few strong directions in noise
        k = max(1, min(r, c) // 8)
        left = torch.randn((b, r, k), generator=g, device="cuda") * torch.logspace(0, -2, k, device="cuda")
        right = torch.randn((b, k, c), generator=g, device="cuda")
        s["g"] = (0.01 * (left @ right + torch.randn((b, r, c), generator=g, device="cuda"))).to(kind)
    return s


# ---- plain forms, in 32 bits (long sums over rows in 64) -------------------------------------------------------------
def _norm_parts(x):
    x = x.float()
    d = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    return d * r, r


def _softmax(logits):
    """Probabilities, the largest logit, the log of the sum over it, the entropy; rows of -inf: no distribution."""
    x = logits.float()
    m = x.amax(1)
    d = x - torch.where(m == -math.inf, 0.0, m)[:, None]
    e = torch.exp(d)
    total = e.sum(1)
    logs = torch.where(m == -math.inf, 0.0, torch.log(total))
    ent = torch.where(m == -math.inf, 0.0, torch.log(total) - torch.where(e > 0, e * d, 0.0).sum(1) / total)
    return e / total[:, None], m, logs, ent


def _top(logits, k):
    """The k largest, ties to the lowest index, by one key of value and index."""
    bits = (logits.float() + 0.0).view(torch.int32)
    order = bits ^ ((bits >> 31) & 0x7FFFFFFF)
    last = logits.shape[1] - 1 - torch.arange(logits.shape[1], device=logits.device)
    key = (order.long() << 32) | last
    best = torch.topk(key, k, dim=1, sorted=True).values
    return (logits.shape[1] - 1 - (best & 0xFFFFFFFF))


def _plain(s):
    op = s["op"]
    if op == "norm":
        xh, _ = _norm_parts(s["x"])
        return (xh * s["weight"].float() + s["bias"].float()).to(s["x"].dtype)
    if op == "norm_grad":
        xh, r = _norm_parts(s["x"])
        dy = s["grad"].float()
        g = dy * s["weight"].float()
        dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        kind = s["x"].dtype
        return (dx.to(kind), (dy * xh).sum(0, dtype=torch.float64).to(kind),
                dy.sum(0, dtype=torch.float64).to(kind))
    if op == "logp":
        x, t, k = s["logits"], s["tokens"], s["top"]
        _, m, logs, ent = _softmax(x)
        at = x.gather(1, t.clamp(min=0)[:, None])[:, 0].float()
        logp = torch.where(t < 0, 0.0, at - m - logs)
        out = (logp, ent, torch.stack([m, logs], 1))
        if k == 0:
            return out
        ids = _top(x, k)
        return out + (ids, x.gather(1, ids).float() - m[:, None] - logs[:, None])
    if op == "logp_grad":
        x, t = s["logits"].float(), s["tokens"]
        logq = x - s["stats"][:, :1] - s["stats"][:, 1:]
        p = torch.exp(logq)
        gl = torch.where(t < 0, 0.0, s["g_logp"])
        d = -gl[:, None] * p
        if s["g_ent"] is not None:
            d -= torch.where(p > 0, s["g_ent"][:, None] * p * (logq + s["ent"][:, None]), 0.0)
        d[torch.arange(x.shape[0], device=x.device), t.clamp(min=0)] += gl
        return d.to(s["logits"].dtype)
    x = s["g"].float()
    wide = x.shape[1] <= x.shape[2]
    if not wide:
        x = x.transpose(1, 2)
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    for _ in range(NS_STEPS):
        a = x @ x.transpose(1, 2)
        x = NS_A * x + (NS_B * a + NS_C * (a @ a)) @ x
    if not wide:
        x = x.transpose(1, 2)
    return x.to(s["g"].dtype)


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _own(s):
    from paper_2504_01506_amd import ops
    op = s["op"]
    if op == "norm":
        return ops.layer_norm(s["x"], s["weight"], s["bias"], EPS)
    if op == "norm_grad":
        return ops.layer_norm_grad(s["x"], s["weight"], s["grad"], EPS)
    if op == "logp":
        r = ops.log_probs(s["logits"], s["tokens"], top=s["top"])
        out = (r.logp, r.entropy, r.stats)
        return out + (r.top_ids, r.top_logp) if s["top"] else out
    if op == "logp_grad":
        return ops.log_probs_grad(s["logits"], s["tokens"], s["stats"], s["ent"], s["g_logp"], s["g_ent"])
    return ops.orthogonalize(s["g"], steps=NS_STEPS, eps=NS_EPS)


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------
def _exact_top(x, k):
    n, vocab = x.shape
    col = torch.arange(vocab, device=x.device)[None, :]
    taken = torch.zeros_like(x, dtype=torch.bool)
    ids = torch.empty((n, k), dtype=torch.int64, device=x.device)
    for j in range(k):
        best = x.masked_fill(taken, -math.inf).amax(1, keepdim=True)
        ids[:, j] = torch.where((x == best) & ~taken, col, vocab).amin(1)
        taken.scatter_(1, ids[:, j:j + 1], True)
    return ids


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "norm_grad"):
        x, w = s["x"].double(), s["weight"].double()
        mean = x.sum(1) / case["dim"]
        std = ((x.square().sum(1) / case["dim"] - mean.square()).clamp(min=0) + EPS).sqrt()
        unit = (x - mean[:, None]) / std[:, None]
        if op == "norm":
            return unit * w + s["bias"].double()
        dy = s["grad"].double()
        dot = (dy * w * unit).sum(1) / case["dim"]
        flat = (dy @ w) / case["dim"]
        return (dy * w - flat[:, None] - unit * dot[:, None]) / std[:, None], (dy * unit).sum(0), dy.sum(0)
    if op in ("logp", "logp_grad"):
        x, t, n = s["logits"].double(), s["tokens"], case["n"]
        lse = torch.logsumexp(x, 1)
        row = torch.arange(n, device=x.device)
        if op == "logp":
            logq = x - lse[:, None]
            ent = -(logq.exp() * logq.clamp(min=-1e9)).sum(1)
            logp = logq[row, t.clamp(min=0)].masked_fill(t < 0, 0.0)
            del logq
            top = x.max(1).values
            out = (logp, ent, torch.stack([top, lse - top], 1))
            if case["top"] == 0:
                return out
            ids = _exact_top(x, case["top"])
            return out + (ids, x.gather(1, ids) - lse[:, None])
        p = torch.softmax(x, 1)
        gl = s["g_logp"].double().masked_fill(t < 0, 0.0)
        d = p * -gl[:, None]
        d[row, t.clamp(min=0)] += gl
        if case["entropy"]:
            logq = (x - lse[:, None]).clamp(min=-1e9)
            ent = -(p * logq).sum(1, keepdim=True)
            d -= p * (logq + ent) * s["g_ent"].double()[:, None]
        return d
    out = []
    for m in s["g"].double():
        y = m if m.shape[0] <= m.shape[1] else m.t()
        y = y / (torch.linalg.norm(y) + NS_EPS)
        for _ in range(NS_STEPS):
            q = torch.mm(y, y.t().contiguous())
            z = torch.mm(q, y)
            y = NS_A * y + NS_B * z + NS_C * torch.mm(q, z)
        out.append(y if m.shape[0] <= m.shape[1] else y.t())
    return torch.stack(out)


def work(case):
    size, op = SIZE[case["type"]], case["op"]
    if op in ("norm", "norm_grad"):
        n, dim = case["n"], case["dim"]
        if op == "norm":
            return {"bytes": 2 * n * dim * size + 2 * dim * size, "flops": 8 * n * dim}
        return {"bytes": 3 * n * dim * size + 3 * dim * size, "flops": 16 * n * dim}
    if op == "logp":
        n, vocab = case["n"], case["vocab"]
        return {"bytes": n * vocab * size + n * (8 + 16 + case["top"] * 12), "flops": 6 * n * vocab}
    if op == "logp_grad":
        n, vocab = case["n"], case["vocab"]
        return {"bytes": 2 * n * vocab * size + n * (8 + 16 + 4 * case["entropy"]),
                "flops": (8 if case["entropy"] else 5) * n * vocab}
    b, m, n = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # x x' and its square are symmetric: half of each
    return {"bytes": 2 * b * m * n * size, "flops": b * NS_STEPS * (m * m * n + m * m * m + 2 * m * m * n)}
