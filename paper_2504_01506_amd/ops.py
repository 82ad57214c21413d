"""The dense operators of a training step around a table, on torch tensors.

What a step computes between the get of its rows and the put_grad of their
gradients, as far as it is row-wise (layer_norm, log_probs and their
gradients), and the update of a dense weight that no table holds
(orthogonalize). Each is one call of the library (include/mlkv.h says what it
computes): tensors are checked here and passed as device pointers, outputs and
workspaces that are not given are allocated by torch, and the work is queued on
`stream` (the current stream of the tensors' device unless given) without
waiting for it. They stand outside torch's autograd: gradients are calls of
their own, and while autograd records, a tensor that requires a gradient is
refused (call under torch.no_grad(), on tensor.detach(), or from the forward and
backward of a torch.autograd.Function). What is written to a given `out` counts
as a change of it in place. There is no fallback: without the built library, or on tensors
that are not on a GPU, a call raises.

As with any torch call on a side stream, a tensor that is given and was made on
another stream than `stream` must be ready there, and kept until the work is
done; what a call allocates belongs to `stream`.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import mlkv

# a stream's handle without the Stream object around it (a microsecond and a half a call), and the current device
# without a look at whether torch has started the GPU (a tensor is there), where torch has those
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_recording = torch.is_grad_enabled

_TYPES = {torch.float32: mlkv.MLKV_F32, torch.bfloat16: mlkv.MLKV_BF16, torch.float16: mlkv.MLKV_F16}


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _dtype(t: torch.Tensor, what: str) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"{what} must be float32, bfloat16 or float16, not {t.dtype}")
    return kind


def _check(t: torch.Tensor, what: str, like: torch.Tensor, dtype=None, shape=None, dense=False):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{what} must be a tensor")
    if t.get_device() != like.get_device():
        raise ValueError(f"{what} is on {t.device}, not on {like.device}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, not {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{what} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    if dense and not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if t.is_neg():
        raise ValueError(f"{what} must be resolved first")


def _on_gpu(t: torch.Tensor, what: str):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} must be a tensor on a GPU")
    if t.is_neg():
        raise ValueError(f"{what} must be resolved first")


def _no_graph(*tensors):
    """Refuses tensors that autograd would expect a gradient for: the result has no history."""
    if _recording():
        for t in tensors:
            if t is not None and getattr(t, "requires_grad", False):
                raise ValueError("the dense operators are not recorded by autograd: call them under torch.no_grad(), "
                                 "on tensor.detach(), or from a torch.autograd.Function")


def _changed(out: Optional[torch.Tensor]):
    """Tells autograd that a given output has been written."""
    if out is not None:
        torch.autograd.graph.increment_version(out)


def _rows(t: torch.Tensor, what: str) -> tuple[int, int, int]:
    """(rows, elements a row, elements from row to row) of a tensor whose last
    dimension is the row and whose others follow one another evenly."""
    if t.dim() == 0:
        raise ValueError(f"{what} must have at least one dimension")
    width = t.shape[-1]
    if width == 0:
        raise ValueError(f"{what} has rows of no elements")
    n = t.numel() // width
    if t.is_contiguous():
        return n, width, width
    if t.stride(-1) != 1 and width > 1:
        raise ValueError(f"{what}: the elements of a row must lie next to each other")
    if n <= 1:
        return n, width, width
    stride = None
    for size, step in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if stride is None:
            stride, reach = step, step * size
        elif step == reach:
            reach *= size
        else:
            raise ValueError(f"{what}: the rows must be evenly spaced")
    return n, width, stride


def _out_rows(t: Optional[torch.Tensor], like: torch.Tensor, width: int) -> tuple[torch.Tensor, int]:
    """The output of rows like `like`'s, and the elements from row to row."""
    if t is None:
        return torch.empty_like(like, memory_format=torch.contiguous_format), width
    _check(t, "out", like, like.dtype, like.shape)
    return t, _rows(t, "out")[2]


class _Queue:
    """Makes a tensor's device current, and `stream` its current stream; entered, gives the stream's handle.
    Where both are so already nothing is changed (a call's host time counts in microseconds)."""
    __slots__ = ("device", "stream", "held")

    def __init__(self, t: torch.Tensor, stream):
        self.device, self.stream, self.held = t.device, stream, None

    def __enter__(self) -> int:
        if self.stream is None and self.device.index == _current_device():
            return _raw_stream(self.device.index)
        s = self.stream
        if s is None:
            s = torch.cuda.current_stream(self.device)
        elif isinstance(s, int):  # (a handle; 0 is the device's default stream)
            s = torch.cuda.ExternalStream(s, device=self.device) if s else torch.cuda.default_stream(self.device)
        elif s.device != self.device:
            raise ValueError(f"the stream is of {s.device}, the tensors are on {self.device}")
        self.held = torch.cuda.stream(s)
        self.held.__enter__()
        return s.cuda_stream

    def __exit__(self, *what):
        if self.held is not None:
            self.held.__exit__(*what)


def _bytes(n: int) -> int:
    if n < 0:
        raise mlkv.MlkvError(n, mlkv.last_error())
    return n


def _param(p: Optional[torch.Tensor], what: str, x: torch.Tensor, dim: int):
    """Checks a weight or a bias: fp32 or of x's type."""
    if p is None:
        return
    _check(p, what, x, None, (dim,), True)
    if p.dtype != torch.float32 and p.dtype != x.dtype:
        raise ValueError(f"{what} must be float32 or {x.dtype}, not {p.dtype}")


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Layer norm over the last dimension of x ([..., dim], fp32, bf16 or fp16);
    weight and bias ([dim], fp32 or of x's type) may be None. `out` may be x."""
    _no_graph(x, weight, bias, out)
    _on_gpu(x, "x")
    kind = _dtype(x, "x")
    n, dim, step = _rows(x, "x")
    _param(weight, "weight", x, dim)
    _param(bias, "bias", x, dim)
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must be of one type")
    p = weight if weight is not None else bias
    wkind = kind if p is None else _TYPES[p.dtype]
    with _Queue(x, stream) as st:
        y, ystep = _out_rows(out, x, dim)
        mlkv._check(mlkv.load().mlkv_layer_norm(x.data_ptr(), step, _ptr(weight), _ptr(bias), n, dim, eps, kind, wkind,
                                                y.data_ptr(), ystep, st))
    _changed(out)
    return y


def layer_norm_grad(x: torch.Tensor, weight: Optional[torch.Tensor], grad: torch.Tensor, eps: float = 1e-5,
                    out: Optional[torch.Tensor] = None, stream=None):
    """(x_grad, weight_grad, bias_grad) of layer_norm(x, weight, bias, eps) for
    the gradient `grad` of its output. x_grad is of x's type (rows for a
    table's put_grad where that is fp32) and goes to `out` if given (which may
    be grad or x); the other two are of weight's type, or x's without a weight."""
    _no_graph(x, weight, grad, out)
    _on_gpu(x, "x")
    kind = _dtype(x, "x")
    n, dim, step = _rows(x, "x")
    _param(weight, "weight", x, dim)
    wkind = kind if weight is None else _TYPES[weight.dtype]
    _check(grad, "grad", x, x.dtype, x.shape)
    gstep = _rows(grad, "grad")[2]
    with _Queue(x, stream) as st:
        dx, dstep = _out_rows(out, x, dim)
        dw = x.new_empty(dim) if weight is None else torch.empty_like(weight)
        db = torch.empty_like(dw)
        lib = mlkv.load()
        nbytes = _bytes(lib.mlkv_layer_norm_grad_workspace(n, dim))
        work = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
        mlkv._check(lib.mlkv_layer_norm_grad(x.data_ptr(), step, _ptr(weight), grad.data_ptr(), gstep, n, dim, eps, kind,
                                             wkind, dx.data_ptr(), dstep, dw.data_ptr(), db.data_ptr(),
                                             work.data_ptr(), nbytes, st))
    _changed(out)
    return dx, dw, db


class LogProbs(NamedTuple):
    logp: torch.Tensor                   # fp32, the tokens' shape
    entropy: torch.Tensor                # fp32
    stats: torch.Tensor                  # fp32 [..., 2]: largest logit, log of the sum of exp(logit - largest)
    top_ids: Optional[torch.Tensor]      # int64 [..., top], largest first, equal ones lowest index first
    top_logp: Optional[torch.Tensor]     # fp32 [..., top]


def log_probs(logits: torch.Tensor, tokens: torch.Tensor, top: int = 0, stream=None) -> LogProbs:
    """Log probability of tokens[...] (int64; < 0: none, gives 0) under
    logits[..., vocab], the distribution's entropy, and the `top` (<= 64) most
    likely alternatives. `stats` and `entropy` are what log_probs_grad takes."""
    _no_graph(logits)
    _on_gpu(logits, "logits")
    kind = _dtype(logits, "logits")
    n, vocab, step = _rows(logits, "logits")
    lead = logits.shape[:-1]
    _check(tokens, "tokens", logits, torch.int64, lead, dense=True)
    top = int(top)
    with _Queue(logits, stream) as st:
        lib = mlkv.load()
        nbytes = _bytes(lib.mlkv_log_probs_workspace(n, vocab, top, kind))

        logp = torch.empty(lead, dtype=torch.float32, device=logits.device)
        r = LogProbs(logp, torch.empty_like(logp), logp.new_empty((*lead, 2)),
                     tokens.new_empty((*lead, top)) if top else None, logp.new_empty((*lead, top)) if top else None)
        work = torch.empty(nbytes, dtype=torch.uint8, device=logits.device) if nbytes else None
        mlkv._check(lib.mlkv_log_probs(logits.data_ptr(), step, tokens.data_ptr(), n, vocab, top, kind, logp.data_ptr(),
                                       r.entropy.data_ptr(), r.stats.data_ptr(), _ptr(r.top_ids), _ptr(r.top_logp),
                                       _ptr(work), nbytes, st))
    return r


def log_probs_grad(logits: torch.Tensor, tokens: Optional[torch.Tensor], stats: torch.Tensor,
                   entropy: Optional[torch.Tensor], logp_grad: Optional[torch.Tensor],
                   entropy_grad: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                   stream=None) -> torch.Tensor:
    """Gradient in the logits, for the gradients logp_grad and entropy_grad
    (fp32, either may be None) of log_probs' first two outputs; `out` may be logits."""
    _no_graph(logits, stats, entropy, logp_grad, entropy_grad, out)
    _on_gpu(logits, "logits")
    kind = _dtype(logits, "logits")
    n, vocab, step = _rows(logits, "logits")
    lead = logits.shape[:-1]
    if logp_grad is not None:
        _check(logp_grad, "logp_grad", logits, torch.float32, lead, dense=True)
        if tokens is None:
            raise ValueError("logp_grad needs tokens")
    if tokens is not None:
        _check(tokens, "tokens", logits, torch.int64, lead, dense=True)
    _check(stats, "stats", logits, torch.float32, (*lead, 2), dense=True)
    if entropy_grad is not None:
        _check(entropy_grad, "entropy_grad", logits, torch.float32, lead, dense=True)
        if entropy is None:
            raise ValueError("entropy_grad needs entropy")
    if entropy is not None:
        _check(entropy, "entropy", logits, torch.float32, lead, dense=True)
    with _Queue(logits, stream) as st:
        grad, gstep = _out_rows(out, logits, vocab)
        mlkv._check(mlkv.load().mlkv_log_probs_grad(logits.data_ptr(), step, _ptr(tokens), stats.data_ptr(),
                                                    _ptr(entropy), _ptr(logp_grad), _ptr(entropy_grad), n, vocab, kind,
                                                    grad.data_ptr(), gstep, st))
    _changed(out)
    return grad


def _matrices(t: torch.Tensor, what: str) -> tuple[int, int]:
    """(elements from matrix to matrix, from row to row) of [rows, cols] or [batch, rows, cols]."""
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{what}: the elements of a row must lie next to each other")
    row = t.stride(-2) if t.shape[-2] > 1 else t.shape[-1]
    if t.dim() == 2 or t.shape[0] <= 1:
        return t.shape[-2] * t.shape[-1], row
    return t.stride(0), row


def _standing(t: torch.Tensor) -> bool:
    """Whether t's matrices are transposed views: columns' elements next to each other."""
    return t.stride(-1) != 1 and t.stride(-2) == 1 and t.shape[-1] > 1


def orthogonalize(g: torch.Tensor, steps: int = 5, eps: float = 1e-7, out: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """The update g ([rows, cols], or [batch, rows, cols] for a stack of them;
    fp32, bf16 or fp16) made nearly orthogonal by `steps` Newton-Schulz steps:
    the same singular vectors, singular values near 1. `out` may be g. A
    transposed view is taken as it lies: its transpose is worked on (one of g and
    `out` alone: the result is copied from a buffer of its own)."""
    _no_graph(g, out)
    _on_gpu(g, "g")
    kind = _dtype(g, "g")
    if g.dim() not in (2, 3):
        raise ValueError("g must have 2 or 3 dimensions")
    if g.shape[-1] == 0 or g.shape[-2] == 0:
        raise ValueError("g has matrices of no elements")
    if out is not None:
        _check(out, "out", g, g.dtype, g.shape)
        if _standing(g) != _standing(out):
            _matrices(out.mT if _standing(out) else out, "out")
            with _Queue(g, stream):
                return out.copy_(orthogonalize(g, steps, eps))
    if _standing(g):
        x = orthogonalize(g.mT, steps, eps, None if out is None else out.mT, stream).mT
        return x if out is None else out
    batch = g.shape[0] if g.dim() == 3 else 1
    rows, cols = g.shape[-2:]
    gb, gr = _matrices(g, "g")
    with _Queue(g, stream) as st:
        x = torch.empty_like(g, memory_format=torch.contiguous_format) if out is None else out
        xb, xr = _matrices(x, "out")
        lib = mlkv.load()
        nbytes = _bytes(lib.mlkv_orthogonalize_workspace(batch, rows, cols))
        work = torch.empty(nbytes, dtype=torch.uint8, device=g.device) if nbytes else None
        mlkv._check(lib.mlkv_orthogonalize(g.data_ptr(), gb, gr, batch, rows, cols, int(steps), eps, kind,
                                           x.data_ptr(), xb, xr, _ptr(work), nbytes, st))
    _changed(out)
    return x
