"""Both ends of the model and the stream between them, for training: autograd
around the C-ABI calls dpb_embedding, dpb_add_norm and
dpb_linear_cross_entropy_forward / _backward.

The paper's backbone is GPT-2 style with one weight for embedding and
unembedding and RMS norms (§3); it does not describe them further. Here the
lookup, the addition of a block's output to the residual with the next norm,
and the cross entropy from the last hidden rows run in the library's kernels.
The scores of tokens x vocabulary are never kept; the loss's gradient keeps theirs
in bf16 for a part of the vocabulary at a time, in 192 MB or, if that is more, 24 KB
a token (all of it where the vocabulary is that small). The gradients have no gradient of
their own: a second differentiation raises.

A forward and backward pass may be captured into a CUDA graph. As with every
function of autograd, no graph of the same parameters that was made on the
default stream may be alive then: autograd would accumulate their gradients on
that stream, outside the capture, which can end the process. Drop its outputs
before, and make the steps before the capture on the capture's stream.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch import nn
from torch.autograd.function import once_differentiable

from . import dpb


def _rows(t: torch.Tensor, dtype) -> torch.Tensor:
    """[..., d] as the [tokens, d] rows that the kernels read, of `dtype`."""
    if t.dtype is not dtype:
        t = t.to(dtype)
    if t.dim() != 2:
        t = t.reshape(-1, t.shape[-1])
    return t if t.stride(-1) == 1 and (t.shape[0] < 2 or t.stride(0) >= t.shape[1]) else t.contiguous()


def _tiles(t: torch.Tensor) -> torch.Tensor:
    """Rows as the matrix products read them: at multiples of 16 bytes."""
    return t if t.data_ptr() % 16 == 0 and (t.shape[0] < 2 or t.stride(0) % 8 == 0) else t.clone(memory_format=torch.contiguous_format)


def _flat(t: torch.Tensor) -> torch.Tensor:
    return t.reshape(-1).contiguous()


class _EmbeddingFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, weight, ids, scale):
        ctx.save_for_backward(ids)
        ctx.at = (weight.shape[0], scale)
        return dpb.embedding(_rows(weight, weight.dtype), _flat(ids), scale).view(*ids.shape, weight.shape[1])

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        ids, = ctx.saved_tensors
        return dpb.embedding_backward(_rows(gy, gy.dtype), _flat(ids), *ctx.at), None, None


def embedding(weight: torch.Tensor, ids: torch.Tensor, scale: float = 1.0) -> torch.Tensor:
    """dpb.embedding with its gradient (dense, by sorted tokens): ids of any shape -> [..., d]."""
    if weight.dim() != 2:
        raise ValueError(f"weight must be [vocab, d], got {list(weight.shape)}")
    return _EmbeddingFunction.apply(weight, ids, scale)


class Embedding(nn.Module):
    """``vocab`` rows of ``d`` values, looked up and multiplied by ``scale``."""

    def __init__(self, vocab: int, d: int, scale: float = 1.0, device=None, dtype=None):
        super().__init__()
        self.weight = nn.Parameter(torch.empty(vocab, d, device=device, dtype=dtype))
        nn.init.normal_(self.weight)
        self.scale = scale

    def forward(self, ids: torch.Tensor) -> torch.Tensor:
        return embedding(self.weight, ids, self.scale)


class _AddNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, delta, weight, eps):
        w = weight if weight is None or weight.dtype is x.dtype else weight.to(x.dtype)
        y, total = dpb.add_norm(_rows(x, x.dtype), None if delta is None else _rows(delta, x.dtype), w, eps)
        ctx.save_for_backward(total, w)
        ctx.at = (x.shape, eps, None if weight is None else weight.dtype, None if delta is None else delta.dtype)
        ctx.set_materialize_grads(False)
        return y.view(x.shape) if delta is None else (y.view(x.shape), total.view(x.shape))

    @staticmethod
    @once_differentiable
    def backward(ctx, gy, gt=None):
        total, w = ctx.saved_tensors
        shape, eps, weight_type, delta_type = ctx.at
        gw = None
        if gy is None:
            gx = gt
        else:
            dt = total.dtype
            gx, gw = dpb.add_norm_backward(total, _rows(gy, dt), None if gt is None else _rows(gt, dt), w, eps,
                                           weight_grad=ctx.needs_input_grad[2])
            gx = gx.view(shape)
        gd = gx if ctx.needs_input_grad[1] and gx is not None else None
        return gx, gd if gd is None or gd.dtype is delta_type else gd.to(delta_type), None if gw is None else gw.to(weight_type), None


def add_norm(x: torch.Tensor, delta: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
             eps: float = 1e-6):
    """dpb.add_norm with its gradient: (y, total) of the shape of x, total = x +
    delta (x itself without delta), y its RMS norm times weight. delta and the
    weight are taken in x's type."""
    if delta is None:
        return _AddNormFunction.apply(x, None, weight, eps), x
    if delta.shape != x.shape:
        raise ValueError(f"delta must have x's shape {list(x.shape)}, got {list(delta.shape)}")
    return _AddNormFunction.apply(x, delta, weight, eps)


class AddRMSNorm(nn.Module):
    """forward(x, delta) -> (y, total): the residual's addition and the norm behind it (add_norm) with a learned weight."""

    def __init__(self, d: int, eps: float = 1e-6, device=None, dtype=None):
        super().__init__()
        self.weight = nn.Parameter(torch.ones(d, device=device, dtype=dtype))
        self.eps = eps

    def forward(self, x: torch.Tensor, delta: Optional[torch.Tensor] = None):
        return add_norm(x, delta, self.weight, self.eps)


class _LossFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets, ignore_index, mean):
        h, w = _tiles(_rows(hidden, hidden.dtype)), _tiles(_rows(weight, hidden.dtype))
        loss, lse, counted = dpb.linear_cross_entropy_forward(h, w, _flat(targets), ignore_index, want_counted=True)
        ctx.save_for_backward(h, w, targets, lse, counted)
        ctx.at = (hidden.shape, weight.dtype, ignore_index, mean)
        return loss.sum() / counted[0] if mean else loss.view(targets.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, g):
        h, w, targets, lse, counted = ctx.saved_tensors
        shape, weight_type, ignore_index, mean = ctx.at
        if mean:
            g = (g / counted).expand(h.shape[0])
        else:
            g = g.reshape(-1)
            if g.stride(0) not in (0, 1):
                g = g.contiguous()
        dh, dw = dpb.linear_cross_entropy_backward(h, w, _flat(targets), lse, g, ignore_index,
                                                   want_hidden=ctx.needs_input_grad[0], want_weight=ctx.needs_input_grad[1])
        return (None if dh is None else dh.view(shape), None if dw is None else dw.to(weight_type)) + (None,) * 3


def linear_cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, ignore_index: int = -100,
                         reduction: str = "mean") -> torch.Tensor:
    """Cross entropy of the scores hidden weight^T without making them: hidden
    [..., d] bf16 (under bf16 autocast of any type, taken in bf16 as a linear
    layer's are), weight [vocab, d] (taken in bf16), targets [...]. ``reduction``
    "mean" (over the tokens that are not ignored; NaN if all are), "sum" or "none",
    in fp32. What the rows of ignored tokens hold does not matter. d has to be a
    multiple of 8."""
    if reduction not in ("mean", "sum", "none"):
        raise ValueError(f"reduction must be 'mean', 'sum' or 'none', got {reduction!r}")
    if hidden.shape[:-1] != targets.shape:
        raise ValueError(f"targets must have the shape {list(hidden.shape[:-1])}, got {list(targets.shape)}")
    if hidden.dtype is not torch.bfloat16 and torch.is_autocast_enabled("cuda") and \
            torch.get_autocast_dtype("cuda") is torch.bfloat16:
        hidden = hidden.to(torch.bfloat16)
    loss = _LossFunction.apply(hidden, weight, targets, ignore_index, reduction == "mean")
    return loss.sum() if reduction == "sum" else loss
