"""Attention with normalised, rotated queries and keys, for training: autograd
around the C-ABI calls dpb_qk_norm_rope and dpb_attention_forward / _backward.

The paper's backbone is a GPT-2 style transformer (§3); its attention is not
described further. ``Attention`` is the drop-in for that place: one packed
projection, RMS norm of every query and key head, rotary positions (either may
be turned off), causal attention over the batch's sequences, one output
projection. Every step between the projections runs in the library's kernels;
the gradient of the whole projection is written by them into one buffer. The
gradients have no gradient of their own: a second differentiation raises.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch import nn
from torch.autograd.function import once_differentiable

from . import dpb


def _dense(g: torch.Tensor) -> torch.Tensor:
    """An output's gradient as the kernels read it: dense and 16-byte aligned,
    which a part of a larger gradient need not be."""
    g = g.contiguous()
    return g if g.data_ptr() % 16 == 0 else g.clone()


def _like(w: Optional[torch.Tensor], x: torch.Tensor) -> Optional[torch.Tensor]:
    """A norm's weight in the rows' type: under autocast fp32 weights meet bf16
    rows, and are rounded to them as a linear layer's are."""
    return None if w is None else w.to(x.dtype)


class _AttentionFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_q, cu_k, max_q, max_k, causal, scale):
        ctx.at = (max_q, max_k, causal, scale)
        o, lse = dpb.attention_forward(q, k, v, cu_q, cu_k, *ctx.at)
        ctx.save_for_backward(q, k, v, o, lse, cu_q, cu_k)  # offsets too: a change in place before the backward raises
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, go):
        q, k, v, o, lse, cu_q, cu_k = ctx.saved_tensors
        return (*dpb.attention_backward(q, k, v, o, lse, _dense(go), cu_q, cu_k, *ctx.at),) + (None,) * 6


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q=None, cu_k=None, max_q: Optional[int] = None,
              max_k: Optional[int] = None, causal: bool = True, scale: Optional[float] = None) -> torch.Tensor:
    """dpb.attention_forward with its gradient: q [Tq, Hq, D], k and v [Tk, Hkv, D] bf16 -> o [Tq, Hq, D]."""
    return _AttentionFunction.apply(q, k, v, cu_q, cu_k, max_q, max_k, causal, scale)


class _NormRopeFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, cos, sin, positions, eps, interleaved, normalise):
        ctx.save_for_backward(q, k, wq, wk, cos, sin, positions)
        ctx.at = (eps, interleaved, normalise)
        return dpb.qk_norm_rope(q, k, _like(wq, q), _like(wk, k), cos, sin, positions, *ctx.at)

    @staticmethod
    @once_differentiable
    def backward(ctx, gq, gk):
        q, k, wq, wk, cos, sin, positions = ctx.saved_tensors
        need = wq is not None and ctx.needs_input_grad[2] or wk is not None and ctx.needs_input_grad[3]
        dq, dk, dwq, dwk = dpb.qk_norm_rope_backward(q, k, gq.contiguous(), gk.contiguous(), _like(wq, q), _like(wk, k), cos,
                                                     sin, positions, *ctx.at, weight_grads=need)
        return (dq, dk, None if wq is None or dwq is None else dwq.to(wq.dtype),
                None if wk is None or dwk is None else dwk.to(wk.dtype)) + (None,) * 6


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, weight_q=None, weight_k=None, cos=None, sin=None, positions=None,
                 eps: float = 1e-6, interleaved: bool = False, normalise: bool = True):
    """dpb.qk_norm_rope with its gradient: (q [T, Hq, D], k [T, Hk, D]) normalised and rotated."""
    return _NormRopeFunction.apply(q, k, weight_q, weight_k, cos, sin, positions, eps, interleaved, normalise)


class _PackedFunction(torch.autograd.Function):
    """From a packed projection [T, Hq + 2 Hkv, D] to attention's output; the
    gradients of q, k and v are written side by side into one buffer."""

    @staticmethod
    def forward(ctx, qkv, hq, hkv, wq, wk, cos, sin, positions, rope, cu, at):
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        if rope is not None:
            q, k = dpb.qk_norm_rope(q, k, _like(wq, q), _like(wk, k), cos, sin, positions, **rope)
        o, lse = dpb.attention_forward(q, k, v, cu, **at)
        ctx.save_for_backward(qkv, q, k, wq, wk, cos, sin, positions, cu, o, lse)
        ctx.hq, ctx.hkv, ctx.rope, ctx.at = hq, hkv, rope, at
        return o

    @staticmethod
    @once_differentiable
    def backward(ctx, go):
        qkv, q, k, wq, wk, cos, sin, positions, cu, o, lse = ctx.saved_tensors
        hq, hkv, rope = ctx.hq, ctx.hkv, ctx.rope
        grad = torch.empty_like(qkv)
        gq, gk, gv = grad[:, :hq], grad[:, hq:hq + hkv], grad[:, hq + hkv:]
        dwq = dwk = None
        if rope is None:
            dpb.attention_backward(q, k, qkv[:, hq + hkv:], o, lse, _dense(go), cu, grad_q=gq, grad_k=gk, grad_v=gv,
                                   **ctx.at)
        else:
            dq, dk, _ = dpb.attention_backward(q, k, qkv[:, hq + hkv:], o, lse, _dense(go), cu, grad_v=gv, **ctx.at)
            _, _, dwq, dwk = dpb.qk_norm_rope_backward(qkv[:, :hq], qkv[:, hq:hq + hkv], dq, dk, _like(wq, q), _like(wk, k), cos,
                                                       sin, positions, grad_q=gq, grad_k=gk, weight_grads=wq is not None, **rope)
        if dwq is not None:
            dwq, dwk = dwq.to(wq.dtype), dwk.to(wk.dtype)
        return (grad, None, None, dwq, dwk) + (None,) * 6


class Attention(nn.Module):
    """Self-attention of a transformer block: x [B, S, d] -> [B, S, d].

    ``heads`` query heads, ``kv_heads`` key and value heads (None: as many),
    head width d / heads (a multiple of 8 up to 128). ``qk_norm``: RMS norm of
    every query and key head with a learned weight. ``rotary``: rotary
    positions up to ``context`` (None or 0: none); ``rope`` holds further
    arguments of dpb.rope_tables (base, scaling, ...). forward() also takes
    packed rows x [T, d] with ``cu`` (int32 token offsets of the sequences) and
    ``longest`` (None: read from ``cu``, which waits for the device, where more
    rows than ``context`` leave open whether the tables reach); positions then
    restart at every sequence, and rows outside of ``cu`` (padding) give 0 and
    take no part in any gradient. The rows are
    bf16; parameters may be fp32 under bf16 autocast."""

    def __init__(self, d: int, heads: int, kv_heads: Optional[int] = None, qk_norm: bool = True, rotary: bool = True,
                 context: Optional[int] = 1024, rope: Optional[dict] = None, device=None, dtype=None):
        super().__init__()
        kv_heads = heads if kv_heads is None else kv_heads
        if d % heads or heads % kv_heads:
            raise ValueError(f"{heads} heads must divide d = {d}, and {kv_heads} key heads the heads")
        self.heads, self.kv_heads, self.dim = heads, kv_heads, d // heads
        if self.dim % 8 or self.dim > 128:
            raise ValueError(f"head width {self.dim} must be a multiple of 8 up to 128")
        kw = dict(device=device, dtype=dtype)
        self.qkv = nn.Linear(d, (heads + 2 * kv_heads) * self.dim, bias=False, **kw)
        self.out = nn.Linear(d, d, bias=False, **kw)
        self.q_norm = nn.Parameter(torch.ones(self.dim, **kw)) if qk_norm else None
        self.k_norm = nn.Parameter(torch.ones(self.dim, **kw)) if qk_norm else None
        cos, sin = dpb.rope_tables(context, self.dim, device=device or "cpu", **(rope or {})) if rotary and context else \
            (None, None)
        # tables stay in fp32 whatever the module is cast to
        self.register_buffer("cos", cos, persistent=False)
        self.register_buffer("sin", sin, persistent=False)
        self.context = context

    def _apply(self, fn, recurse=True):
        cos, sin = self.cos, self.sin
        super()._apply(fn, recurse)
        if cos is not None:
            self.cos, self.sin = cos.to(self.cos.device), sin.to(self.cos.device)
        return self

    def forward(self, x: torch.Tensor, cu: Optional[torch.Tensor] = None, longest: Optional[int] = None) -> torch.Tensor:
        positions = None
        if cu is None:
            B, S = x.shape[0], x.shape[1]
            longest = S
            cu = torch.arange(0, (B + 1) * S, S, dtype=torch.int32, device=x.device) if S else \
                torch.zeros(B + 1, dtype=torch.int32, device=x.device)
            if self.cos is not None:
                positions = torch.arange(S, dtype=torch.int32, device=x.device).repeat(B)
        elif self.cos is not None:
            rows = torch.arange(x.shape[0], dtype=torch.int32, device=x.device)
            # padding has no position: any row of the tables will do
            positions = (rows - cu[torch.searchsorted(cu, rows, right=True) - 1]).clamp_(0, self.context - 1)
        if self.cos is not None and longest is None and x.shape[0] > self.context:
            if torch.cuda.is_current_stream_capturing():
                raise ValueError(f"longest is needed: {x.shape[0]} rows, rotary tables for {self.context}")
            longest = int((cu[1:] - cu[:-1]).max()) if cu.numel() > 1 else 0
        if self.cos is not None and longest is not None and longest > self.context:
            raise ValueError(f"sequences of {longest} tokens, rotary tables for {self.context}")
        rope = None
        if self.q_norm is not None or self.cos is not None:
            rope = dict(normalise=self.q_norm is not None)
        qkv = self.qkv(x).view(-1, self.heads + 2 * self.kv_heads, self.dim)
        o = _PackedFunction.apply(qkv, self.heads, self.kv_heads, self.q_norm, self.k_norm, self.cos, self.sin, positions, rope,
                                  cu, dict(max_q=longest, causal=True))
        return self.out(o.reshape(*x.shape[:-1], self.heads * self.dim))
