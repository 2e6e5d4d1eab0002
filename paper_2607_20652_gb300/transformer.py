"""A ParityTransformer of GPT-2 shape for timing the DPB inside a training step.

§3 of the paper: a GPT-2-style backbone (learned positional embeddings, tied
embedding and unembedding, RMSNorm in place of LayerNorm) with a Deep Parity
Bottleneck inserted before the input of every MLP. Weights are random
(nothing here is trained); attention and the dense layers are PyTorch's own
(cuBLAS / fused attention), the DPB layers are this library's kernels;
``attention="dpb"`` takes this library's attention as well, ``ends="dpb"`` its
embedding lookup, residual norms and cross entropy. The model exists
to measure the DPB's share of a forward + backward + optimiser step at the
paper's scale; it is not a training recipe.
"""
from __future__ import annotations

import math
from typing import Optional

import torch
import torch.nn.functional as F
from torch import nn

from . import ends as _ends
from .attention import Attention
from .layer import DPBLayer


class _Attention(nn.Module):
    def __init__(self, d: int, heads: int):
        super().__init__()
        self.heads = heads
        self.qkv = nn.Linear(d, 3 * d, bias=False)
        self.out = nn.Linear(d, d, bias=False)

    def forward(self, x):
        B, S, d = x.shape
        q, k, v = self.qkv(x).view(B, S, 3, self.heads, d // self.heads).permute(2, 0, 3, 1, 4)
        o = F.scaled_dot_product_attention(q, k, v, is_causal=True)
        return self.out(o.transpose(1, 2).reshape(B, S, d))


class _Lookup(nn.Embedding):
    """The embedding by the library's lookup."""

    def forward(self, ids):
        return _ends.embedding(self.weight, ids)


class _AddNorm(nn.RMSNorm):
    """The norm by the library's, with the residual's addition before it: (x, what is to be added) -> (norm, sum)."""

    def forward(self, x, delta=None):
        # without an eps nn.RMSNorm takes that of the type it computes bf16 rows in
        return _ends.add_norm(x, delta, self.weight, torch.finfo(torch.float32).eps if self.eps is None else self.eps)


class _Block(nn.Module):
    norm = nn.RMSNorm

    def __init__(self, d: int, heads: int, d_mlp: int, dpb: Optional[DPBLayer], attn: nn.Module):
        super().__init__()
        self.n1 = self.norm(d)
        self.attn = attn
        self.n2 = self.norm(d)
        self.dpb = dpb
        self.up = nn.Linear(d, d_mlp, bias=False)
        self.down = nn.Linear(d_mlp, d, bias=False)

    def forward(self, x):
        x = x + self.attn(self.n1(x))
        h = self.n2(x)
        if self.dpb is not None:
            h = self.dpb(h)  # the bottleneck sits before the MLP's input (§3)
        return x + self.down(F.gelu(self.up(h)))


class _StreamBlock(_Block):
    """The same with the library's residual norms: takes and gives the residual's rows and what is still to be added
    to them."""

    norm = _AddNorm

    def forward(self, x, delta=None):
        h, x = self.n1(x, delta)
        h, x = self.n2(x, self.attn(h))
        if self.dpb is not None:
            h = self.dpb(h)
        return x, self.down(F.gelu(self.up(h)))


class ParityTransformer(nn.Module):
    """GPT-2 shape (12 layers, d = 768, 12 heads, MLP 3072, vocab 50257,
    context 1024 by default) with a DPB before every MLP; ``dpb=None`` gives
    the dense model of the same shape. ``dpb`` holds DPBLayer arguments.
    ``attention="dpb"`` uses this library's attention, with normalised queries
    and keys and rotary positions in place of the learned ones (bf16;
    ``kv_heads`` key and value heads). ``ends="dpb"`` uses this library's
    embedding lookup, residual norms and, with targets, its cross entropy (bf16):
    the same model without its scores in memory (ends.py: what the loss's gradient
    keeps of them). Its modules keep their
    names and are called in the same order; blocks then take and give the
    residual's rows and what is still to be added to them, norms the norm and the sum."""

    def __init__(self, layers: int = 12, d: int = 768, heads: int = 12, d_mlp: int = 3072, vocab: int = 50257,
                 context: int = 1024, dpb: Optional[dict] = None, device=None, dtype=torch.bfloat16,
                 attention: str = "torch", kv_heads: Optional[int] = None, ends: str = "torch"):
        super().__init__()
        if ends not in ("torch", "dpb"):
            raise ValueError(f"ends must be 'torch' or 'dpb', got {ends!r}")
        if ends == "dpb" and (d % 8 or dtype is not torch.bfloat16):
            raise ValueError(f"ends='dpb' needs bfloat16 and d a multiple of 8, got {dtype} and {d}")
        self.ends = ends
        if attention not in ("torch", "dpb"):
            raise ValueError(f"attention must be 'torch' or 'dpb', got {attention!r}")
        if attention == "torch" and kv_heads not in (None, heads):
            raise ValueError("kv_heads needs attention='dpb'")
        lookup, block = (_Lookup, _StreamBlock) if ends == "dpb" else (nn.Embedding, _Block)
        self.tok = lookup(vocab, d)
        self.pos = nn.Embedding(context, d) if attention == "torch" else None
        blocks = []
        for i in range(layers):
            layer = DPBLayer(seed=i, device=device, d=d, **dpb) if dpb is not None else None
            attn = _Attention(d, heads) if attention == "torch" else Attention(d, heads, kv_heads, context=context)
            blocks.append(block(d, heads, d_mlp, layer, attn))
        self.blocks = nn.ModuleList(blocks)
        self.norm = block.norm(d)
        std = 0.02
        for p in self.parameters():
            if p.dim() >= 2:
                nn.init.normal_(p, std=std)
        for b in self.blocks:  # scaled residual projections, as in GPT-2
            nn.init.normal_(b.attn.out.weight, std=std / math.sqrt(2 * layers))
            nn.init.normal_(b.down.weight, std=std / math.sqrt(2 * layers))
        self.to(device=device)
        for p in self.parameters():  # weights in dtype; the DPB tables stay fp32
            p.data = p.data.to(dtype)

    def dpb_layers(self):
        return [b.dpb for b in self.blocks if b.dpb is not None]

    def forward(self, ids, targets=None):
        B, S = ids.shape
        x = self.tok(ids)
        if self.pos is not None:
            x = x + self.pos(torch.arange(S, device=ids.device))
        if self.ends == "dpb":
            delta = None
            for b in self.blocks:
                x, delta = b(x, delta)
            h, _ = self.norm(x, delta)
            if targets is None:
                return F.linear(h, self.tok.weight)
            return _ends.linear_cross_entropy(h, self.tok.weight, targets)
        for b in self.blocks:
            x = b(x)
        logits = F.linear(self.norm(x), self.tok.weight)  # tied unembedding
        if targets is None:
            return logits
        return F.cross_entropy(logits.float().view(-1, logits.shape[-1]), targets.view(-1))
