"""The vocabulary head of a language model on MX storage: hidden states and vocabulary weights are quantized along the reduction dimension,
the softmax cross entropy of their product is taken without storing the logits, and its gradients are those of the quantized operands.
This module only sequences calls of the C ABI.
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as bdr


@dataclass
class HeadBuffers:
    """Everything the head writes, allocated once by the caller."""
    cfg: bdr.Config
    hidden: bdr.Planes      # [tokens, d_model]
    weight: bdr.Planes      # [vocab, d_model]
    loss: torch.Tensor      # [tokens] float32
    lse: torch.Tensor       # [tokens] float32
    d_hidden: torch.Tensor  # [tokens, d_model]
    d_weight: torch.Tensor  # [vocab, d_model]
    workspace: torch.Tensor


def alloc(cfg: bdr.Config, tokens: int, vocab: int, d_model: int, dtype=torch.bfloat16, device="cuda") -> HeadBuffers:
    """dtype: of the gradients.  Any sizes."""
    size = max(bdr.mx_cross_entropy_workspace_bytes(tokens, vocab, d_model), bdr.mx_cross_entropy_bwd_workspace_bytes(tokens, vocab, d_model, dtype))
    new = lambda *s, dt=torch.float32: torch.empty(s, dtype=dt, device=device)  # noqa: E731
    return HeadBuffers(cfg, bdr.alloc_planes(cfg, tokens, d_model, device=device), bdr.alloc_planes(cfg, vocab, d_model, device=device), new(tokens), new(tokens),
                       new(tokens, d_model, dt=dtype), new(vocab, d_model, dt=dtype), new(size, dt=torch.uint8))


def losses(hidden: torch.Tensor, weight: torch.Tensor | None, targets: torch.Tensor, buf: HeadBuffers, stream=None) -> torch.Tensor:
    """Loss of every token: hidden [tokens, d_model], weight [vocab, d_model] (None: as packed by the call before), targets int64 [tokens]
    (negative: the token does not count, loss 0)."""
    cfg, (tokens, d_model), vocab = buf.cfg, hidden.shape, buf.d_weight.shape[0]
    bdr.bdr_pack(cfg, hidden, buf.hidden, stream=stream)
    if weight is not None:
        bdr.bdr_pack(cfg, weight, buf.weight, stream=stream)
    bdr.mx_cross_entropy(cfg, buf.hidden, cfg, buf.weight, tokens, vocab, d_model, targets, buf.loss, buf.lse, buf.workspace, stream=stream)
    return buf.loss


def gradients(targets: torch.Tensor, dloss: torch.Tensor, buf: HeadBuffers, stream=None):
    """d_hidden and d_weight from dloss (float32 [tokens]); `buf` is as the call of `losses` left it."""
    (tokens, d_model), vocab = buf.d_hidden.shape, buf.d_weight.shape[0]
    bdr.mx_cross_entropy_bwd(buf.cfg, buf.hidden, buf.cfg, buf.weight, tokens, vocab, d_model, targets, buf.lse, dloss, buf.d_hidden, buf.d_weight, buf.workspace,
                             stream=stream)
    return buf.d_hidden, buf.d_weight
