"""One gated feed-forward layer in MX training form: like ``linear``, every product takes MX-quantized operands, and the two products
of the gated half are one kernel.  This module only sequences calls of the C ABI (and rounds dh to bf16 with a copy); all arithmetic is in
the kernels.

    H  = act(X Wg^T) * (X Wu^T)                mx_gated_gemm: X, [Wg; Wu] row-wise
    Y  = H Wd^T         reduce over d_ff     : H row-wise, Wd row-wise
    dH = dY Wd          reduce over d_model  : dY row-wise, Wd column-wise
    dWd = dY^T H        reduce over tokens   : dY column-wise, H column-wise
    dX, [dWg; dWu]                             mx_gated_gemm_bwd: the gradients of the first line with regard to the quantized X and weights

(the gradients inside the gated half enter their products in bf16 instead of being quantized, which is this library's choice: they
are exactly the gradients of what the forward pass computed).
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as bdr
from . import linear


@dataclass
class FeedForwardBuffers:
    """Everything the layer writes, allocated once by the caller."""
    cfg: bdr.Config
    act: int
    planes: dict            # (name, axis) -> Planes
    h: torch.Tensor         # [tokens, d_ff] bfloat16
    gate_up: torch.Tensor   # [tokens, 2 d_ff] bfloat16: both products, for the backward pass
    y: torch.Tensor         # [tokens, d_model] float32
    dh: torch.Tensor        # [tokens, d_ff] float32
    dx: torch.Tensor        # [tokens, d_model] bfloat16
    dw_gate_up: torch.Tensor  # [2 d_ff, d_model] bfloat16
    dw_down: torch.Tensor   # [d_model, d_ff] float32
    workspace: torch.Tensor


def alloc(cfg: bdr.Config, tokens: int, d_model: int, d_ff: int, act: int = bdr.ACT_SILU, device="cuda") -> FeedForwardBuffers:
    """Sizes are multiples of 256 (the products of ``mx_gemm_ws`` and ``mx_gemm_f8`` take whole tiles)."""
    if tokens % 256 or d_model % 256 or d_ff % 256 or min(tokens, d_model, d_ff) < 256:
        raise ValueError("tokens, d_model and d_ff are multiples of 256")
    shapes = {"x": (tokens, d_model), "w_gate_up": (2 * d_ff, d_model), "h": (tokens, d_ff), "w_down": (d_model, d_ff), "dy": (tokens, d_model)}
    both = ("h", "w_down", "dy")
    planes = {(n, ax): bdr.alloc_planes(cfg, *s, ax, device=device) for n, s in shapes.items() for ax in ((1, 0) if n in both else (1,))}
    new = lambda r, c, dt: torch.empty((r, c), dtype=dt, device=device)  # noqa: E731
    b16, f32 = torch.bfloat16, torch.float32
    product = bdr.mx_gemm_f8_workspace_bytes if cfg.m <= 4 else bdr.mx_gemm_workspace_bytes
    size = max(bdr.mx_gated_gemm_workspace_bytes(tokens, d_ff, d_model), bdr.mx_gated_gemm_bwd_workspace_bytes(tokens, d_ff, d_model),
               product(tokens, d_model, d_ff), product(tokens, d_ff, d_model), product(d_model, d_ff, tokens))
    return FeedForwardBuffers(cfg, act, planes, new(tokens, d_ff, b16), new(tokens, 2 * d_ff, b16), new(tokens, d_model, f32), new(tokens, d_ff, f32),
                              new(tokens, d_model, b16), new(2 * d_ff, d_model, b16), new(d_model, d_ff, f32),
                              torch.empty(size, dtype=torch.uint8, device=device))


def forward(x: torch.Tensor, w_gate_up: torch.Tensor, w_down: torch.Tensor, buf: FeedForwardBuffers, stream=None) -> torch.Tensor:
    """Y [tokens, d_model] for x [tokens, d_model], w_gate_up [2 d_ff, d_model] (the gate's rows first) and w_down [d_model, d_ff]."""
    cfg, p = buf.cfg, buf.planes
    (tokens, d_model), d_ff = x.shape, w_down.shape[1]
    bdr.bdr_pack(cfg, x, p["x", 1], stream=stream)
    bdr.bdr_pack(cfg, w_gate_up, p["w_gate_up", 1], stream=stream)
    bdr.bdr_pack2(cfg, w_down, p["w_down", 1], p["w_down", 0], stream=stream)
    bdr.mx_gated_gemm(cfg, p["x", 1], cfg, p["w_gate_up", 1], tokens, d_ff, d_model, buf.h, buf.workspace, act=buf.act, gate_up=buf.gate_up, stream=stream)
    bdr.bdr_pack2(cfg, buf.h, p["h", 1], p["h", 0], stream=stream)
    linear.product(cfg, p["h", 1], p["w_down", 1], tokens, d_model, d_ff, buf.y, buf.workspace, stream)
    return buf.y


def backward(dy: torch.Tensor, buf: FeedForwardBuffers, stream=None):
    """dX, d[Wg; Wu] and dWd from dy [tokens, d_model]; `buf` is as the forward call left it."""
    cfg, p = buf.cfg, buf.planes
    (tokens, d_model), d_ff = dy.shape, buf.h.shape[1]
    bdr.bdr_pack2(cfg, dy, p["dy", 1], p["dy", 0], stream=stream)
    linear.product(cfg, p["dy", 1], p["w_down", 0], tokens, d_ff, d_model, buf.dh, buf.workspace, stream)
    linear.product(cfg, p["dy", 0], p["h", 0], d_model, d_ff, tokens, buf.dw_down, buf.workspace, stream)
    with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
        buf.h.copy_(buf.dh)                     # h is not needed any more: dH takes its place, rounded to its type
    bdr.mx_gated_gemm_bwd(cfg, p["x", 1], cfg, p["w_gate_up", 1], tokens, d_ff, d_model, buf.h, buf.dx, buf.dw_gate_up, buf.workspace, act=buf.act,
                          gate_up=buf.gate_up, stream=stream)
    return buf.dx, buf.dw_gate_up, buf.dw_down
