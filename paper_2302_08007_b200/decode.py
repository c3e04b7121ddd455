"""The two halves of a decoder block, one new token per sequence, on MX storage: the weights (Section V, inferencing) and the
key-value cache are kept in the MX format; the activations stay in bf16 or fp32, which is this library's choice (the section
quantizes them too).  Like ``linear``, this module only sequences calls of the C ABI; all arithmetic is in the kernels.

    qkv  = h Wqkv^T                      mx_gemv
    k, q rotated by position; k, v       mx_kv_append: quantized and written to the sequences' next slots
    a    = attention of q over the cache mx_attn_decode
    out  = a Wout^T                      mx_gemv

    f    = act(h Wg^T) * (h Wu^T)        mx_gated_gemv
    out  = f Wdown^T                     mx_gemv
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as bdr


@dataclass
class AttentionBlock:
    """Weights, cache and buffers of one block for a fixed number of sequences, allocated once by the caller."""
    cfg_w: bdr.Config
    w_qkv: bdr.Planes        # packed along K: [(n_q + 2 n_kv) * head_dim, d_model]
    w_out: bdr.Planes        # packed along K: [d_model, n_q * head_dim]
    cache: bdr.KVCache
    n_q: int
    cos: torch.Tensor        # float32 [n_pos, rot_dim / 2]
    sin: torch.Tensor
    qkv: torch.Tensor        # [n_seqs, n_q + 2 n_kv, head_dim]
    q: torch.Tensor          # [n_seqs, n_q, head_dim], rotated
    attended: torch.Tensor   # [n_seqs, n_q, head_dim]
    workspace: torch.Tensor


def rotation_tables(n_pos: int, rot_dim: int, base: float = 10000.0, device="cuda"):
    """cos and sin of position * base^(-2 i / rot_dim), rounded to float32 from 64 bits."""
    freq = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
    angle = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * freq
    return torch.cos(angle).float(), torch.sin(angle).float()


def pack_weight(cfg: bdr.Config, w: torch.Tensor) -> bdr.Planes:
    """A [N, K] weight packed along K."""
    return bdr.bdr_pack(cfg, w, bdr.alloc_planes(cfg, w.shape[0], w.shape[1], 1, device=w.device))


def alloc(cfg_w: bdr.Config, w_qkv: torch.Tensor, w_out: torch.Tensor, cache: bdr.KVCache, n_q: int, n_seqs: int, n_pos: int,
          rot_dim: int | None = None, dtype=torch.bfloat16) -> AttentionBlock:
    heads, d = n_q + 2 * cache.n_kv, cache.head_dim
    if w_qkv.shape[0] != heads * d or w_out.shape != (w_qkv.shape[1], n_q * d):
        raise ValueError("w_qkv is [(n_q + 2 n_kv) * head_dim, d_model], w_out [d_model, n_q * head_dim]")
    dev = w_qkv.device
    cos, sin = rotation_tables(n_pos, d if rot_dim is None else rot_dim, device=dev)
    new = lambda h: torch.empty((n_seqs, h, d), dtype=dtype, device=dev)  # noqa: E731
    ws = torch.empty(bdr.mx_attn_decode_workspace_bytes(cache, n_seqs, n_q), dtype=torch.uint8, device=dev)
    return AttentionBlock(cfg_w, pack_weight(cfg_w, w_qkv), pack_weight(cfg_w, w_out), cache, n_q, cos, sin, new(heads), new(n_q), new(n_q), ws)


def slots_of(page_table: torch.Tensor, positions: torch.Tensor, page_size: int) -> torch.Tensor:
    """Cache slot of position `positions[s]` of every sequence s (int64).  A negative position gives a negative slot (padding), one beyond
    the page table a slot that no cache has, which mx_kv_append reports; neither is looked up."""
    pos, n = positions.long(), page_table.shape[1]
    absent = pos * 2 ** 31                                       # caches have fewer slots than 2^31
    if n == 0:
        return torch.where(pos < 0, absent, 2 ** 31)
    page = torch.div(pos, page_size, rounding_mode="floor")
    known = page.clamp(0, n - 1)
    slots = page_table.gather(1, known[:, None])[:, 0].long() * page_size + pos % page_size
    return torch.where(page == known, slots, absent)


def step(block: AttentionBlock, h: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor, out: torch.Tensor | None = None,
         window: int = 0, stream=None, advance: bool = True) -> torch.Tensor:
    """One token per sequence: h [n_seqs, d_model] of the tokens at positions lengths[s] (int32: how many tokens the cache holds before
    this one).  Appends their keys and values and returns the block's output [n_seqs, d_model]; `lengths` is raised by one if
    `advance` (the blocks of a model share one tensor of lengths, which only the last of them advances).  Everything runs on
    `stream` (the current one when None): the inputs have to be ready there, and an output that the step allocates belongs to it."""
    if lengths.dtype != torch.int32:
        raise ValueError("lengths: int32 [sequences]")
    c, n_q = block.cache, block.n_q
    n_seqs, d_model = h.shape
    heads = n_q + 2 * c.n_kv
    with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
        if out is None:
            out = torch.empty_like(h)
        bdr.mx_gemv(block.cfg_w, block.w_qkv, heads * c.head_dim, d_model, h, block.qkv.view(n_seqs, -1))
        q, k, v = block.qkv.split((n_q, c.n_kv, c.n_kv), 1)
        positions = lengths.long()
        bdr.mx_kv_append(c, k, v, slots_of(page_table, positions, c.page_size), positions, block.cos, block.sin, q=q, q_out=block.q)
        held = lengths.add_(1) if advance else lengths + 1
        bdr.mx_attn_decode(c, block.q, page_table, held, block.attended, block.workspace, window=window)
        bdr.mx_gemv(block.cfg_w, block.w_out, d_model, n_q * c.head_dim, block.attended.view(n_seqs, -1), out)
    return out


@dataclass
class FeedForwardBlock:
    """Weights and buffer of the gated feed-forward half for a fixed number of sequences."""
    cfg_w: bdr.Config
    w_gate_up: bdr.Planes    # packed along K: [2 d_ff, d_model], the gate's rows first
    w_down: bdr.Planes       # packed along K: [d_model, d_ff]
    act: int
    hidden: torch.Tensor     # [n_seqs, d_ff]


def alloc_feed_forward(cfg_w: bdr.Config, w_gate_up: torch.Tensor, w_down: torch.Tensor, n_seqs: int, act: int = bdr.ACT_SILU,
                       dtype=torch.bfloat16) -> FeedForwardBlock:
    d_model, d_ff = w_down.shape
    if w_gate_up.shape != (2 * d_ff, d_model):
        raise ValueError("w_gate_up is [2 d_ff, d_model], w_down [d_model, d_ff]")
    return FeedForwardBlock(cfg_w, pack_weight(cfg_w, w_gate_up), pack_weight(cfg_w, w_down), act,
                            torch.empty((n_seqs, d_ff), dtype=dtype, device=w_down.device))


def feed_forward(block: FeedForwardBlock, h: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The block's output [n_seqs, d_model] for h [n_seqs, d_model].  Everything runs on `stream` (the current one when None): h has to
    be ready there, and an output that the call allocates belongs to it."""
    n_seqs, d_model = h.shape
    d_ff = block.hidden.shape[1]
    with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
        if out is None:
            out = torch.empty_like(h)
        bdr.mx_gated_gemv(block.cfg_w, block.w_gate_up, d_ff, d_model, h, block.hidden[:n_seqs], act=block.act)
        bdr.mx_gemv(block.cfg_w, block.w_down, d_model, d_ff, block.hidden[:n_seqs], out)
    return out
