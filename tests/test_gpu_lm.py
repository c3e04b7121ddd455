"""The operators as a model runs them: a feed-forward layer and the head through a training step, and a decoded token through both halves of a block."""
import pytest
import torch

import fused_helpers as f
from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import decode, ffn, head

pytestmark = pytest.mark.gpu


def values(cfg, planes, rows, cols, axis=1):
    return bdr.bdr_unpack(cfg, planes, torch.empty(rows, cols, device="cuda"), axis).double()


@pytest.mark.parametrize("fmt", ["mx4", "mx6", "mx9"])
def test_training_step(fmt):
    tokens, d_model, d_ff, vocab = 512, 256, 768, 1111
    cfg = f.CFG[fmt]
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    x, w1, w2, wv = rand(tokens, d_model).bfloat16(), (rand(2 * d_ff, d_model) * d_model ** -0.5).bfloat16(), (rand(d_model, d_ff) * d_ff ** -0.5).bfloat16(), rand(vocab, d_model) * d_model ** -0.5
    targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    targets[:50] = -100
    layer, top = ffn.alloc(cfg, tokens, d_model, d_ff, act=bdr.ACT_GELU), head.alloc(cfg, tokens, vocab, d_model)
    y = ffn.forward(x, w1, w2, layer)
    loss = head.losses(y, wv, targets, top)
    counted = (targets >= 0).float()
    dy, dwv = head.gradients(targets, counted / counted.sum(), top)
    h, gate_up = layer.h.clone(), layer.gate_up.clone()              # the backward pass reuses h
    dx, dw1, dw2 = ffn.backward(dy, layer)

    # each kernel against the formula of the operands it was given, as they are quantized
    p = layer.planes
    xq, w1q = values(cfg, p["x", 1], tokens, d_model), values(cfg, p["w_gate_up", 1], 2 * d_ff, d_model)
    want, products, eh, e = f.gated(xq, w1q, d_ff, "gelu")
    half = f.HALF_STEP[torch.bfloat16]
    f.check(gate_up, products, e + half * (products.abs() + e), "gate_up")
    f.check(h, want, eh + half * (want.abs() + eh) + 2.0 ** -126, "h")
    hq, w2q = values(cfg, p["h", 1], tokens, d_ff), values(cfg, p["w_down", 1], d_model, d_ff)
    f.check(y, hq @ w2q.T, f.sum_bound(d_ff, hq.abs() @ w2q.abs().T), "y")
    yq, wvq = values(cfg, top.hidden, tokens, d_model), values(cfg, top.weight, vocab, d_model)
    want_loss, want_lse, _, eloss, elog, _ = f.entropy(yq, wvq, targets)
    f.check(loss, want_loss, eloss, "loss")
    want_dy, want_dwv, edy, edwv = f.entropy_grads(yq, wvq, targets, top.lse.double(), (counted / counted.sum()).double(), torch.bfloat16)
    f.check(dy, want_dy, edy, "dy")
    f.check(dwv, want_dwv, edwv, "dwv")
    dyr, dyc = values(cfg, p["dy", 1], tokens, d_model), values(cfg, p["dy", 0], tokens, d_model, 0)
    w2c, hc = values(cfg, p["w_down", 0], d_model, d_ff, 0), values(cfg, p["h", 0], tokens, d_ff, 0)
    f.check(layer.dh, dyr @ w2c, f.sum_bound(d_model, dyr.abs() @ w2c.abs()), "dh")
    f.check(dw2, dyc.T @ hc, f.sum_bound(tokens, dyc.abs().T @ hc.abs()), "dw2")
    dh = layer.dh.bfloat16().double()
    want_dx, want_dw1, edx, edw1 = f.gated_grads(xq, w1q, d_ff, "gelu", dh, gate_up.double(), torch.zeros_like(gate_up, dtype=torch.float64), torch.bfloat16)
    f.check(dx, want_dx, edx, "dx")
    f.check(dw1, want_dw1, edw1, "dw1")
    assert bdr.bdr_device_status() == 0 and bdr.mx_gemm_status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_token_through_a_whole_block(dtype):
    n_seqs, d_model, n_q, n_kv, d, d_ff = 3, 512, 8, 2, 64, 1000
    gen = torch.Generator(device="cuda").manual_seed(2)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    cache = bdr.alloc_kv_cache(bdr.MX9, bdr.MX6, 8, 16, n_kv, d)
    block = decode.alloc(bdr.MX6, rand((n_q + 2 * n_kv) * d, d_model) / 20, rand(d_model, n_q * d) / 20, cache, n_q, n_seqs, 64, 32, dtype)
    w1, w2 = rand(2 * d_ff, d_model) * d_model ** -0.5, rand(d_model, d_ff) * d_ff ** -0.5
    feed = decode.alloc_feed_forward(bdr.MX6, w1, w2, n_seqs, act=bdr.ACT_SILU, dtype=dtype)
    table = torch.arange(n_seqs, dtype=torch.int32, device="cuda")[:, None]
    lengths = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")
    w1q, w2q = values(bdr.MX6, feed.w_gate_up, 2 * d_ff, d_model), values(bdr.MX6, feed.w_down, d_model, d_ff)
    half = f.HALF_STEP[dtype]
    for _ in range(2):
        h = rand(n_seqs, d_model).to(dtype)
        a = h + decode.step(block, h, table, lengths)
        out = decode.feed_forward(feed, a)
        want, _, eh, _ = f.gated(a.double(), w1q, d_ff, "silu")
        f.check(feed.hidden, want, eh + half * (want.abs() + eh) + 2.0 ** -126, "hidden")
        hidden = feed.hidden.double()
        f.check(out, hidden @ w2q.T, (1 + half) * f.sum_bound(d_ff, hidden.abs() @ w2q.abs().T) + half * (hidden @ w2q.T).abs() + 2.0 ** -126, "out")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = decode.feed_forward(feed, a, stream=side)
    side.synchronize()
    assert torch.equal(other, out) and (lengths == 2).all()


def test_the_head_keeps_the_weights_it_packed():
    tokens, vocab, d_model = 100, 333, 200
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    x, z, w = rand(tokens, d_model), rand(tokens, d_model), rand(vocab, d_model) * d_model ** -0.5
    targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    kept, fresh = head.alloc(bdr.MX9, tokens, vocab, d_model), head.alloc(bdr.MX9, tokens, vocab, d_model)
    head.losses(x, w, targets, kept)
    assert torch.equal(head.losses(z, None, targets, kept), head.losses(z, w, targets, fresh))


# rows around those that one pass of the search for the largest weight holds in flight (256 threads, 16 rows each); the largest is the last
@pytest.mark.parametrize("tokens", [4095, 4096, 4097, 4353, 8192, 8193])
def test_the_largest_weight_of_many_rows(tokens):
    vocab, d_model = 70, 48
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    dloss = torch.rand(tokens, device="cuda", generator=gen) * 2.0 ** -12
    dloss[-1] = 3.0
    buf = head.alloc(bdr.MX6, tokens, vocab, d_model)
    head.losses(rand(tokens, d_model), rand(vocab, d_model) * d_model ** -0.5, targets, buf)
    da, dw = head.gradients(targets, dloss, buf)
    xq, wq = values(bdr.MX6, buf.hidden, tokens, d_model), values(bdr.MX6, buf.weight, vocab, d_model)
    want_da, want_dw, ea, ew = f.entropy_grads(xq, wq, targets, buf.lse.double(), dloss.double(), torch.bfloat16)
    f.check(da, want_da, ea, "da")
    f.check(dw, want_dw, ew, "dw")


def test_a_captured_training_step_is_the_eager_one():
    tokens, d_model, d_ff, vocab = 256, 256, 512, 777
    gen = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    x, w1, w2, wv = rand(tokens, d_model).bfloat16(), (rand(2 * d_ff, d_model) / 16).bfloat16(), (rand(d_model, d_ff) / 22).bfloat16(), rand(vocab, d_model) / 16
    targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=gen)
    dloss = torch.full((tokens,), 1 / tokens, device="cuda")
    layer, top = ffn.alloc(bdr.MX6, tokens, d_model, d_ff), head.alloc(bdr.MX6, tokens, vocab, d_model)

    def step():
        head.losses(ffn.forward(x, w1, w2, layer), wv, targets, top)
        dy, dwv = head.gradients(targets, dloss, top)
        return (top.loss, dwv, *ffn.backward(dy, layer))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(2):
        x.copy_(rand(tokens, d_model))
        targets.copy_(torch.randint(-1, vocab, (tokens,), device="cuda", generator=gen))
        graph.replay()
        got = [t.clone() for t in held]
        for t in held:
            t.zero_()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
    assert bdr.bdr_device_status() == 0 and bdr.mx_gemm_status() == 0
