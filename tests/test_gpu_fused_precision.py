"""32-bit results keep 32 bits: the norm of their error beside their own.  For gradients two things are there for it, each of which a bound on every single
element would let pass: sums are handed on every sixteen instructions of the tensor core, which cuts its additions off, and the gradient of a
product enters as three bf16 parts.

Every error below is relative.  A product's gradient in three parts is off by 2^-25; sixteen truncated additions lose 16 x 2^-25 = 4.8e-7 at most of a sum
whose terms have one sign; adding the spans' sums up, with rounded additions whose errors are independent, leaves sqrt(spans) x 2^-25, 2e-7 for 48 of them; the
result's own rounding 2^-25.  In all below 1e-6.  One chain over 4096 terms in three parts would lose up to 256 x 2^-25 = 7.6e-6, and two parts leave 2^-17 / sqrt(3) = 4.4e-6 of
every term, which sums of few terms show.
"""
import pytest
import torch

import fused_helpers as f
from paper_2302_08007_b200 import binding as bdr

pytestmark = pytest.mark.gpu


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


# long sums over tokens and over outputs, and sums of two and three terms
@pytest.mark.parametrize("m,n,k", [(4096, 2048, 512), (4100, 100, 300), (130, 4099, 520), (2, 3000, 777), (2000, 1, 260), (3, 2, 100)])
@pytest.mark.parametrize("fmt", ["mx6", "mx9"])
def test_gated(m, n, k, fmt):
    gen = torch.Generator(device="cuda").manual_seed(31)
    positive = lambda *s: torch.rand(s, device="cuda", generator=gen) + 0.5  # noqa: E731
    (pa, a), (pw, w) = f.packed(f.CFG[fmt], positive(m, k)), f.packed(f.CFG[fmt], positive(2 * n, k))
    dh, gate_up = positive(m, n) * 1e-2, positive(m, 2 * n)             # (of relu, with both factors above zero: no activation's error beside the sums')
    da, dw = torch.empty(m, k, device="cuda"), torch.empty(2 * n, k, device="cuda")
    bdr.mx_gated_gemm_bwd(f.CFG[fmt], pa, f.CFG[fmt], pw, m, n, k, dh, da, dw, f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k, torch.float32)),
                          act=bdr.ACT_RELU, gate_up=gate_up)
    d = torch.cat((dh.double() * gate_up[:, n:].double(), dh.double() * gate_up[:, :n].double()), 1)
    assert off(da, d @ w) < 1e-6 and off(dw, d.T @ a) < 1e-6


# one target a row: a line of dW is one token's, or several thousand tokens'
@pytest.mark.parametrize("m,v,k", [(64, 3000, 256), (4096, 2, 320), (200, 5000, 100)])
def test_entropy(m, v, k):
    gen = torch.Generator(device="cuda").manual_seed(32)
    (pa, a), (pw, w) = f.packed(bdr.MX9, torch.rand(m, k, device="cuda", generator=gen) + 0.5), f.packed(bdr.MX6, torch.randn(v, k, device="cuda", generator=gen) * 0.1)
    targets = torch.randint(0, v, (m,), device="cuda", generator=gen) if v > 2 else torch.zeros(m, dtype=torch.int64, device="cuda")
    logits = a @ w.T
    lse, dloss = torch.logsumexp(logits, 1).float(), torch.rand(m, device="cuda", generator=gen) + 0.5
    da, dw = torch.empty(m, k, device="cuda"), torch.empty(v, k, device="cuda")
    bdr.mx_cross_entropy_bwd(bdr.MX9, pa, bdr.MX6, pw, m, v, k, targets, lse, dloss, da, dw,
                             f.workspace(bdr.mx_cross_entropy_bwd_workspace_bytes(m, v, k, torch.float32)))
    d = torch.exp(logits - lse.double()[:, None])
    d[torch.arange(m, device="cuda"), targets] -= 1
    d *= dloss.double()[:, None]
    # besides, exponentials of arguments up to 10 are off by 2^-21 and 10 x 2^-24 of themselves: 1.1e-6, and less of norms that the targets' terms make up
    assert off(da, d @ w) < 2e-6 and off(dw, d.T @ a) < 2e-6


# Products of MX9 operands: terms of one sign, the first channels far larger, so that the sum is at its size when most of its terms are added.  Sums are handed
# on every 128 instructions: 128 x 2^-25 = 3.8e-6 at most are lost in them, and 2^-25 of the total with every further addition.  (One chain: 4.4e-6 to 6e-5.)
LOST = 4.1e-6


def one_sign(m, n, k, gen, size=1.0):
    a = torch.rand(m, k, device="cuda", generator=gen) + 0.5
    a[:, :k // 100] *= 64
    return f.packed(bdr.MX9, a), f.packed(bdr.MX9, (torch.rand(n, k, device="cuda", generator=gen) + 0.5) * (size / k))


# many tiles, ragged ones, tiles whose sums are shared out, and few rows
@pytest.mark.parametrize("m,n,k", [(4096, 1024, 8192), (777, 1003, 5000), (130, 70, 16384), (2100, 4700, 4111), (9, 800, 8192)])
def test_products_of_long_sums(m, n, k):
    gen = torch.Generator(device="cuda").manual_seed(33)
    (pa, a), (pw, w) = one_sign(m, 2 * n, k, gen)
    h, gate_up = torch.empty(m, n, device="cuda"), torch.empty(m, 2 * n, device="cuda")
    bdr.mx_gated_gemm(bdr.MX9, pa, bdr.MX9, pw, m, n, k, h, f.workspace(bdr.mx_gated_gemm_workspace_bytes(m, n, k)), act=bdr.ACT_RELU, gate_up=gate_up)
    g = a @ w.T
    assert off(gate_up, g) < LOST and off(h, g[:, :n] * g[:, n:]) < 2 * LOST
    # the gradients' own products: dG = dh u, dU = dh g
    dh = torch.rand(m, n, device="cuda", generator=gen) + 0.5
    da, dw = torch.empty(m, k, device="cuda"), torch.empty(2 * n, k, device="cuda")
    bdr.mx_gated_gemm_bwd(bdr.MX9, pa, bdr.MX9, pw, m, n, k, dh, da, dw, f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k, torch.float32)), act=bdr.ACT_RELU)
    d = torch.cat((dh.double() * g[:, n:], dh.double() * g[:, :n]), 1)
    assert off(da, d @ w) < LOST + 1e-6 and off(dw, d.T @ a) < LOST + 1e-6


@pytest.mark.parametrize("m,v,k", [(1024, 4096, 8192), (777, 3001, 5000), (130, 140, 16384)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits_of_long_sums(m, v, k, dtype):
    gen = torch.Generator(device="cuda").manual_seed(34)
    (pa, a), (pw, w) = one_sign(m, v, k, gen, 16.0)
    logits = a @ w.T
    largest = float(logits.max())
    targets = torch.randint(0, v, (m,), device="cuda", generator=gen)
    loss, lse = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    bdr.mx_cross_entropy(bdr.MX9, pa, bdr.MX9, pw, m, v, k, targets, loss, lse, f.workspace(bdr.mx_cross_entropy_workspace_bytes(m, v, k)))
    want = torch.logsumexp(logits, 1)
    # the logits' own error, and of the logarithm of the sum what fused_helpers.entropy allows
    assert float((lse.double() - want).abs().max()) < LOST * largest + (160 + v / 128) * 2.0 ** -24 + 2.0 ** -22 * float(want.max()) + 2.0 ** -21
    # d beside the lse in 64 bits: exponentials move with the logits
    lse, dloss = want.float(), torch.ones(m, device="cuda")
    da, dw = torch.empty(m, k, device="cuda", dtype=dtype), torch.empty(v, k, device="cuda", dtype=dtype)
    bdr.mx_cross_entropy_bwd(bdr.MX9, pa, bdr.MX9, pw, m, v, k, targets, lse, dloss, da, dw, f.workspace(bdr.mx_cross_entropy_bwd_workspace_bytes(m, v, k, dtype)))
    d = torch.exp(logits - lse.double()[:, None])
    d[torch.arange(m, device="cuda"), targets] -= 1
    each = LOST * largest + 2.0 ** -21 + 2 * f.HALF_STEP[dtype]
    assert off(dw, d.T @ a) < each
