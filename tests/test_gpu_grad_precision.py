"""32-bit gradients keep 32 bits: the norm of their error beside that of the gradient.  Two things are there for it, each of which a bound on every single
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
