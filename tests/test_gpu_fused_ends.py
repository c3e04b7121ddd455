"""The gated layer and the cross entropy at the ends of what they accept: no tokens, rows that do not count, confident rows."""
import pytest
import torch

import fused_helpers as f
from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import head

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_tokens_with_workspaces_of_their_own(dtype):
    n, k = 40, 64
    pa, pw = bdr.alloc_planes(bdr.MX6, 0, k), f.packed(bdr.MX6, torch.randn(2 * n, k, device="cuda"))[0]
    new = lambda *s, dt=dtype: torch.full(s, 7.0, device="cuda", dtype=dt)  # noqa: E731
    h = new(0, n)
    bdr.mx_gated_gemm(bdr.MX6, pa, bdr.MX6, pw, 0, n, k, h, f.workspace(bdr.mx_gated_gemm_workspace_bytes(0, n, k)))
    dw = new(2 * n, k)
    bdr.mx_gated_gemm_bwd(bdr.MX6, pa, bdr.MX6, pw, 0, n, k, h, new(0, k), dw, f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(0, n, k, dtype)))
    assert (dw == 0).all()
    px, none = f.packed(bdr.MX6, torch.randn(5, k, device="cuda"))[0], bdr.alloc_planes(bdr.MX6, 0, k)
    bdr.mx_gated_gemm(bdr.MX6, px, bdr.MX6, none, 5, 0, k, new(5, 0), f.workspace(bdr.mx_gated_gemm_workspace_bytes(5, 0, k)))
    da = new(5, k)
    bdr.mx_gated_gemm_bwd(bdr.MX6, px, bdr.MX6, none, 5, 0, k, new(5, 0), da, new(0, k), f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(5, 0, k, dtype)))
    assert (da == 0).all()

    buf = head.alloc(bdr.MX6, 0, 2 * n, k, dtype=dtype)
    targets = torch.empty(0, dtype=torch.int64, device="cuda")
    loss = head.losses(torch.empty(0, k, device="cuda"), torch.randn(2 * n, k, device="cuda"), targets, buf)
    buf.d_weight.fill_(7.0)
    d_hidden, d_weight = head.gradients(targets, torch.empty(0, device="cuda"), buf)
    assert loss.shape == (0,) and d_hidden.shape == (0, k) and (d_weight == 0).all()


# rows decoded by either kernel, one and several pieces of the vocabulary, sums of few tiles cut or not, and the 8-bit path (which falls back)
@pytest.mark.parametrize("m,v,k,fmt", [(40, 300, 64, "mx6"), (33, 60, 8192, "mx9"), (300, 1000, 1111, "mx4"), (4100, 500, 2048, "mx9"), (4000, 34567, 96, "mx6"),
                                       (1024, 16640, 2176, "mx6")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_do_not_count_hold_no_values(m, v, k, fmt, dtype):
    gen = torch.Generator(device="cuda").manual_seed(21)
    (pa, a), (pw, w) = (f.packed(f.CFG[fmt], torch.randn(r, k, device="cuda", generator=gen) * s) for r, s in ((m, 1.0), (v, k ** -0.5)))
    targets = torch.randint(0, v, (m,), device="cuda", generator=gen)
    out = torch.zeros(m, dtype=torch.bool, device="cuda")
    out[torch.tensor([0, 7, m // 2, m - 1], device="cuda")] = True
    targets[out] = torch.tensor([-100, v, -1, 2 ** 40], device="cuda")
    pa.exps[out] = 0xFF
    loss, lse = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    bdr.mx_cross_entropy(f.CFG[fmt], pa, f.CFG[fmt], pw, m, v, k, targets, loss, lse, f.workspace(bdr.mx_cross_entropy_workspace_bytes(m, v, k)))
    assert torch.equal(lse.isnan(), out) and (loss[targets < 0] == 0).all()
    assert bdr.bdr_device_status_reset() == -5
    dloss = torch.rand(m, device="cuda", generator=gen)
    dloss[out] = float("nan")

    def grads():
        da, dw = torch.full((m, k), float("nan"), device="cuda", dtype=dtype), torch.full((v, k), float("nan"), device="cuda", dtype=dtype)
        ws = f.workspace(bdr.mx_cross_entropy_bwd_workspace_bytes(m, v, k, dtype))
        bdr.mx_cross_entropy_bwd(f.CFG[fmt], pa, f.CFG[fmt], pw, m, v, k, targets, lse, dloss, da, dw, ws)
        return da, dw

    da, dw = grads()
    a[out] = 0.0
    clean = torch.where(out, 0.0, lse.double())
    want_a, want_w, ea, ew = f.entropy_grads(a, w, targets, clean, torch.where(out, 0.0, dloss.double()), dtype)
    f.check(da, want_a, ea, "da")
    f.check(dw, want_w, ew, "dw")
    assert (da[out] == 0).all()
    # a line of the weights without values leaves its own in every row that counts, in no other
    pw.exps[v - 1, 0] = 0xFF
    da, _ = grads()
    assert (da[out] == 0).all() and da[~out][:, :16].isnan().all()
    assert bdr.bdr_device_status() == 0


# the two kernels that join a row's parts; many rows, few of a short vocabulary, few of a long one
@pytest.mark.parametrize("m,v,below", [(200, 300, 13), (3, 300, 13), (200, 36069, 18), (3, 36069, 18)])
def test_small_losses_beside_large_logits(m, v, below):
    # logits 1024 (the target's) and 1024 - below, exact in every step; the log of their sum lies half way between two fp32 numbers, 6e-5 from each
    k = 64
    a, w = torch.zeros(m, k, device="cuda"), torch.zeros(v, k, device="cuda")
    a[:, 0], a[:, 16] = 1024.0, -1.0
    w[:, 0], w[:, 16] = 1.0, float(below)
    w[v // 2, 16] = 0.0
    (pa, a), (pw, w) = f.packed(bdr.MX9, a), f.packed(bdr.MX9, w)
    logits = a @ w.T
    assert (logits == 1024).sum() == m and (logits == 1024 - below).sum() == m * (v - 1)
    targets = torch.full((m,), v // 2, device="cuda", dtype=torch.int64)
    loss, lse = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    bdr.mx_cross_entropy(bdr.MX9, pa, bdr.MX9, pw, m, v, k, targets, loss, lse, f.workspace(bdr.mx_cross_entropy_workspace_bytes(m, v, k)))
    want = torch.log1p((v - 1) * torch.exp(torch.tensor(-float(below), dtype=torch.float64, device="cuda"))).expand(m)
    # a sum just above 1: what its additions round off, as in fused_helpers.entropy, exponentials within 2^-21 of themselves, and the logarithm
    f.check(loss, want, (160 + v / 128) * 2.0 ** -24 + 2.0 ** -20 * want, "loss")
    f.check(lse, 1024 + want, 2.0 ** -23 * (1024 + want), "lse")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_columns_decoded_beside_a_product(dtype):
    # a vocabulary of long lines that is decoded in four parts; the last part is ragged
    m, v, k = 2100, 18100, 4100
    gen = torch.Generator(device="cuda").manual_seed(22)
    (pa, a), (pw, w) = f.packed(bdr.MX9, torch.randn(m, k, device="cuda", generator=gen)), f.packed(bdr.MX6, torch.randn(v, k, device="cuda", generator=gen) * k ** -0.5)
    targets = torch.randint(0, v, (m,), device="cuda", generator=gen)
    targets[:5] = torch.tensor([0, v - 1, 4608, 9215, -100], device="cuda")
    dloss = torch.full((m,), 1.0 / m, device="cuda")
    runs = []
    for _ in range(2):
        loss, lse = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
        bdr.mx_cross_entropy(bdr.MX9, pa, bdr.MX6, pw, m, v, k, targets, loss, lse, f.workspace(bdr.mx_cross_entropy_workspace_bytes(m, v, k)))
        da, dw = torch.empty(m, k, device="cuda", dtype=dtype), torch.empty(v, k, device="cuda", dtype=dtype)
        ws = f.workspace(bdr.mx_cross_entropy_bwd_workspace_bytes(m, v, k, dtype))
        bdr.mx_cross_entropy_bwd(bdr.MX9, pa, bdr.MX6, pw, m, v, k, targets, lse, dloss, da, dw, ws)
        runs.append((loss, lse, da, dw))
    assert all(torch.equal(x, y) for x, y in zip(*runs))
    loss, lse, da, dw = runs[0]
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, else_, "lse")
    f.check(loss, want, eloss, "loss")
    want_a, want_w, ea, ew = f.entropy_grads(a, w, targets, lse.double(), dloss.double(), dtype)
    f.check(da, want_a, ea, "da")
    f.check(dw, want_w, ew, "dw")
