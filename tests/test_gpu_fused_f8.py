"""The gated layer and the cross entropy where MX4 / MX6 operands take the 8-bit tensor-core path, and where they fall back from it."""
import pytest
import torch

import fused_helpers as f
from paper_2302_08007_b200 import binding as bdr

pytestmark = pytest.mark.gpu


def planes(fmt, rows, k, gen, scale, spread):
    x = torch.randn(rows, k, device="cuda", generator=gen) * scale
    if spread:  # neighbouring blocks too far apart for one scale: not representable in eight bits
        x[rows // 2, 16:32] *= 2.0 ** -30
    return f.packed(f.CFG[fmt], x)


@pytest.mark.parametrize("fa,fw", [("mx6", "mx6"), ("mx4", "mx6"), ("mx6", "mx4"), ("mx4", "mx4")])
@pytest.mark.parametrize("spread", [False, True])
def test_gated(fa, fw, spread):
    m, n, k = 2304, 1920, 4096                                   # 2304 x 3840 x 4096 multiplications are enough
    gen = torch.Generator(device="cuda").manual_seed(11)
    pa, a = planes(fa, m, k, gen, 1.0, spread)
    pw, w = planes(fw, 2 * n, k, gen, k ** -0.5, False)
    h, gu = torch.full((m, n), float("nan"), device="cuda"), torch.full((m, 2 * n), float("nan"), device="cuda")
    ws = f.workspace(bdr.mx_gated_gemm_workspace_bytes(m, n, k))
    for _ in range(2):                                           # the flag of a call does not outlive it
        bdr.mx_gated_gemm(f.CFG[fa], pa, f.CFG[fw], pw, m, n, k, h, ws, gate_up=gu)
    want, products, eh, e = f.gated(a, w, n, "silu")
    f.check(gu, products, e + 2.0 ** -24 * products.abs(), "gate_up")
    f.check(h, want, eh + 2.0 ** -24 * want.abs() + 2.0 ** -126, "h")
    dh = torch.randn(m, n, device="cuda", generator=gen).bfloat16()
    da, dw = torch.empty(m, k, device="cuda", dtype=torch.bfloat16), torch.empty(2 * n, k, device="cuda", dtype=torch.bfloat16)
    ws = f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k))
    bdr.mx_gated_gemm_bwd(f.CFG[fa], pa, f.CFG[fw], pw, m, n, k, dh, da, dw, ws)
    want_a, want_w, ea, ew = f.gated_grads(a, w, n, "silu", dh.double(), products, e, torch.bfloat16)
    f.check(da, want_a, ea, "da")
    f.check(dw, want_w, ew, "dw")
    assert bdr.bdr_device_status() == 0


@pytest.mark.parametrize("fa,fw", [("mx6", "mx6"), ("mx4", "mx6")])
@pytest.mark.parametrize("spread", [False, True])
def test_entropy(fa, fw, spread):
    m, v, k = 1024, 16640, 2176
    gen = torch.Generator(device="cuda").manual_seed(12)
    pa, a = planes(fa, m, k, gen, 2.0, spread)
    pw, w = planes(fw, v, k, gen, k ** -0.5, False)
    targets = torch.randint(0, v, (m,), device="cuda", generator=gen)
    targets[::9] = -100
    targets[1] = v - 1
    loss, lse = (torch.full((m,), float("nan"), device="cuda") for _ in range(2))
    ws = f.workspace(bdr.mx_cross_entropy_workspace_bytes(m, v, k))
    for _ in range(2):
        bdr.mx_cross_entropy(f.CFG[fa], pa, f.CFG[fw], pw, m, v, k, targets, loss, lse, ws)
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, else_, "lse")
    f.check(loss, want, eloss, "loss")
    dloss = torch.rand(m, device="cuda", generator=gen)
    da, dw = torch.empty(m, k, device="cuda", dtype=torch.bfloat16), torch.empty(v, k, device="cuda", dtype=torch.bfloat16)
    ws = f.workspace(bdr.mx_cross_entropy_bwd_workspace_bytes(m, v, k))
    bdr.mx_cross_entropy_bwd(f.CFG[fa], pa, f.CFG[fw], pw, m, v, k, targets, lse, dloss, da, dw, ws)
    want_a, want_w, ea, ew = f.entropy_grads(a, w, targets, lse.double(), dloss.double(), torch.bfloat16)
    f.check(da, want_a, ea, "da")
    f.check(dw, want_w, ew, "dw")
    assert bdr.bdr_device_status() == 0


def test_a_block_without_values_poisons_its_own_row():
    m, n, k = 2304, 1920, 4096
    gen = torch.Generator(device="cuda").manual_seed(13)
    pa, a = planes("mx6", m, k, gen, 1.0, False)
    pw, w = planes("mx6", 2 * n, k, gen, k ** -0.5, False)
    pa.exps[1000, 3] = 0xFF
    h = torch.zeros((m, n), device="cuda")
    bdr.mx_gated_gemm(bdr.MX6, pa, bdr.MX6, pw, m, n, k, h, f.workspace(bdr.mx_gated_gemm_workspace_bytes(m, n, k)))
    assert h[1000].isnan().all() and int(h.isnan().sum()) == n
