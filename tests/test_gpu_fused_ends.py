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
