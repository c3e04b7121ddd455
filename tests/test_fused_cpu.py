"""Refusals of the gated layer and the cross entropy, and their workspace sizes: no GPU is used."""
import ctypes as C

import pytest
import torch

from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import decode, ffn

OK, NULL, BAD, UNSUPPORTED, MISALIGNED, SIZE, WORKSPACE = 0, -1, -2, -3, -4, -5, -6
MX6 = bdr.MX6.c()
M, N, K = 40, 24, 64
HUGE = 1 << 50


def planes(ld=(16, 16, 48), at=4096):
    return bdr._Planes(at, at, at, *ld)


def call(fn, order, **change):
    """Calls `fn` with valid arguments but for the changed ones; addresses are never dereferenced, since the changes are refused."""
    args = dict(cfg_a=C.addressof(MX6), a=C.addressof(GOOD), cfg_w=C.addressof(MX6), w=C.addressof(GOOD), M=M, N=N, K=K, act=0, h=4096, dt=1, ldh=64, gu=None,
                ldgu=0, da=4096, lda=64, dw=4096, ldw=64, targets=4096, loss=4096, lse=4096, dloss=4096, ws=4096, bytes=HUGE, stream=None)
    args.update(change)
    return fn(*(args[k] for k in order.split()))


GOOD = planes()
GATED = "cfg_a a cfg_w w M N K act h dt ldh gu ldgu ws bytes stream"
GATED_BWD = "cfg_a a cfg_w w M N K act h dt ldh gu ldgu da lda dw ldw ws bytes stream"
ENTROPY = "cfg_a a cfg_w w M N K targets loss lse ws bytes stream"
ENTROPY_BWD = "cfg_a a cfg_w w M N K targets lse dloss da lda dw ldw dt ws bytes stream"


def all_calls():
    L = bdr.lib()
    return ((L.mx_gated_gemm, GATED), (L.mx_gated_gemm_bwd, GATED_BWD), (L.mx_cross_entropy, ENTROPY), (L.mx_cross_entropy_bwd, ENTROPY_BWD))


def test_operands_are_checked():
    bad, bfp, narrow, odd, low = bdr.Config(16, 8, 3, 1, 4).c(), bdr.Config(16, 8, 2, 0, 4).c(), planes(ld=(16, 16, 32)), planes(at=4104), planes(ld=(8, 16, 48))
    short = planes(ld=(0, 16, 48))                               # (named: the addresses have to stay valid)
    for fn, order in all_calls():
        for side in "aw":
            assert call(fn, order, **{"cfg_" + side: None}) == NULL
            assert call(fn, order, **{"cfg_" + side: C.addressof(bad)}) == BAD
            assert call(fn, order, **{"cfg_" + side: C.addressof(bfp)}) == UNSUPPORTED
            assert call(fn, order, **{side: None}) == NULL
            assert call(fn, order, **{side: C.addressof(narrow)}) == SIZE
            assert call(fn, order, **{side: C.addressof(odd)}) == MISALIGNED
            assert call(fn, order, **{side: C.addressof(low)}) == MISALIGNED
            assert call(fn, order, **{side: C.addressof(short)}) == SIZE
        assert call(fn, order, M=-1) == SIZE and call(fn, order, N=-1) == SIZE and call(fn, order, K=-1) == SIZE
        assert call(fn, order, M=1 << 31) == SIZE and call(fn, order, N=1 << 31) == SIZE and call(fn, order, K=1 << 31) == SIZE
        assert call(fn, order, K=0) == UNSUPPORTED
        assert call(fn, order, ws=None) == WORKSPACE and call(fn, order, ws=4096 + 128) == MISALIGNED


def test_sizes_of_the_workspaces_are_demanded():
    L = bdr.lib()
    sizes = {"mx_gated_gemm": L.mx_gated_gemm_workspace_bytes(M, N, K), "mx_gated_gemm_bwd": L.mx_gated_gemm_bwd_workspace_bytes(M, N, K, 1),
             "mx_cross_entropy": L.mx_cross_entropy_workspace_bytes(M, N, K), "mx_cross_entropy_bwd": L.mx_cross_entropy_bwd_workspace_bytes(M, N, K, 1)}
    for fn, order in all_calls():
        assert sizes[fn.__name__] > 0 and call(fn, order, bytes=sizes[fn.__name__] - 1) == WORKSPACE
    assert L.mx_gated_gemm_bwd_workspace_bytes(M, N, K, 0) > sizes["mx_gated_gemm_bwd"]      # 32-bit gradients: three parts
    for bad in ((-1, N, K), (M, -1, K), (M, N, -1), (1 << 40, N, K)):
        assert L.mx_gated_gemm_workspace_bytes(*bad) == 0 and L.mx_gated_gemm_bwd_workspace_bytes(*bad, 1) == 0
        assert L.mx_cross_entropy_workspace_bytes(*bad) == 0 and L.mx_cross_entropy_bwd_workspace_bytes(*bad, 1) == 0
    assert L.mx_cross_entropy_workspace_bytes(M, 0, K) == 0
    most = 1 << 28                                               # the largest sizes: nothing overflows
    for size in (L.mx_gated_gemm_workspace_bytes(most, most, most), L.mx_gated_gemm_bwd_workspace_bytes(most, most, most, 0),
                 L.mx_cross_entropy_workspace_bytes(most, most, most), L.mx_cross_entropy_bwd_workspace_bytes(most, most, most, 0)):
        assert size > most * most * 2
    assert L.mx_gated_gemm_workspace_bytes(most + 1, 1, 1) == 0 and L.mx_cross_entropy_workspace_bytes(1, most + 1, 1) == 0


def test_tensors_are_checked():
    L = bdr.lib()
    for fn, order in all_calls()[:2]:
        assert call(fn, order, act=4) == UNSUPPORTED and call(fn, order, act=-1) == UNSUPPORTED
        assert call(fn, order, dt=2) == UNSUPPORTED
        assert call(fn, order, h=None) == NULL and call(fn, order, h=4097) == MISALIGNED and call(fn, order, ldh=N - 1) == SIZE
        assert call(fn, order, dt=0, h=4098) == MISALIGNED
        assert call(fn, order, gu=4096, ldgu=2 * N - 1) == SIZE and call(fn, order, gu=4097, ldgu=2 * N) == MISALIGNED
    for fn, order in all_calls()[1::2]:
        assert call(fn, order, lda=K - 1) == SIZE and call(fn, order, ldw=K - 1) == SIZE
        assert call(fn, order, da=4097) == MISALIGNED and call(fn, order, dw=4097) == MISALIGNED
    assert call(L.mx_cross_entropy_bwd, ENTROPY_BWD, dt=2) == UNSUPPORTED
    for fn, order in all_calls()[2:]:
        assert call(fn, order, N=0) == SIZE
        for name in order.split():
            if name in ("targets", "loss", "lse", "dloss"):
                assert call(fn, order, **{name: None}) == NULL
                assert call(fn, order, **{name: 4098}) == MISALIGNED
        assert call(fn, order, targets=4100) == MISALIGNED


def test_nothing_is_wanted_or_there():
    L = bdr.lib()
    assert call(L.mx_gated_gemm, GATED, M=0, a=None, w=None, h=None, ws=None) == OK
    assert call(L.mx_gated_gemm, GATED, N=0, a=None, w=None, h=None, ws=None) == OK
    assert call(L.mx_gated_gemm_bwd, GATED_BWD, da=None, dw=None, h=None, ws=None) == OK
    assert call(L.mx_gated_gemm_bwd, GATED_BWD, M=0, dw=None, h=None, ws=None) == OK
    assert call(L.mx_cross_entropy, ENTROPY, M=0, a=None, w=None, loss=None, ws=None) == OK
    assert call(L.mx_cross_entropy_bwd, ENTROPY_BWD, da=None, dw=None, loss=None, ws=None) == OK
    assert call(L.mx_cross_entropy_bwd, ENTROPY_BWD, M=0, dw=None, ws=None) == OK


def test_few_tokens_are_checked():
    L = bdr.lib()
    order = "cfg_w w N K h dt ldh M act da dt lda stream"
    assert call(L.mx_gated_gemv, order, act=7) == UNSUPPORTED
    narrow = planes(ld=(16, 16, 32))
    assert call(L.mx_gated_gemv, order, w=C.addressof(narrow)) == SIZE
    assert call(L.mx_gated_gemv, order, h=None) == NULL and call(L.mx_gated_gemv, order, da=None) == NULL
    assert call(L.mx_gated_gemv, order, lda=N - 1) == SIZE and call(L.mx_gated_gemv, order, ldh=K - 1) == SIZE
    assert call(L.mx_gated_gemv, order, M=0) == OK


def test_the_binding_refuses_what_does_not_fit():
    cpu = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    a, w = (bdr.alloc_planes(bdr.MX6, r, K, device="cpu") for r in (M, 2 * N))
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    ok = (bdr.MX6, a, bdr.MX6, w, M, N, K)
    with pytest.raises(ValueError, match="fewer"):
        bdr._operand(a, 2 * N, "w", -1)
    with pytest.raises(ValueError, match="CUDA"):
        bdr.mx_gated_gemm(*ok, cpu(M, N), ws)
    with pytest.raises(ValueError, match="CUDA"):
        bdr.mx_cross_entropy(bdr.MX6, a, bdr.MX6, w, M, N, K, cpu(M, dt=torch.int64), cpu(M, dt=torch.float32), cpu(M, dt=torch.float32), ws)
    with pytest.raises(ValueError):
        bdr.mx_gated_gemv(bdr.MX6, w, N + 1, K, cpu(2, K), cpu(2, N + 1))
    with pytest.raises(ValueError, match="CUDA"):
        bdr.mx_gated_gemv(bdr.MX6, w, N, K, cpu(2, K), cpu(2, N))
    # what _matrix and _vector look at, with a device that the tensors are on
    assert bdr._matrix(cpu(M, 2 * N)[:, :N], M, N, torch.bfloat16, "h", -1) == 2 * N
    assert bdr._matrix(cpu(1, N).expand(1, N), 1, N, torch.bfloat16, "h", -1) == N
    for bad in (cpu(N, M).T, cpu(1, N).expand(M, N), cpu(M, N + 1), cpu(M, N, dt=torch.float16)):
        with pytest.raises(ValueError):
            bdr._matrix(bad, M, N, torch.bfloat16, "h", -1)
    for bad in (cpu(M, dt=torch.int32), cpu(M + 1, dt=torch.int64), cpu(2 * M, dt=torch.int64)[::2]):
        with pytest.raises(ValueError):
            bdr._vector(bad, M, torch.int64, "targets", -1)
    with pytest.raises(ValueError):
        bdr._scratch(ws[::2], -1)


def test_modules_refuse_sizes():
    with pytest.raises(ValueError):
        ffn.alloc(bdr.MX6, 100, 256, 256, device="cpu")
    with pytest.raises(ValueError):
        ffn.alloc(bdr.MX6, 256, 256, 0, device="cpu")
    with pytest.raises(ValueError):
        decode.alloc_feed_forward(bdr.MX6, torch.zeros(60, 32), torch.zeros(32, 40), 2)
