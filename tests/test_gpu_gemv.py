"""mx_gemv: few-token products with packed weights, against the product in 64 bits of the oracle's dequantized weights.

Tolerance.  Every product of a decoded weight (at most 8 significant bits) and a bf16 activation part (8 bits) is exact.  A
matrix instruction adds 16 products to an fp32 accumulator; its sum is at most a few units of 2^-24 of the largest term off,
2^-22 of the sum of magnitudes covers it.  An element passes through at most K / 16 of them one after the other, then through the
joins of at most eight shares of K and three parts, 16 more additions:  |error| <= (K / 16 + 16) 2^-22 sum |w x|, and half a
unit (2^-9 relative) for a bf16 result."""
import numpy as np
import pytest
import torch

from oracle import oracle as orc
from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import synth
from tests import helpers as H

pytestmark = pytest.mark.gpu

FMT = {"MX4": bdr.MX4, "MX6": bdr.MX6, "MX9": bdr.MX9}


def bf16(a):
    return synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(np.ascontiguousarray(a, dtype=np.float32))).reshape(a.shape)


def check(y, x, w_dq, k, out):
    x64, w64 = x.astype(np.float64), w_dq.astype(np.float64)
    want = x64 @ w64.T
    bound = (k / 16 + 16) * 2.0 ** -22 * (np.abs(x64) @ np.abs(w64).T)
    if out == "bf16":
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
    got = H.device_to_host_f32(y).astype(np.float64)
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= bound + 1e-300)
    assert not bad.any(), (int(bad.sum()), float(np.max(np.abs(got - want)[bad])), float(np.max(bound)))


def make(n, k, t, seed, dtype):
    w = synth.normal_matrix(n, k, seed=seed, stream=2, sigma=k ** -0.5)
    x = synth.outlier_channel_matrix(t, k, seed=seed, stream=1, frac=0.02, gain=20.0)
    return w, bf16(x) if dtype == "bf16" else x


def packed(cfg, w):
    planes = bdr.alloc_planes(cfg, w.shape[0], w.shape[1], 1)
    bdr.bdr_pack(cfg, torch.from_numpy(w).cuda(), planes, axis=1)
    return planes, orc.quant_dequant(H.to_orc(cfg), w, axis=1)[0]


@pytest.mark.parametrize("fmt", list(FMT))
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_products_of_every_format_and_type(fmt, dtype, out):
    cfg = FMT[fmt]
    for n, k, t in ((16, 256, 1), (1, 1, 1), (37, 100, 2), (129, 2063, 3), (64, 4096, 8), (200, 528, 9), (33, 1040, 17), (48, 272, 40)):
        w, x = make(n, k, t, n + k, dtype)
        planes, w_dq = packed(cfg, w)
        y = torch.full((t, n), float("nan"), dtype=torch.bfloat16 if out == "bf16" else torch.float32, device="cuda")
        bdr.mx_gemv(cfg, planes, n, k, H.host_to_device(x, dtype), y)
        check(y, x, w_dq, k, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("t", [1, 5, 8, 16, 21, 22, 32, 64, 65, 130])
def test_every_width_of_a_pass_and_several_passes(t, dtype):
    n, k = 80, 6000                                     # several phases of activations once there are many columns
    w, x = make(n, k, t, t, dtype)
    planes, w_dq = packed(bdr.MX6, w)
    y = torch.empty((t, n), dtype=torch.float32, device="cuda")
    bdr.mx_gemv(bdr.MX6, planes, n, k, H.host_to_device(x, dtype), y)
    check(y, x, w_dq, k, "f32")


@pytest.mark.parametrize("fmt,n,k,t", [("MX9", 19040, 1100, 60), ("MX6", 7110, 2999, 30), ("MX4", 7110, 2999, 20)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rounds_of_tiles_that_go_through_the_phases_again(fmt, n, k, t, dtype):
    w, x = make(n, k, t, 8, dtype)
    planes, w_dq = packed(FMT[fmt], w)
    xd = H.host_to_device(x, dtype)
    shifted = torch.zeros((t, k + 8), dtype=xd.dtype, device="cuda")[:, 1:1 + k]
    shifted.copy_(xd)                                    # not on 16-byte boundaries
    y = torch.empty((t, n), dtype=torch.float32, device="cuda")
    bdr.mx_gemv(FMT[fmt], planes, n, k, shifted, y)
    check(y, x, w_dq, k, "f32")
    again = torch.zeros_like(y)
    aligned = torch.zeros((t, (k + 7) // 8 * 8), dtype=xd.dtype, device="cuda")[:, :k]
    aligned.copy_(xd)
    bdr.mx_gemv(FMT[fmt], planes, n, k, aligned, again)
    assert torch.equal(y, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_and_misaligned_operands(dtype):
    n, k, t = 50, 333, 4
    w, x = make(n, k, t, 3, dtype)
    planes, w_dq = packed(bdr.MX9, w)
    wide = bdr.Planes(*(torch.cat((p, torch.full((n, 32), 0xFF, dtype=torch.uint8, device="cuda")), 1) for p in (planes.exps, planes.micro, planes.elems)))
    xd = H.host_to_device(x, dtype, 344)                 # pitch of whole 16-byte words
    shifted = torch.zeros((t, 351), dtype=xd.dtype, device="cuda")[:, 1:1 + k]
    shifted.copy_(xd)                                    # neither base nor pitch aligned
    buf = torch.full((t, n + 7), -5.0, dtype=torch.float32, device="cuda")
    for src in (xd, shifted):
        for pl in (planes, wide):
            bdr.mx_gemv(bdr.MX9, pl, n, k, src, buf[:, 3:3 + n])
            check(buf[:, 3:3 + n], x, w_dq, k, "f32")
            assert bool((buf[:, :3] == -5).all()) and bool((buf[:, 3 + n:] == -5).all())


def test_the_result_does_not_change_from_run_to_run():
    w, x = make(512, 4096, 3, 9, "bf16")
    planes, _ = packed(bdr.MX4, w)
    xd = H.host_to_device(x, "bf16")
    first = bdr.mx_gemv(bdr.MX4, planes, 512, 4096, xd, torch.empty((3, 512), device="cuda"))
    for _ in range(3):
        assert torch.equal(first, bdr.mx_gemv(bdr.MX4, planes, 512, 4096, xd, torch.empty((3, 512), device="cuda")))


@pytest.mark.parametrize("fmt", list(FMT))
def test_extreme_exponents_zero_blocks_and_nonfinite_values(fmt):
    cfg = FMT[fmt]
    n, k = 24, 512
    w = synth.normal_matrix(n, k, seed=5, stream=2)
    w[0] *= np.float32(1e-37)                            # block exponents down to the bottom of the range
    w[1] = np.float32(2.0 ** 127)                        # block exponent 254
    w[2] = 0
    w[3, 7] = np.inf
    w[4, 500] = np.nan
    w[5, :16] = 0
    x = bf16(synth.normal_matrix(2, k, seed=6, stream=1))
    x[:, :] = np.where(np.arange(k) % 64 == 0, x, x * np.float32(2.0 ** -12))
    x[1] *= np.float32(2.0 ** -20)
    planes, w_dq = packed(cfg, w)
    y = torch.empty((2, n), dtype=torch.float32, device="cuda")
    xd = H.host_to_device(x, "bf16")
    bdr.mx_gemv(cfg, planes, n, k, xd, y)
    got = y.cpu().numpy()
    assert np.isnan(got[:, 3]).all() and np.isnan(got[:, 4]).all()
    rest = [i for i in range(n) if i not in (3, 4)]
    # blocks below 2^-126 count as zero: at most 512 elements of that size times |x| < 8
    w64 = w_dq[rest].astype(np.float64)
    want = x.astype(np.float64) @ w64.T
    bound = (k / 16 + 16) * 2.0 ** -22 * (np.abs(x.astype(np.float64)) @ np.abs(w64).T) + 512 * 8 * 2.0 ** -126
    big = np.abs(want) >= 2.0 ** 127                     # the sum of row 1 may pass the fp32 range
    assert (np.abs(got[:, rest] - want) <= bound)[~big].all()
    assert not got[:, 2].any()
    # activations that are not finite poison their row only
    x[1, 9] = np.inf
    bdr.mx_gemv(cfg, planes, n, k, H.host_to_device(x, "bf16"), y)
    again = y.cpu().numpy()
    assert np.array_equal(again[0], got[0], equal_nan=True) and not np.isfinite(again[1, rest]).any()
    x32 = torch.from_numpy(x).cuda()
    bdr.mx_gemv(cfg, planes, n, k, x32, y)
    assert np.array_equal(y.cpu().numpy()[0], got[0], equal_nan=True) and not np.isfinite(y.cpu().numpy()[1, rest]).any()


def test_zero_sizes_and_another_stream():
    w, x = make(40, 128, 2, 1, "bf16")
    planes, w_dq = packed(bdr.MX6, w)
    y = torch.full((2, 40), 3.0, device="cuda")
    bdr.mx_gemv(bdr.MX6, planes, 40, 0, torch.empty((2, 0), device="cuda"), y)
    assert not y.any()
    bdr.mx_gemv(bdr.MX6, planes, 40, 128, torch.empty((0, 128), device="cuda"), torch.empty((0, 40), device="cuda"))
    xd = H.host_to_device(x, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    bdr.mx_gemv(bdr.MX6, planes, 40, 128, xd, y, stream=side)
    side.synchronize()
    check(y, x, w_dq, 128, "f32")


def test_offsets_beyond_32_bits():
    # 270,000 rows of 16,384 codes are 4.1 GiB: the last rows lie beyond 32-bit byte offsets
    n, k = 270000, 16384
    planes = bdr.Planes(*(torch.zeros((n, b), dtype=torch.uint8, device="cuda") for b in (k // 16, k // 16, k)))
    w, x = make(64, k, 1, 4, "bf16")
    tail, w_dq = packed(bdr.MX9, w)
    for dst, src in zip((planes.exps, planes.micro, planes.elems), (tail.exps, tail.micro, tail.elems)):
        dst[n - 64:] = src
    y = torch.empty((1, n), dtype=torch.float32, device="cuda")
    bdr.mx_gemv(bdr.MX9, planes, n, k, H.host_to_device(x, "bf16"), y)
    check(y[:, n - 64:], x, w_dq, k, "f32")
    assert not y[:, :n - 64].any()
