"""mx_kv_append: rotated and quantized keys and values in a paged MX cache.  The rotation is defined in fp32 operations that are
rounded one by one, so everything is compared bit for bit: the cache lines with the oracle's packing of the rotated tensor, the
quantized values with its quantize-dequantize, the rotated queries with the fp32 result (rounded once to the tensor's type)."""
import numpy as np
import pytest
import torch

from oracle import oracle as orc
from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import synth
from tests import helpers as H

pytestmark = pytest.mark.gpu


def rotate(x, cos, sin, interleaved):
    """fp32 numpy, x [T, heads, d], cos / sin [T, rot / 2]."""
    half = cos.shape[1]
    y = x.copy()
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    c, s = cos[:, None, :], sin[:, None, :]
    with np.errstate(invalid="ignore"):
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    assert y.dtype == np.float32
    return y


def table(n_pos, rot):
    ang = np.arange(n_pos)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def to_dtype(a, dtype):
    return synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(a)).reshape(a.shape) if dtype == "bf16" else a


def dev(a, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t.to(torch.bfloat16) if dtype == "bf16" else t).cuda()


def run(fk, fv, t, n_q, n_kv, d, dtype, rot, interleaved, page=16, padding=0, fused=True, kind="normal", seed=0, shift=0):
    rng = np.random.default_rng(seed + t)
    heads = n_q + 2 * n_kv
    x = H.make_input(kind, t, heads * d, dtype, seed=seed + 1).reshape(t, heads, d)
    n_pages = -(-t // page) + 2
    cache = bdr.alloc_kv_cache(fk, fv, n_pages, page, n_kv, d)
    planes = [p for pl in (cache.k, cache.v) for p in (pl.exps, pl.micro, pl.elems)]
    for p in planes:
        p.fill_(0xA5)
    slots = rng.permutation(n_pages * page)[:t]
    slots[rng.permutation(t)[:padding]] = -1
    n_pos = 500
    pos = rng.integers(0, n_pos, t)
    cos, sin = table(n_pos, rot)
    buf = torch.zeros((t, heads * d + 16 + shift), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    view = buf[:, shift:shift + heads * d]
    view.copy_(dev(x.reshape(t, -1), dtype))
    q, k, v = (view[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, n_q), (n_q, n_q + n_kv), (n_q + n_kv, heads)))
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    q_out = torch.empty((t, n_q, d), dtype=q.dtype, device="cuda")
    k_dq, v_dq = (torch.empty((t, n_kv, d), dtype=q.dtype, device="cuda") for _ in range(2))
    kw = dict(positions=torch.from_numpy(pos).cuda(), cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda(), interleaved=interleaved) if rot else {}
    bdr.mx_kv_append(cache, k, v, torch.from_numpy(slots).cuda(), q=q, q_out=q_out, k_dq=k_dq, v_dq=v_dq, **kw)
    torch.cuda.synchronize()
    rotated = rotate(x[:, :n_q + n_kv], cos[pos], sin[pos], interleaved) if rot else x[:, :n_q + n_kv]
    H.assert_bits_equal(H.device_to_host_f32(q_out), to_dtype(rotated[:, :n_q], dtype), "rotated queries")
    for cfg, pl, dq, val, name in ((fk, cache.k, k_dq, rotated[:, n_q:], "keys"), (fv, cache.v, v_dq, x[:, n_q + n_kv:], "values")):
        line = np.ascontiguousarray(val.reshape(t, -1))
        want, _ = orc.quant_dequant(H.to_orc(cfg), line, axis=1)
        got = H.device_to_host_f32(dq).reshape(t, -1)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        H.assert_bits_equal(np.nan_to_num(got), np.nan_to_num(want), name)
        for what, p, w in zip(("exps", "micro", "elems"), H.planes_to_host(pl), orc.pack(H.to_orc(cfg), line, axis=1)):
            full = np.full_like(p, 0xA5)                          # lines of other slots keep what they held
            full[slots[slots >= 0]] = w[slots >= 0]
            assert np.array_equal(p, full), (name, what)
    assert bdr.bdr_device_status() == 0
    return cache


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("fk,fv", [(bdr.MX9, bdr.MX9), (bdr.MX6, bdr.MX4), (bdr.MX4, bdr.MX6)], ids=["99", "64", "46"])
def test_lines_values_and_queries_bit_for_bit(fk, fv, interleaved, dtype):
    for t, n_q, n_kv, d, rot in ((1, 8, 2, 128, 128), (37, 4, 4, 64, 64), (3, 6, 3, 80, 32), (20, 5, 1, 16, 16), (9, 3, 3, 48, 48), (70, 2, 1, 256, 64),
                                 (5, 7, 7, 112, 112), (2, 4, 2, 80, 80), (11, 2, 2, 32, 10), (4, 1, 1, 96, 2), (2100, 2, 1, 32, 32)):
        run(fk, fv, t, n_q, n_kv, d, dtype, rot, interleaved)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padding_page_sizes_strides_and_no_rotation(dtype):
    run(bdr.MX6, bdr.MX6, 33, 4, 2, 64, dtype, 64, False, page=24, padding=9)
    run(bdr.MX9, bdr.MX4, 33, 4, 2, 64, dtype, 0, False, page=1, padding=33)
    run(bdr.MX4, bdr.MX9, 8, 4, 2, 128, dtype, 128, False, page=7, fused=False)
    for shift in (1, 2, 4):                                        # token rows that start off a 16-byte boundary
        run(bdr.MX6, bdr.MX9, 6, 2, 2, 64, dtype, 64, False, shift=shift)
        run(bdr.MX6, bdr.MX9, 6, 2, 2, 64, dtype, 40, True, shift=shift)


@pytest.mark.parametrize("kind", ["edge", "tiny", "huge", "laplace_outliers"])
def test_values_at_the_ends_of_the_range(kind):
    # without the rotation the inputs reach the quantizer as they are (a rotation of huge values overflows, see below)
    run(bdr.MX9, bdr.MX6, 40, 2, 2, 64, "f32", 0, False, kind=kind)
    run(bdr.MX4, bdr.MX9, 40, 2, 2, 64, "bf16", 0, False, kind=kind)
    run(bdr.MX4, bdr.MX9, 40, 2, 2, 64, "f32", 32 if kind != "huge" else 0, True, kind=kind)


def test_only_what_is_asked_for_is_written():
    t, n_kv, d = 5, 2, 64
    x = H.make_input("normal", t, 2 * n_kv * d, "bf16", seed=2).reshape(t, 2 * n_kv, d)
    cache = bdr.alloc_kv_cache(bdr.MX6, bdr.MX6, 1, 16, n_kv, d)
    k, v = dev(x[:, :n_kv], "bf16"), dev(x[:, n_kv:], "bf16")
    bdr.mx_kv_append(cache, k, v, torch.arange(t, device="cuda"))
    for pl, val in ((cache.k, x[:, :n_kv]), (cache.v, x[:, n_kv:])):
        want = orc.pack(orc.MX6, np.ascontiguousarray(val.reshape(t, -1)), axis=1)
        for p, w in zip(H.planes_to_host(pl), want):
            assert np.array_equal(p[:t], w)
    back = torch.empty((t, n_kv * d), dtype=torch.float32, device="cuda")   # the cache is an ordinary packed table
    bdr.bdr_gather_rows(bdr.MX6, cache.k, 16, torch.arange(t, device="cuda"), back)
    H.assert_bits_equal(back.cpu().numpy(), orc.quant_dequant(orc.MX6, np.ascontiguousarray(x[:, :n_kv].reshape(t, -1)), axis=1)[0])


def test_nonfinite_values_mark_their_block():
    t, n_kv, d = 4, 1, 64
    x = H.make_input("normal", t, 2 * d, "f32", seed=8).reshape(t, 2, d)
    x[1, 0, 5], x[2, 1, 20] = np.inf, np.nan
    cache = bdr.alloc_kv_cache(bdr.MX9, bdr.MX9, 1, 4, n_kv, d)
    cos, sin = table(10, 64)
    bdr.mx_kv_append(cache, dev(x[:, :1], "f32"), dev(x[:, 1:], "f32"), torch.arange(t, device="cuda"), torch.arange(t, device="cuda"),
                     torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    ke, ve = cache.k.exps[:, :4].cpu().numpy(), cache.v.exps[:, :4].cpu().numpy()
    # the infinite element and its partner 32 further on are spoilt by the rotation
    assert (ke == 255).tolist() == [[False] * 4, [True, False, True, False], [False] * 4, [False] * 4]
    assert (ve == 255).tolist() == [[False] * 4, [False] * 4, [False, True, False, False], [False] * 4]


def test_bad_slots_and_positions_are_reported_and_store_nothing():
    t, n_kv, d = 4, 2, 32
    x = H.make_input("normal", t, 3 * n_kv * d, "f32", seed=4).reshape(t, 3 * n_kv, d)
    cache = bdr.alloc_kv_cache(bdr.MX6, bdr.MX6, 2, 4, n_kv, d)
    for pl in (cache.k, cache.v):
        for p in (pl.exps, pl.micro, pl.elems):
            p.fill_(0xA5)
    cos, sin = table(6, 32)
    q, k, v = (dev(x[:, i * n_kv:(i + 1) * n_kv], "f32") for i in range(3))
    q_out, k_dq, v_dq = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    assert bdr.bdr_device_status() == 0
    bdr.mx_kv_append(cache, k, v, torch.tensor([8, 1, 2, 3], device="cuda"), torch.tensor([0, 6, -1, 5], device="cuda"),
                     torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), q=q, q_out=q_out, k_dq=k_dq, v_dq=v_dq)
    torch.cuda.synchronize()
    assert bdr.bdr_device_status_reset() == -5
    assert (cache.k.elems.cpu().numpy() != 0xA5).any(1).tolist() == [False, False, False, True] + [False] * 4
    assert torch.isnan(q_out).flatten(1).all(1).tolist() == [False, True, True, False]
    assert torch.isnan(k_dq).flatten(1).all(1).tolist() == [False, True, True, False]
    assert not torch.isnan(v_dq).any()


def test_slots_beyond_32_bit_offsets():
    # 2,200,000 slots of 2,048 codes: the last pages lie beyond 4 GiB
    n_pages, page, n_kv, d, t = 137500, 16, 16, 128, 3
    cache = bdr.alloc_kv_cache(bdr.MX9, bdr.MX4, n_pages, page, n_kv, d)
    x = H.make_input("normal", t, 2 * n_kv * d, "bf16", seed=3).reshape(t, 2 * n_kv, d)
    slots = torch.tensor([n_pages * page - 1, 5, n_pages * page - 17], device="cuda")
    bdr.mx_kv_append(cache, dev(x[:, :n_kv], "bf16"), dev(x[:, n_kv:], "bf16"), slots)
    for cfg, pl, val in ((orc.MX9, cache.k, x[:, :n_kv]), (orc.MX4, cache.v, x[:, n_kv:])):
        for p, w in zip((pl.exps, pl.micro, pl.elems), orc.pack(cfg, np.ascontiguousarray(val.reshape(t, -1)), axis=1)):
            assert np.array_equal(p[slots].cpu().numpy(), w)
