"""mx_attn_decode: attention of one new token over a paged MX cache, against the formula in 64 bits on the oracle's dequantized
keys and values.

Tolerance.  With w the exact weights, A = sum w |v| and n positions:  a score is a sum of head_dim exact products in fp32
matrix instructions, off by at most ds = |scale| (head_dim / 16 + 16) 2^-22 sum |q k|; the exponent's argument and the approximate
exp2 add 2^-22 (2 + |score - reference|), where |score - reference| <= 2 max |score| + 8, so a weight is relatively off by
dw = 2 ds + 2^-22 (4 + 2 max |score| + 8) to first order (twice, for numerator and sum; the test scores keep it below 0.01).
Rounding the weights costs 2^-8 (bf16 queries; eight significant bits) or 2^-16 (32-bit: two bf16 parts), accumulation and joins (n / 16 + 64) 2^-22:
|error| <= 1.1 A (2 dw + rounding + (n / 16 + 64) 2^-22), plus half a unit of a bf16 result.  The log-sum is off by
1.1 (dw + (n / 16 + 64) 2^-22) + 2^-22 |lse|."""
import numpy as np
import pytest
import torch

from oracle import oracle as orc
from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import synth
from tests import helpers as H

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, fk, fv, lens, n_q, n_kv, d, dtype="bf16", page=16, window=0, seed=0, spread=1.0, spare=3):
        self.fk, self.fv, self.lens, self.n_q, self.n_kv, self.d, self.dtype, self.page, self.window = fk, fv, lens, n_q, n_kv, d, dtype, page, window
        rng = np.random.default_rng(seed + 7)
        need = [-(-n // page) for n in lens]
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(lens), max(1, max(need)) + 1), -1, dtype=np.int32)
        first = 0
        for i, x in enumerate(need):
            self.table[i, :x] = order[first:first + x]
            first += x
        rows = self.n_pages * page
        self.keys = synth.outlier_channel_matrix(rows, n_kv * d, seed=seed + 1, stream=1, frac=0.05, gain=4.0) * np.float32(0.5)
        self.vals = synth.normal_matrix(rows, n_kv * d, seed=seed + 1, stream=2)
        q = synth.normal_matrix(len(lens), n_q * d, seed=seed + 1, stream=3) * np.float32(spread)
        self.q = q if dtype == "f32" else synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(q)).reshape(q.shape)
        self.scale = d ** -0.5
        self.cache = bdr.alloc_kv_cache(fk, fv, self.n_pages, page, n_kv, d)
        for cfg, pl, x in ((fk, self.cache.k, self.keys), (fv, self.cache.v, self.vals)):
            bdr.bdr_pack(cfg, torch.from_numpy(np.ascontiguousarray(x)).cuda(), pl, axis=1)

    def call(self, pad=0, want_lse=True, lens=None, table=None, stream=None):
        B = len(self.lens)
        q = H.host_to_device(self.q, self.dtype, self.n_q * self.d + pad).unflatten(1, (self.n_q, self.d))
        out = torch.full((B, self.n_q * self.d + pad), -7.0, dtype=q.dtype, device="cuda")
        o = out[:, :self.n_q * self.d].unflatten(1, (self.n_q, self.d))
        lse = torch.empty((B, self.n_q), dtype=torch.float32, device="cuda") if want_lse else None
        ws = torch.empty(bdr.mx_attn_decode_workspace_bytes(self.cache, B, self.n_q), dtype=torch.uint8, device="cuda")
        ws.fill_(0xFF)                                           # the workspace needs no preparation
        tab = torch.from_numpy(self.table if table is None else table).cuda()
        ln = torch.tensor(self.lens if lens is None else lens, dtype=torch.int32, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        bdr.mx_attn_decode(self.cache, q, tab, ln, o, ws, scale=self.scale, window=self.window, lse=lse, stream=stream)
        torch.cuda.synchronize()
        if pad:
            assert bool((out[:, self.n_q * self.d:] == -7).all())
        return H.device_to_host_f32(o), lse.cpu().numpy() if want_lse else None

    def slots(self, i):
        n = self.lens[i]
        t = np.arange(max(0, n - self.window) if self.window else 0, n)
        return self.table[i, t // self.page].astype(np.int64) * self.page + t % self.page

    def check(self, got, lse, skip=()):
        G = self.n_q // self.n_kv
        for i, n in enumerate(self.lens):
            if i in skip:
                continue
            at = self.slots(i)
            if len(at) == 0:
                assert not got[i].any() and (lse is None or (lse[i] == -np.inf).all())
                continue
            k = orc.quant_dequant(H.to_orc(self.fk), np.ascontiguousarray(self.keys[at]), axis=1)[0].astype(np.float64).reshape(-1, self.n_kv, self.d)
            v = orc.quant_dequant(H.to_orc(self.fv), np.ascontiguousarray(self.vals[at]), axis=1)[0].astype(np.float64).reshape(-1, self.n_kv, self.d)
            q = self.q[i].astype(np.float64).reshape(self.n_kv, G, self.d)
            s = np.einsum("hgd,thd->hgt", q, k) * self.scale
            mag = np.einsum("hgd,thd->hgt", np.abs(q), np.abs(k)) * self.scale
            top = s.max(-1, keepdims=True)
            w = np.exp(s - top)
            tot = w.sum(-1, keepdims=True)
            w /= tot
            want = np.einsum("hgt,thd->hgd", w, v).reshape(self.n_q, self.d)
            A = np.einsum("hgt,thd->hgd", w, np.abs(v)).reshape(self.n_q, self.d)
            eps = 2.0 ** -22
            ds = (self.d / 16 + 16) * eps * mag.max(-1)
            dw = 2 * ds + eps * (4 + 2 * np.abs(s).max(-1) + 8)
            assert dw.max() < 0.01
            acc = (len(at) / 16 + 64) * eps
            bound = 1.1 * A * (2 * dw.reshape(-1, 1) + (2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -16) + acc)
            if self.dtype == "bf16":
                bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
            err = np.abs(got[i].astype(np.float64) - want)
            assert (err <= bound).all(), (i, n, float(err.max()), float(bound.max()), float((err / bound).max()))
            if lse is not None:
                ref = (top + np.log(tot)).reshape(-1)
                assert (np.abs(lse[i] - ref) <= 1.1 * (dw.reshape(-1) + acc) + eps * np.abs(ref)).all()


FMTS = [(bdr.MX9, bdr.MX9), (bdr.MX6, bdr.MX6), (bdr.MX4, bdr.MX4), (bdr.MX9, bdr.MX4), (bdr.MX4, bdr.MX6), (bdr.MX6, bdr.MX9), (bdr.MX4, bdr.MX9),
        (bdr.MX9, bdr.MX6), (bdr.MX6, bdr.MX4)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fk,fv", FMTS, ids=lambda c: "m%d" % c.m)
def test_every_pair_of_formats(fk, fv, dtype):
    c = Case(fk, fv, [1, 17, 300, 0, 64], 8, 2, 128, dtype)
    got, lse = c.call()
    c.check(got, lse)
    assert bdr.bdr_device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,d", [(1, 1, 16), (4, 4, 32), (3, 3, 48), (16, 2, 64), (5, 5, 64), (14, 2, 64), (20, 4, 80), (12, 4, 112), (16, 16, 128),
                                        (24, 2, 128), (32, 1, 128), (40, 1, 128), (8, 8, 144), (16, 2, 192), (10, 1, 256), (8, 4, 256), (9, 9, 96)])
def test_head_layouts(n_q, n_kv, d, dtype):
    for i, (fk, fv) in enumerate(((bdr.MX9, bdr.MX9), (bdr.MX6, bdr.MX4), (bdr.MX4, bdr.MX6))):
        c = Case(fk, fv, [130, 1, 33], n_q, n_kv, d, dtype, page=(16, 5, 64)[i], seed=i)
        got, lse = c.call(pad=8 * i)
        c.check(got, lse)


@pytest.mark.parametrize("page", [1, 3, 16, 24, 128, 1000])
def test_page_sizes_and_lengths_around_tiles(page):
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 257, 1000]
    for window in (0, 1, 16, 50):
        c = Case(bdr.MX6, bdr.MX9, lens, 8, 2, 64, page=page, window=window)
        got, lse = c.call()
        c.check(got, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ragged_batches_and_long_sequences(dtype):
    rng = np.random.default_rng(5)
    c = Case(bdr.MX6, bdr.MX6, rng.integers(0, 900, 70).tolist(), 8, 2, 128, dtype)
    got, lse = c.call()
    c.check(got, lse)
    c = Case(bdr.MX4, bdr.MX9, [20011, 0, 3, 5000], 4, 1, 128, dtype, page=32)
    got, lse = c.call()
    c.check(got, lse)
    c = Case(bdr.MX9, bdr.MX9, [9000], 8, 8, 64, dtype, page=16, window=4000)
    got, lse = c.call(want_lse=False)
    c.check(got, lse)


def test_scores_that_grow_along_the_sequence():
    # the running reference is raised again and again, and the first positions' weights vanish
    c = Case(bdr.MX9, bdr.MX9, [700, 333], 4, 1, 64, spread=1.0)
    direction = np.sign(c.q[0].reshape(4, 64)[0])
    for i in range(2):
        at = c.slots(i)
        c.keys[at] = (np.linspace(-6, 12, len(at))[:, None] * direction * 0.25 + c.keys[at] * 0.1).astype(np.float32)
    bdr.bdr_pack(c.fk, torch.from_numpy(np.ascontiguousarray(c.keys)).cuda(), c.cache.k, axis=1)
    got, lse = c.call()
    c.check(got, lse)


def test_positions_outside_the_range_are_never_seen():
    c = Case(bdr.MX6, bdr.MX6, [21, 40, 0], 4, 2, 64, window=10)
    want, wl = c.call()
    used = np.concatenate([c.slots(i) for i in range(3)])
    rest = np.setdiff1d(np.arange(c.n_pages * c.page), used)
    for pl in (c.cache.k, c.cache.v):                            # every other line: infinities and NaN
        pl.exps[torch.from_numpy(rest).cuda()] = 255
        pl.micro[torch.from_numpy(rest).cuda()] = 255
        pl.elems[torch.from_numpy(rest).cuda()] = 255
    got, gl = c.call()
    assert np.array_equal(got, want) and np.array_equal(gl, wl)
    # one NaN block within the range: that sequence's heads, no other
    c.cache.v.exps[int(c.slots(1)[3]), 0] = 255
    got, gl = c.call()
    assert np.array_equal(got[0], want[0]) and np.array_equal(gl, wl)
    assert np.isnan(got[1, :2, :16]).all() and not np.isnan(got[1, :2, 16:]).any() and not np.isnan(got[1, 2:]).any()
    c.cache.k.exps[int(c.slots(1)[3]), 0] = 255
    got, gl = c.call()
    assert np.array_equal(got[0], want[0]) and np.isnan(got[1, :2]).all() and np.isnan(gl[1, :2]).all() and not np.isnan(got[1, 2:]).any()
    assert bdr.bdr_device_status() == 0


def test_bad_pages_and_lengths_are_reported():
    c = Case(bdr.MX6, bdr.MX6, [21, 40, 30], 4, 2, 64)
    want, wl = c.call()
    for bad in (-1, c.n_pages, 2 ** 31 - 1):
        table = c.table.copy()
        table[1, 1] = bad
        got, gl = c.call(table=table)
        assert bdr.bdr_device_status_reset() == -5
        assert np.isnan(got[1]).all() and np.isnan(gl[1]).all()
        assert np.array_equal(got[[0, 2]], want[[0, 2]]) and np.array_equal(gl[[0, 2]], wl[[0, 2]])
    got, gl = c.call(lens=[21, 2 ** 31 - 1, 30])
    assert bdr.bdr_device_status_reset() == -5
    assert np.isnan(got[1]).all() and np.array_equal(got[[0, 2]], want[[0, 2]])
    got, gl = c.call(lens=[21, -4, 30])
    assert bdr.bdr_device_status() == 0
    assert not got[1].any() and (gl[1] == -np.inf).all() and np.array_equal(got[[0, 2]], want[[0, 2]])


def test_same_result_every_time_on_every_stream_and_alone_or_in_a_batch():
    c = Case(bdr.MX9, bdr.MX6, [5000, 100, 2500], 8, 2, 128)
    want, wl = c.call()
    for stream in (None, torch.cuda.Stream()):
        got, gl = c.call(stream=stream)
        assert np.array_equal(got, want) and np.array_equal(gl, wl)


def test_joining_two_ranges_by_their_log_sums_gives_the_whole():
    c = Case(bdr.MX9, bdr.MX9, [400], 4, 2, 64, "f32")
    whole, wl = c.call()
    head, hl = c.call(lens=[250])
    c.window = 150
    tail, tl = c.call()
    a, b = np.exp(hl - wl)[..., None], np.exp(tl - wl)[..., None]
    # each part is within 2^-16 + (n / 16 + 64) 2^-22 of its own value and each weight within 2^-18; values are below 6
    assert np.abs(a * head + b * tail - whole).max() <= 6 * 4 * (2.0 ** -16 + 89 * 2.0 ** -22 + 2.0 ** -18)


def test_slots_beyond_32_bit_offsets():
    n_pages, page, n_kv, d = 137500, 16, 16, 128                 # 2,200,000 slots of 2,048 codes
    cache = bdr.alloc_kv_cache(bdr.MX9, bdr.MX9, n_pages, page, n_kv, d)
    small = Case(bdr.MX9, bdr.MX9, [45], 16, n_kv, d)
    want, wl = small.call()
    pages = [n_pages - 1, 3, n_pages - 2]
    for dst, src in ((cache.k, small.cache.k), (cache.v, small.cache.v)):
        for a, b in ((dst.exps, src.exps), (dst.micro, src.micro), (dst.elems, src.elems)):
            for i, p in enumerate(pages):
                a[p * page:(p + 1) * page] = b[int(small.table[0, i]) * page:(int(small.table[0, i]) + 1) * page]
    small.cache = cache
    got, gl = small.call(table=np.array([pages + [-1]], dtype=np.int32))
    assert np.array_equal(got, want) and np.array_equal(gl, wl)


def test_in_a_cuda_graph_with_lengths_that_grow():
    c = Case(bdr.MX6, bdr.MX6, [100, 37], 8, 2, 128)
    full = list(c.lens)
    q = H.host_to_device(c.q, "bf16").unflatten(1, (8, 128))
    out, lse = torch.empty_like(q), torch.empty((2, 8), dtype=torch.float32, device="cuda")
    ws = torch.empty(bdr.mx_attn_decode_workspace_bytes(c.cache, 2, 8), dtype=torch.uint8, device="cuda")
    table, lens = torch.from_numpy(c.table).cuda(), torch.tensor([1, 1], dtype=torch.int32, device="cuda")
    call = lambda: bdr.mx_attn_decode(c.cache, q, table, lens, out, ws, scale=c.scale, lse=lse)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for now in ([1, 1], [50, 20], full, [0, 5]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        c.lens = now
        c.check(H.device_to_host_f32(out), lse.cpu().numpy())
