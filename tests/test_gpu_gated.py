"""The gated feed-forward layer on packed operands: forward, gradients and the form for a few tokens, against the formulas in 64 bits."""
import pytest
import torch

import fused_helpers as f
from paper_2302_08007_b200 import binding as bdr

pytestmark = pytest.mark.gpu


def operands(m, n, k, fmt_a="mx6", fmt_w="mx6", seed=0, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    a = torch.randn(m, k, device="cuda", generator=gen) * scale
    w = torch.randn(2 * n, k, device="cuda", generator=gen) * k ** -0.5
    return f.packed(f.CFG[fmt_a], a), f.packed(f.CFG[fmt_w], w), gen


def run_forward(pa, pw, fa, fw, m, n, k, dtype, act, keep=True):
    h = torch.full((m, n), float("nan"), device="cuda", dtype=dtype)
    gu = torch.full((m, 2 * n), float("nan"), device="cuda", dtype=dtype) if keep else None
    ws = f.workspace(bdr.mx_gated_gemm_workspace_bytes(m, n, k))
    bdr.mx_gated_gemm(f.CFG[fa], pa, f.CFG[fw], pw, m, n, k, h, ws, act=f.ACTS[act], gate_up=gu)
    return h, gu


SIZES = [(1, 1, 1), (1, 128, 64), (2, 3, 5), (128, 128, 128), (129, 127, 65), (255, 129, 100), (256, 256, 256), (257, 384, 2048), (300, 250, 1111),
         (1000, 500, 777), (640, 1300, 160)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_forward(m, n, k, dtype):
    (pa, a), (pw, w), _ = operands(m, n, k)
    for act in f.ACTS if m == 300 else ("silu",):
        h, gu = run_forward(pa, pw, "mx6", "mx6", m, n, k, dtype, act)
        want, products, eh, e = f.gated(a, w, n, act)
        f.check(gu, products, e + f.HALF_STEP[dtype] * (products.abs() + e), "gate_up")
        f.check(h, want, eh + f.HALF_STEP[dtype] * (want.abs() + eh) + 2.0 ** -126, "h " + act)


@pytest.mark.parametrize("fa", ["mx4", "mx6", "mx9"])
@pytest.mark.parametrize("fw", ["mx4", "mx6", "mx9"])
def test_formats(fa, fw):
    m, n, k = 200, 136, 336
    (pa, a), (pw, w), gen = operands(m, n, k, fa, fw, 1)
    h, gu = run_forward(pa, pw, fa, fw, m, n, k, torch.float32, "silu")
    want, products, eh, e = f.gated(a, w, n, "silu")
    f.check(gu, products, e + 2.0 ** -24 * products.abs(), "gate_up")
    f.check(h, want, eh + 2.0 ** -24 * want.abs() + 2.0 ** -126, "h")
    again, _ = run_forward(pa, pw, fa, fw, m, n, k, torch.float32, "silu", keep=False)
    assert torch.equal(h, again)


@pytest.mark.parametrize("m,n,k", [(256, 256, 3584), (40, 100, 4001), (33, 20, 8192), (300, 64, 2000), (520, 300, 1500), (1, 31, 640)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_tiles_with_long_sums(m, n, k, dtype):
    # the sums of a tile are shared out to several clusters
    (pa, a), (pw, w), gen = operands(m, n, k, "mx9", "mx6", 8)
    runs = [run_forward(pa, pw, "mx9", "mx6", m, n, k, dtype, "silu") for _ in range(3)]
    want, products, eh, e = f.gated(a, w, n, "silu")
    f.check(runs[0][1], products, e + f.HALF_STEP[dtype] * (products.abs() + e), "gate_up")
    f.check(runs[0][0], want, eh + f.HALF_STEP[dtype] * (want.abs() + eh) + 2.0 ** -126, "h")
    for h, gu in runs[1:]:
        assert torch.equal(h, runs[0][0]) and torch.equal(gu, runs[0][1])
    dh = (torch.randn(m, n, device="cuda", generator=gen) * 1e-2).to(dtype)
    ws = f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k, dtype))
    out = []
    for _ in range(3):
        da, dw = torch.empty(m, k, device="cuda", dtype=dtype), torch.empty(2 * n, k, device="cuda", dtype=dtype)
        bdr.mx_gated_gemm_bwd(bdr.MX9, pa, bdr.MX6, pw, m, n, k, dh, da, dw, ws)
        out.append((da, dw))
    want_a, want_w, ea, ew = f.gated_grads(a, w, n, "silu", dh.double(), products, e, dtype)
    f.check(out[0][0], want_a, ea, "da")
    f.check(out[0][1], want_w, ew, "dw")
    for da, dw in out[1:]:
        assert torch.equal(da, out[0][0]) and torch.equal(dw, out[0][1])


@pytest.mark.parametrize("m,n,k", [(1, 4100, 260), (7, 35001, 33), (24, 2050, 530), (25, 2050, 530), (48, 16401, 1029), (49, 16401, 1029)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_rows(m, n, k, dtype):
    # both sides of the limits up to which the few-token kernel takes the packed rows
    (pa, a), (pw, w), _ = operands(m, n, k, "mx9", "mx4", 9)
    for act in f.ACTS if m == 24 else ("silu",):
        h, gu = run_forward(pa, pw, "mx9", "mx4", m, n, k, dtype, act)
        want, products, eh, e = f.gated(a, w, n, act)
        f.check(gu, products, e + f.HALF_STEP[dtype] * (products.abs() + e), "gate_up")
        f.check(h, want, eh + f.HALF_STEP[dtype] * (want.abs() + eh) + 2.0 ** -126, "h " + act)
        assert torch.equal(run_forward(pa, pw, "mx9", "mx4", m, n, k, dtype, act, keep=False)[0], h)


GRAD_SIZES = [(1, 1, 1), (1, 130, 70), (3, 5, 300), (128, 64, 256), (257, 129, 200), (300, 250, 1111), (700, 300, 264)]


@pytest.mark.parametrize("m,n,k", GRAD_SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("keep", [False, True])
def test_gradients(m, n, k, dtype, keep):
    (pa, a), (pw, w), gen = operands(m, n, k, "mx9", "mx6", 2)
    dh = (torch.randn(m, n, device="cuda", generator=gen) * 1e-2).to(dtype)
    for act in f.ACTS if m == 300 else ("silu",):
        gu = run_forward(pa, pw, "mx9", "mx6", m, n, k, dtype, act)[1] if keep else None
        da, dw = torch.full((m, k), float("nan"), device="cuda", dtype=dtype), torch.full((2 * n, k), float("nan"), device="cuda", dtype=dtype)
        ws = f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k, dtype))
        call = lambda x, y: bdr.mx_gated_gemm_bwd(bdr.MX9, pa, bdr.MX6, pw, m, n, k, dh, x, y, ws, act=f.ACTS[act], gate_up=gu)  # noqa: E731
        call(da, dw)
        if keep:
            products, e = gu.double(), torch.zeros_like(gu, dtype=torch.float64)
        else:
            _, products, _, e = f.gated(a, w, n, act)
        want_a, want_w, ea, ew = f.gated_grads(a, w, n, act, dh.double(), products, e, dtype)
        f.check(da, want_a, ea, "da " + act)
        f.check(dw, want_w, ew, "dw " + act)
        one, other = torch.empty_like(da), torch.empty_like(dw)
        call(one, None)
        call(None, other)
        assert torch.equal(one, da) and torch.equal(other, dw)


def test_gradients_by_differences():
    # a weight and a hidden value one step further in their format, in the formula itself: the kernel's gradient against the difference
    m, n, k = 40, 24, 64
    (pa, a), (pw, w), gen = operands(m, n, k, "mx9", "mx9", 3)
    dh = torch.randn(m, n, device="cuda", generator=gen)
    da, dw = torch.empty(m, k, device="cuda"), torch.empty(2 * n, k, device="cuda")
    bdr.mx_gated_gemm_bwd(bdr.MX9, pa, bdr.MX9, pw, m, n, k, dh, da, dw, f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k, torch.float32)),
                          act=bdr.ACT_GELU)
    loss = lambda a, w: (f.gated(a, w, n, "gelu")[0] * dh.double()).sum()  # noqa: E731
    step = 2.0 ** -12
    for i, j in ((0, 0), (7, 63), (23, 5), (24, 1), (47, 30)):
        e = torch.zeros_like(w)
        e[i, j] = step
        # the formula's third derivative times step^2 / 6, below 1e-6 here, and fp32's own
        assert abs(float((loss(a, w + e) - loss(a, w - e)) / (2 * step) - dw[i, j])) < 1e-4
    for i, j in ((0, 0), (39, 63), (11, 17)):
        e = torch.zeros_like(a)
        e[i, j] = step
        assert abs(float((loss(a + e, w) - loss(a - e, w)) / (2 * step) - da[i, j])) < 1e-4


def test_strides_and_surroundings():
    m, n, k = 133, 70, 90
    (pa, a), (pw, w), gen = operands(m, n, k, "mx6", "mx4", 4)
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.full((m + 2, n + 5), 7.0, device="cuda", dtype=dtype)
        kept = torch.full((m + 2, 2 * n + 3), 7.0, device="cuda", dtype=dtype)
        ws = f.workspace(bdr.mx_gated_gemm_workspace_bytes(m, n, k))
        bdr.mx_gated_gemm(bdr.MX6, pa, bdr.MX4, pw, m, n, k, wide[1:-1, 3:3 + n], ws, gate_up=kept[1:-1, 1:1 + 2 * n])
        h, gu = run_forward(pa, pw, "mx6", "mx4", m, n, k, dtype, "silu")
        assert torch.equal(wide[1:-1, 3:3 + n], h) and torch.equal(kept[1:-1, 1:1 + 2 * n], gu)
        wide[1:-1, 3:3 + n] = 7.0
        kept[1:-1, 1:1 + 2 * n] = 7.0
        assert (wide == 7).all() and (kept == 7).all()
        dh = torch.randn(m, n + 1, device="cuda", generator=gen).to(dtype)
        da, dw = torch.full((m + 2, k + 9), 7.0, device="cuda", dtype=dtype), torch.full((2 * n + 2, k + 1), 7.0, device="cuda", dtype=dtype)
        ws = f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k, dtype))
        for x, y, g, s in ((da[1:-1, 4:4 + k], dw[1:-1, 1:], kept[1:-1, 1:1 + 2 * n], dh[:, 1:]), (torch.empty(m, k, device="cuda", dtype=dtype), torch.empty(2 * n, k, device="cuda", dtype=dtype), gu, dh[:, 1:].contiguous())):
            g.copy_(gu)
            bdr.mx_gated_gemm_bwd(bdr.MX6, pa, bdr.MX4, pw, m, n, k, s, x, y, ws, gate_up=g)
        assert torch.equal(da[1:-1, 4:4 + k], x) and torch.equal(dw[1:-1, 1:], y)
        da[1:-1, 4:4 + k] = 7.0
        dw[1:-1, 1:] = 7.0
        assert (da == 7).all() and (dw == 7).all()


def test_padding_of_planes_is_not_used():
    # pitches of lines of K elements leave bytes behind the last block: whatever they hold, results are the same
    for fmt in ("mx4", "mx6", "mx9"):
        m, n, k = 40, 24, 16 * 5
        (pa, a), (pw, w), gen = operands(m, n, k, fmt, fmt, 5)
        first, _ = run_forward(pa, pw, fmt, fmt, m, n, k, torch.float32, "silu")
        for p in (pa, pw):
            p.exps[:, 5:] = 0xFF
            p.micro[:, 5:] = 0xFF
            p.elems[:, 5 * 2 * (f.CFG[fmt].m + 1):] = 0xFF
        second, _ = run_forward(pa, pw, fmt, fmt, m, n, k, torch.float32, "silu")
        assert torch.equal(first, second)
        dh = torch.ones(m, n, device="cuda")
        da, dw = torch.empty(m, k, device="cuda"), torch.empty(2 * n, k, device="cuda")
        bdr.mx_gated_gemm_bwd(f.CFG[fmt], pa, f.CFG[fmt], pw, m, n, k, dh, da, dw, f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k, torch.float32)))
        assert da.isfinite().all() and dw.isfinite().all()


def test_blocks_without_values_poison_their_own_rows():
    m, n, k = 150, 140, 64
    (pa, a), (pw, w), _ = operands(m, n, k, seed=6)
    pa.exps[3, 1] = 0xFF
    pw.exps[n + 7, 0] = 0xFF
    h, _ = run_forward(pa, pw, "mx6", "mx6", m, n, k, torch.float32, "silu")
    bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    bad[3] = True
    bad[:, 7] = True
    assert torch.equal(h.isnan(), bad)


@pytest.mark.parametrize("act", list(f.ACTS))
def test_large_arguments(act):
    # gates far out on both sides: the activation is its limit, not NaN
    m, n, k = 4, 6, 16
    a, w = torch.zeros(m, k, device="cuda"), torch.zeros(2 * n, k, device="cuda")
    a[:, 0] = 1.0
    w[:n, 0] = torch.tensor([2.0 ** 10, -2.0 ** 10, 2.0 ** 60, -2.0 ** 60, 100.0, -100.0], device="cuda")
    w[n:, 0] = 1.0
    (pa, a), (pw, w) = f.packed(bdr.MX9, a), f.packed(bdr.MX9, w)
    h, _ = run_forward(pa, pw, "mx9", "mx9", m, n, k, torch.float32, act)
    want, _, _, _ = f.gated(a, w, n, act)
    f.check(h, want, 2.0 ** -20 * want.abs() + 2.0 ** -120, act)
    dh = torch.ones(m, n, device="cuda")
    da, dw = torch.empty(m, k, device="cuda"), torch.empty(2 * n, k, device="cuda")
    bdr.mx_gated_gemm_bwd(bdr.MX9, pa, bdr.MX9, pw, m, n, k, dh, da, dw, f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k, torch.float32)), act=f.ACTS[act])
    assert da.isfinite().all() and dw.isfinite().all()


def test_nothing_to_do():
    (pa, _), (pw, _), _ = operands(4, 4, 32)
    ws = f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(4, 4, 32, torch.float32))
    new = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731
    bdr.mx_gated_gemm(bdr.MX6, pa, bdr.MX6, pw, 0, 4, 32, new(0, 4), ws)
    bdr.mx_gated_gemm(bdr.MX6, pa, bdr.MX6, pw, 4, 0, 32, new(4, 0), ws)
    dw = new(8, 32)
    bdr.mx_gated_gemm_bwd(bdr.MX6, pa, bdr.MX6, pw, 0, 4, 32, new(0, 4), new(0, 32), dw, ws)
    assert (dw == 0).all()
    da = new(4, 40)
    bdr.mx_gated_gemm_bwd(bdr.MX6, pa, bdr.MX6, pw, 4, 0, 32, new(4, 0), da[:, :32], new(0, 32), ws)
    assert (da[:, :32] == 0).all() and (da[:, 32:] == 7).all()


def test_captured_and_replayed():
    m, n, k = 260, 140, 200
    (pa, a), (pw, w), gen = operands(m, n, k, seed=7)
    h, gu = run_forward(pa, pw, "mx6", "mx6", m, n, k, torch.bfloat16, "silu")
    dh = torch.randn(m, n, device="cuda", generator=gen).bfloat16()
    ws = f.workspace(bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k))
    da, dw = torch.empty(m, k, device="cuda", dtype=torch.bfloat16), torch.empty(2 * n, k, device="cuda", dtype=torch.bfloat16)

    def both(h, gu, da, dw):
        bdr.mx_gated_gemm(bdr.MX6, pa, bdr.MX6, pw, m, n, k, h, ws, gate_up=gu)
        bdr.mx_gated_gemm_bwd(bdr.MX6, pa, bdr.MX6, pw, m, n, k, dh, da, dw, ws, gate_up=gu)

    both(h, gu, da, dw)
    out = [torch.empty_like(t) for t in (h, gu, da, dw)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both(*out)
    for _ in range(3):
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for t, want in zip(out, (h, gu, da, dw)):
            assert torch.equal(t, want)
    assert bdr.bdr_device_status() == 0


# ---- a few tokens ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["mx4", "mx6", "mx9"])
@pytest.mark.parametrize("t,n,k", [(1, 1, 1), (1, 7, 16), (1, 8, 256), (2, 9, 300), (3, 1000, 4100), (8, 130, 2063), (9, 2400, 512), (16, 500, 5000), (17, 64, 1024),
                                   (33, 100, 700), (64, 31, 272), (65, 40, 100)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_tokens(fmt, t, n, k, dtype):
    gen = torch.Generator(device="cuda").manual_seed(t * 1000 + n)
    pw, w = f.packed(f.CFG[fmt], torch.randn(2 * n, k, device="cuda", generator=gen) * k ** -0.5)
    x = torch.randn(t, k, device="cuda", generator=gen).to(dtype)
    for act in f.ACTS if t == 3 else ("silu",):
        h = bdr.mx_gated_gemv(f.CFG[fmt], pw, n, k, x, torch.full((t, n), float("nan"), device="cuda", dtype=dtype), act=f.ACTS[act])
        want, _, eh, _ = f.gated(x.double(), w, n, act)
        f.check(h, want, eh + f.HALF_STEP[dtype] * (want.abs() + eh) + 2.0 ** -126, act)


def test_few_tokens_strides_types_and_surroundings():
    t, n, k = 5, 37, 200
    gen = torch.Generator(device="cuda").manual_seed(9)
    pw, w = f.packed(bdr.MX6, torch.randn(2 * n, k, device="cuda", generator=gen))
    x = torch.randn(t, k + 3, device="cuda", generator=gen).bfloat16()[:, 1:1 + k]
    for out in (torch.float32, torch.bfloat16):
        wide = torch.full((t + 2, n + 5), 7.0, device="cuda", dtype=out)
        bdr.mx_gated_gemv(bdr.MX6, pw, n, k, x, wide[1:-1, 2:2 + n])
        want, _, eh, _ = f.gated(x.double(), w, n, "silu")
        f.check(wide[1:-1, 2:2 + n], want, eh + f.HALF_STEP[out] * (want.abs() + eh), "h")
        wide[1:-1, 2:2 + n] = 7.0
        assert (wide == 7).all()
    h = bdr.mx_gated_gemv(bdr.MX6, pw, n, 0, x[:, :0], torch.full((t, n), 7.0, device="cuda"))
    assert (h == 0).all()                                         # act(0) * 0
