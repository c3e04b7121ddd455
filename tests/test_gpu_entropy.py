"""Cross entropy over a packed vocabulary without the logits: loss, lse and gradients against the formulas in 64 bits."""
import pytest
import torch

import fused_helpers as f
from paper_2302_08007_b200 import binding as bdr

pytestmark = pytest.mark.gpu


def operands(m, v, k, fa="mx6", fw="mx6", seed=0, scale=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    a = torch.randn(m, k, device="cuda", generator=gen) * scale
    w = torch.randn(v, k, device="cuda", generator=gen) * k ** -0.5
    targets = torch.randint(0, v, (m,), device="cuda", generator=gen)
    return f.packed(f.CFG[fa], a), f.packed(f.CFG[fw], w), targets, gen


def run(pa, pw, fa, fw, m, v, k, targets):
    loss, lse = (torch.full((m,), float("nan"), device="cuda") for _ in range(2))
    ws = f.workspace(bdr.mx_cross_entropy_workspace_bytes(m, v, k))
    bdr.mx_cross_entropy(f.CFG[fa], pa, f.CFG[fw], pw, m, v, k, targets, loss, lse, ws)
    return loss, lse


def run_grads(pa, pw, fa, fw, m, v, k, targets, lse, dloss, dtype):
    da, dw = torch.full((m, k), float("nan"), device="cuda", dtype=dtype), torch.full((v, k), float("nan"), device="cuda", dtype=dtype)
    ws = f.workspace(bdr.mx_cross_entropy_bwd_workspace_bytes(m, v, k, dtype))
    bdr.mx_cross_entropy_bwd(f.CFG[fa], pa, f.CFG[fw], pw, m, v, k, targets, lse, dloss, da, dw, ws)
    return da, dw


SIZES = [(1, 1, 1), (1, 2, 17), (1, 300, 64), (3, 127, 100), (16, 129, 256), (17, 513, 300), (128, 256, 64), (129, 255, 65), (300, 1000, 1111), (515, 4100, 256)]


@pytest.mark.parametrize("m,v,k", SIZES)
def test_loss(m, v, k):
    (pa, a), (pw, w), targets, gen = operands(m, v, k)
    targets[::7] = -100
    targets[-1] = v - 1
    targets[0] = 0
    loss, lse = run(pa, pw, "mx6", "mx6", m, v, k, targets)
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, else_, "lse")
    f.check(loss, want, eloss, "loss")
    assert (loss[targets < 0] == 0).all()


@pytest.mark.parametrize("fa", ["mx4", "mx6", "mx9"])
@pytest.mark.parametrize("fw", ["mx4", "mx6", "mx9"])
@pytest.mark.parametrize("m", [5, 150])
def test_formats(fa, fw, m):
    v, k = 700, 336
    (pa, a), (pw, w), targets, _ = operands(m, v, k, fa, fw, 1)
    loss, lse = run(pa, pw, fa, fw, m, v, k, targets)
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, else_, "lse")
    f.check(loss, want, eloss, "loss")


@pytest.mark.parametrize("m,v,k", [(256, 500, 3584), (40, 100, 4001), (33, 60, 8192), (300, 300, 2000), (520, 700, 1500)])
def test_few_tiles_with_long_sums(m, v, k):
    # the sums of a tile are shared out to several clusters
    (pa, a), (pw, w), targets, gen = operands(m, v, k, "mx9", "mx6", 10, 1.0)
    runs = [run(pa, pw, "mx9", "mx6", m, v, k, targets) for _ in range(3)]
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(runs[0][1], want_lse, else_, "lse")
    f.check(runs[0][0], want, eloss, "loss")
    dloss = torch.rand(m, device="cuda", generator=gen)
    out = [run_grads(pa, pw, "mx9", "mx6", m, v, k, targets, runs[0][1], dloss, torch.float32) for _ in range(3)]
    want_a, want_w, ea, ew = f.entropy_grads(a, w, targets, runs[0][1].double(), dloss.double(), torch.float32)
    f.check(out[0][0], want_a, ea, "da")
    f.check(out[0][1], want_w, ew, "dw")
    for i in (1, 2):
        assert all(torch.equal(x, y) for x, y in zip(runs[i], runs[0])) and all(torch.equal(x, y) for x, y in zip(out[i], out[0]))


GRAD_SIZES = [(1, 1, 1), (1, 300, 64), (3, 127, 300), (128, 256, 64), (257, 130, 200), (300, 1000, 1111), (70, 2100, 520)]


@pytest.mark.parametrize("m,v,k", GRAD_SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients(m, v, k, dtype):
    (pa, a), (pw, w), targets, gen = operands(m, v, k, "mx9", "mx6", 2)
    targets[1::5] = -1
    _, lse = run(pa, pw, "mx9", "mx6", m, v, k, targets)
    dloss = torch.randn(m, device="cuda", generator=gen)
    da, dw = run_grads(pa, pw, "mx9", "mx6", m, v, k, targets, lse, dloss, dtype)
    want_a, want_w, ea, ew = f.entropy_grads(a, w, targets, lse.double(), dloss.double(), dtype)
    f.check(da, want_a, ea, "da")
    f.check(dw, want_w, ew, "dw")
    assert (da[targets < 0] == 0).all()
    ws = f.workspace(bdr.mx_cross_entropy_bwd_workspace_bytes(m, v, k, dtype))
    one, other = torch.empty_like(da), torch.empty_like(dw)
    bdr.mx_cross_entropy_bwd(bdr.MX9, pa, bdr.MX6, pw, m, v, k, targets, lse, dloss, one, None, ws)
    bdr.mx_cross_entropy_bwd(bdr.MX9, pa, bdr.MX6, pw, m, v, k, targets, lse, dloss, None, other, ws)
    assert torch.equal(one, da) and torch.equal(other, dw)


def test_gradients_by_differences():
    m, v, k = 20, 50, 48
    (pa, a), (pw, w), targets, gen = operands(m, v, k, "mx9", "mx9", 3)
    targets[4] = -100
    _, lse = run(pa, pw, "mx9", "mx9", m, v, k, targets)
    dloss = torch.rand(m, device="cuda", generator=gen)
    da, dw = run_grads(pa, pw, "mx9", "mx9", m, v, k, targets, lse, dloss, torch.float32)
    total = lambda a, w: (f.entropy(a, w, targets)[0] * dloss.double()).sum()  # noqa: E731
    step = 2.0 ** -12
    for t, g, at in ((w, dw, ((0, 0), (49, 47), (int(targets[0]), 3))), (a, da, ((0, 0), (4, 9), (19, 47)))):
        for i, j in at:
            e = torch.zeros_like(t)
            e[i, j] = step
            up, down = (total(a, w + s * e) if t is w else total(a + s * e, w) for s in (1, -1))
            assert abs(float((up - down) / (2 * step) - g[i, j])) < 1e-4      # (fp32 logits, and a third derivative times step^2 / 6)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_pieces_of_the_vocabulary(dtype):
    # enough rows that the vocabulary is taken in more than one piece, the last one ragged
    m, v, k = 4000, 34567, 96
    (pa, a), (pw, w), targets, gen = operands(m, v, k, "mx6", "mx4", 4)
    loss, lse = run(pa, pw, "mx6", "mx4", m, v, k, targets)
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, else_, "lse")
    f.check(loss, want, eloss, "loss")
    dloss = torch.full((m,), 1.0 / m, device="cuda")
    da, dw = run_grads(pa, pw, "mx6", "mx4", m, v, k, targets, lse, dloss, dtype)
    want_a, want_w, ea, ew = f.entropy_grads(a, w, targets, lse.double(), dloss.double(), dtype)
    f.check(da, want_a, ea, "da")
    f.check(dw, want_w, ew, "dw")


@pytest.mark.parametrize("m,v,k", [(33, 1024, 100), (700, 1025, 64), (300, 2048, 300), (2000, 4096, 200), (5000, 4097, 130), (64, 33, 4000), (9500, 4000, 9000)])
def test_parts_of_a_row(m, v, k):
    # few and many parts to join; in the last case they come from several launches
    (pa, a), (pw, w), targets, _ = operands(m, v, k, "mx6", "mx9", 14, 1.0)
    targets[-1], targets[1] = v - 1, -100
    runs = [run(pa, pw, "mx6", "mx9", m, v, k, targets) for _ in range(3)]
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(runs[0][1], want_lse, else_, "lse")
    f.check(runs[0][0], want, eloss, "loss")
    assert all(torch.equal(x, y) for r in runs[1:] for x, y in zip(r, runs[0]))


@pytest.mark.parametrize("m,fmt", [(60, "mx9"), (256, "mx4")])
def test_pieces_of_a_large_vocabulary(m, fmt):
    # decoded weights of more than half a GB: two pieces, in the second case on the 8-bit path
    v, k = 140032, 2048
    gen = torch.Generator(device="cuda").manual_seed(13)
    (pa, a), (pw, w) = (f.packed(f.CFG[fmt], torch.randn(r, k, device="cuda", generator=gen) * s) for r, s in ((m, 1.0), (v, k ** -0.5)))
    targets = torch.randint(0, v, (m,), device="cuda", generator=gen)
    targets[:5] = torch.tensor([v - 1, 70143, 70144, 0, -1], device="cuda")
    loss, lse = run(pa, pw, fmt, fmt, m, v, k, targets)
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, else_, "lse")
    f.check(loss, want, eloss, "loss")
    dloss = torch.rand(m, device="cuda", generator=gen)
    da, dw = run_grads(pa, pw, fmt, fmt, m, v, k, targets, lse, dloss, torch.bfloat16)
    want_a, want_w, ea, ew = f.entropy_grads(a, w, targets, lse.double(), dloss.double(), torch.bfloat16)
    f.check(da, want_a, ea, "da")
    f.check(dw, want_w, ew, "dw")
    assert bdr.bdr_device_status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_parts_of_a_piece(dtype):
    # large enough that the next columns are decoded while the ones before are multiplied; the last part is ragged
    m, v, k = 2100, 18100, 2000
    (pa, a), (pw, w), targets, gen = operands(m, v, k, "mx9", "mx9", 11, 1.0)
    targets[:4] = torch.tensor([0, v - 1, 4700, 9300], device="cuda")
    dloss = torch.full((m,), 1.0 / m, device="cuda")
    runs = []
    for _ in range(2):
        loss, lse = run(pa, pw, "mx9", "mx9", m, v, k, targets)
        runs.append((loss, lse, *run_grads(pa, pw, "mx9", "mx9", m, v, k, targets, lse, dloss, dtype)))
    assert all(torch.equal(x, y) for x, y in zip(*runs))
    loss, lse, da, dw = runs[0]
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, else_, "lse")
    f.check(loss, want, eloss, "loss")
    want_a, want_w, ea, ew = f.entropy_grads(a, w, targets, lse.double(), dloss.double(), dtype)
    f.check(da, want_a, ea, "da")
    f.check(dw, want_w, ew, "dw")


@pytest.mark.parametrize("m,v,k", [(1, 8200, 260), (7, 70001, 33), (24, 4099, 530), (25, 4099, 530), (1, 32800, 1030), (48, 32801, 1029), (49, 32801, 1029)])
@pytest.mark.parametrize("fw", ["mx4", "mx9"])
def test_few_rows(m, v, k, fw):
    # both sides of the limits up to which the few-token kernel computes the logits
    (pa, a), (pw, w), targets, gen = operands(m, v, k, "mx9", fw, 12)
    targets[0] = v - 1
    if m > 1:
        targets[1], targets[-1] = -100, 2048
    bdr.bdr_device_status_reset()
    loss, lse = run(pa, pw, "mx9", fw, m, v, k, targets)
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, else_, "lse")
    f.check(loss, want, eloss, "loss")
    if m > 3:
        targets[2] = v
        other, other_lse = run(pa, pw, "mx9", fw, m, v, k, targets)
        assert other.isnan().nonzero()[:, 0].tolist() == [2] and torch.equal(lse, other_lse)
        assert bdr.bdr_device_status_reset() == -5
        pa.exps[3, 0] = 0xFF
        assert run(pa, pw, "mx9", fw, m, v, k, targets)[1].isnan().nonzero()[:, 0].tolist() == [3]
        bdr.bdr_device_status_reset()


def test_rows_that_do_not_count():
    m, v, k = 130, 300, 64
    (pa, a), (pw, w), targets, _ = operands(m, v, k, seed=5)
    targets[:] = -100
    loss, lse = run(pa, pw, "mx6", "mx6", m, v, k, targets)
    assert (loss == 0).all() and lse.isfinite().all()
    nothing = torch.full((m,), float("nan"), device="cuda")
    da, dw = run_grads(pa, pw, "mx6", "mx6", m, v, k, targets, nothing, nothing, torch.float32)
    assert (da == 0).all() and (dw == 0).all()


def test_a_target_beyond_the_vocabulary_is_reported():
    m, v, k = 40, 300, 64
    (pa, a), (pw, w), targets, _ = operands(m, v, k, seed=6)
    bad = targets.clone()
    bad[3], bad[17] = v, 2 ** 40
    bdr.bdr_device_status_reset()
    loss, lse = run(pa, pw, "mx6", "mx6", m, v, k, targets)
    assert bdr.bdr_device_status() == 0
    other, other_lse = run(pa, pw, "mx6", "mx6", m, v, k, bad)
    assert bdr.bdr_device_status_reset() == -5
    assert other.isnan().nonzero()[:, 0].tolist() == [3, 17] and torch.equal(lse, other_lse)
    there = bad < v
    assert torch.equal(other[there], loss[there])
    dloss = torch.ones(m, device="cuda")
    da, dw = run_grads(pa, pw, "mx6", "mx6", m, v, k, bad, lse, dloss, torch.float32)
    none = torch.where(there, bad, -1)
    ca, cw = run_grads(pa, pw, "mx6", "mx6", m, v, k, none, lse, dloss, torch.float32)
    assert torch.equal(da, ca) and torch.equal(dw, cw)
    assert bdr.bdr_device_status() == 0


def test_large_and_equal_logits():
    # one logit of thousands, and rows whose logits are all equal
    m, v, k = 6, 300, 32
    a, w = torch.zeros(m, k, device="cuda"), torch.zeros(v, k, device="cuda")
    a[0, 0], a[1, 0], a[2, 1] = 100.0, -100.0, 2.0 ** 40
    w[7, 0], w[9, 1] = 64.0, -1.0
    (pa, a), (pw, w) = f.packed(bdr.MX9, a), f.packed(bdr.MX9, w)
    targets = torch.tensor([7, 7, 9, 0, 299, -1], device="cuda")
    loss, lse = run(pa, pw, "mx9", "mx9", m, v, k, targets)
    want, want_lse, _, _, _, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, 2.0 ** -20 * (1 + want_lse.abs()), "lse")
    f.check(loss, want, 2.0 ** -20 * (1 + want.abs()), "loss")
    da, dw = run_grads(pa, pw, "mx9", "mx9", m, v, k, targets, lse, torch.ones(m, device="cuda"), torch.float32)
    assert da.isfinite().all() and dw.isfinite().all()


def test_blocks_without_values_poison_their_own_rows():
    m, v, k = 150, 400, 64
    (pa, a), (pw, w), targets, _ = operands(m, v, k, seed=7)
    clean = run(pa, pw, "mx6", "mx6", m, v, k, targets)
    pa.exps[3, 1] = 0xFF
    loss, lse = run(pa, pw, "mx6", "mx6", m, v, k, targets)
    assert lse.isnan().nonzero()[:, 0].tolist() == [3] and loss.isnan().nonzero()[:, 0].tolist() == [3]
    rest = torch.arange(m, device="cuda") != 3
    assert torch.equal(lse[rest], clean[1][rest])
    pw.exps[399, 0] = 0xFF
    assert run(pa, pw, "mx6", "mx6", m, v, k, targets)[1].isnan().all()


def test_strides_and_surroundings():
    m, v, k = 133, 270, 90
    (pa, a), (pw, w), targets, gen = operands(m, v, k, "mx6", "mx4", 8)
    _, lse = run(pa, pw, "mx6", "mx4", m, v, k, targets)
    dloss = torch.randn(m, device="cuda", generator=gen)
    for dtype in (torch.bfloat16, torch.float32):
        x, y = run_grads(pa, pw, "mx6", "mx4", m, v, k, targets, lse, dloss, dtype)
        da, dw = torch.full((m + 2, k + 9), 7.0, device="cuda", dtype=dtype), torch.full((v + 2, k + 1), 7.0, device="cuda", dtype=dtype)
        ws = f.workspace(bdr.mx_cross_entropy_bwd_workspace_bytes(m, v, k, dtype))
        bdr.mx_cross_entropy_bwd(bdr.MX6, pa, bdr.MX4, pw, m, v, k, targets, lse, dloss, da[1:-1, 4:4 + k], dw[1:-1, 1:], ws)
        assert torch.equal(da[1:-1, 4:4 + k], x) and torch.equal(dw[1:-1, 1:], y)
        da[1:-1, 4:4 + k] = 7.0
        dw[1:-1, 1:] = 7.0
        assert (da == 7).all() and (dw == 7).all()


def test_no_rows():
    (pa, _), (pw, _), _, _ = operands(4, 40, 32)
    ws = f.workspace(bdr.mx_cross_entropy_bwd_workspace_bytes(4, 40, 32, torch.float32))
    none, at = torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    bdr.mx_cross_entropy(bdr.MX6, pa, bdr.MX6, pw, 0, 40, 32, at, none, none.clone(), ws)
    dw = torch.full((40, 32), 7.0, device="cuda")
    bdr.mx_cross_entropy_bwd(bdr.MX6, pa, bdr.MX6, pw, 0, 40, 32, at, none, none, torch.empty(0, 32, device="cuda"), dw, ws)
    assert (dw == 0).all()


def test_captured_and_replayed():
    m, v, k = 260, 700, 200
    (pa, a), (pw, w), targets, gen = operands(m, v, k, seed=9)
    dloss = torch.rand(m, device="cuda", generator=gen)
    size = max(bdr.mx_cross_entropy_workspace_bytes(m, v, k), bdr.mx_cross_entropy_bwd_workspace_bytes(m, v, k))
    ws = f.workspace(size)
    new = lambda *s, **kw: torch.empty(s, device="cuda", **kw)  # noqa: E731
    outs = [(new(m), new(m), new(m, k, dtype=torch.bfloat16), new(v, k, dtype=torch.bfloat16)) for _ in range(2)]

    def step(loss, lse, da, dw):
        bdr.mx_cross_entropy(bdr.MX6, pa, bdr.MX6, pw, m, v, k, targets, loss, lse, ws)
        bdr.mx_cross_entropy_bwd(bdr.MX6, pa, bdr.MX6, pw, m, v, k, targets, lse, dloss, da, dw, ws)

    step(*outs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(*outs[1])
    for _ in range(3):
        for t in outs[1]:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for t, want in zip(outs[1], outs[0]):
            assert torch.equal(t, want)


# few rows of a long vocabulary: blocks of 2048 columns, the last of which may hold one; more of them than the last block has threads, in one case
@pytest.mark.parametrize("m,v,k", [(1, 32768, 64), (24, 32769, 64), (7, 34815, 64), (48, 40961, 840), (3, 530000, 64)])
def test_few_rows_of_many_blocks(m, v, k):
    (pa, a), (pw, w), targets, _ = operands(m, v, k, "mx9", "mx6", v)
    targets[0] = v - 1
    if m > 2:
        targets[1], targets[2] = 2047, 2048
    loss, lse = run(pa, pw, "mx9", "mx6", m, v, k, targets)
    want, want_lse, _, eloss, else_, _ = f.entropy(a, w, targets)
    f.check(lse, want_lse, else_, "lse")
    f.check(loss, want, eloss, "loss")
    # whichever block comes last, the sums are the same; a target behind the vocabulary is reported, a negative one does not count
    workspace = f.workspace(bdr.mx_cross_entropy_workspace_bytes(m, v, k))
    again, again_lse = torch.empty_like(loss), torch.empty_like(lse)
    for _ in range(5):
        bdr.mx_cross_entropy(f.CFG["mx9"], pa, f.CFG["mx6"], pw, m, v, k, targets, again, again_lse, workspace)
        assert torch.equal(again, loss) and torch.equal(again_lse, lse)
    targets[0] = v
    targets[m - 1] = -1 if m > 1 else v
    bdr.mx_cross_entropy(f.CFG["mx9"], pa, f.CFG["mx6"], pw, m, v, k, targets, again, again_lse, workspace)
    assert torch.equal(again_lse, lse) and again[0].isnan() and (m == 1 or again[-1] == 0)
    assert torch.equal(again[1:m - 1], loss[1:m - 1])
    assert bdr.bdr_device_status() != 0
    bdr.bdr_device_status_reset()
