"""The gated layer and the cross entropy on streams of their own: two at a time, and graphs that share a workspace."""
import pytest
import torch

import fused_helpers as f
from paper_2302_08007_b200 import binding as bdr

pytestmark = pytest.mark.gpu


class Layer:
    """Operands, outputs and a workspace of one layer or head."""

    def __init__(self, kind, m, n, k, fmt, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.cfg, self.sizes, self.kind = f.CFG[fmt], (m, n, k), kind
        lines = 2 * n if kind == "gated" else n
        self.a, _ = f.packed(self.cfg, torch.randn(m, k, device="cuda", generator=gen))
        self.w, _ = f.packed(self.cfg, torch.randn(lines, k, device="cuda", generator=gen) * k ** -0.5)
        new = lambda *s, dt=torch.bfloat16: torch.empty(s, dtype=dt, device="cuda")  # noqa: E731
        if kind == "gated":
            self.dh = torch.randn(m, n, device="cuda", generator=gen).bfloat16()
            self.out = [new(m, n), new(m, 2 * n), new(m, k), new(lines, k)]
            size = max(bdr.mx_gated_gemm_workspace_bytes(m, n, k), bdr.mx_gated_gemm_bwd_workspace_bytes(m, n, k))
        else:
            self.targets = torch.randint(0, n, (m,), device="cuda", generator=gen)
            self.dloss = torch.rand(m, device="cuda", generator=gen)
            self.out = [new(m, dt=torch.float32), new(m, dt=torch.float32), new(m, k), new(lines, k)]
            size = max(bdr.mx_cross_entropy_workspace_bytes(m, n, k), bdr.mx_cross_entropy_bwd_workspace_bytes(m, n, k))
        self.ws = f.workspace(size)

    def run(self, stream=None, ws=None):
        ops, ws = (self.cfg, self.a, self.cfg, self.w, *self.sizes), self.ws if ws is None else ws
        if self.kind == "gated":
            h, kept, da, dw = self.out
            bdr.mx_gated_gemm(*ops, h, ws, gate_up=kept, stream=stream)
            bdr.mx_gated_gemm_bwd(*ops, self.dh, da, dw, ws, gate_up=kept, stream=stream)
        else:
            loss, lse, da, dw = self.out
            bdr.mx_cross_entropy(*ops, self.targets, loss, lse, ws, stream=stream)
            bdr.mx_cross_entropy_bwd(*ops, self.targets, lse, self.dloss, da, dw, ws, stream=stream)


SIZES = [(("gated", 300, 500, 700, "mx9"), ("entropy", 260, 1000, 3000, "mx6")), (("gated", 2304, 1920, 4096, "mx6"), ("entropy", 2100, 18100, 2000, "mx9")),
         (("gated", 20, 4100, 260, "mx4"), ("entropy", 256, 256, 4096, "mx4"))]


@pytest.mark.parametrize("first,second", SIZES)
def test_two_streams_at_a_time(first, second):
    layers = [Layer(*first, 1), Layer(*second, 2)]
    want = []
    for x in layers:
        x.run()
        want.append([t.clone() for t in x.out])
        for t in x.out:
            t.fill_(float("nan"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for x, s in zip(layers, streams):
            x.run(stream=s)
    torch.cuda.synchronize()
    for x, w in zip(layers, want):
        assert all(torch.equal(t, u) for t, u in zip(x.out, w))
    assert bdr.bdr_device_status() == 0


def test_two_graphs_that_share_a_workspace():
    layers = [Layer("gated", 300, 500, 700, "mx9", 3), Layer("entropy", 260, 1000, 3000, "mx6", 4)]
    ws = f.workspace(max(x.ws.numel() for x in layers))
    want, graphs = [], []
    side = torch.cuda.Stream()
    for x in layers:
        x.run()
        want.append([t.clone() for t in x.out])
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            x.run(ws=ws)
        graphs.append(graph)
    for _ in range(3):
        for x in layers:
            for t in x.out:
                t.fill_(float("nan"))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for x, w in zip(layers, want):
            assert all(torch.equal(t, u) for t, u in zip(x.out, w))
