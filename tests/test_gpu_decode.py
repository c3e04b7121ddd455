"""One decoder block's attention step on MX storage (decode.py): several tokens per sequence through the three serving operators
together.  Every stage is compared with its definition in 64 bits on the oracle's quantized values, taking the stage's inputs
from the GPU (so that a bf16 rounding of one stage is not counted against the next), with the bounds of the operators' own tests."""
import numpy as np
import pytest
import torch

from oracle import oracle as orc
from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import decode, synth
from tests import helpers as H
from tests import test_gpu_gemv as G
from tests import test_gpu_kv_append as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt_w,fk,fv,dtype", [(bdr.MX6, bdr.MX9, bdr.MX6, "bf16"), (bdr.MX4, bdr.MX6, bdr.MX4, "f32")], ids=["bf16", "f32"])
def test_tokens_through_a_block(fmt_w, fk, fv, dtype):
    n_seqs, d_model, n_q, n_kv, d, page = 3, 320, 8, 2, 64, 4
    heads = n_q + 2 * n_kv
    w_qkv = synth.normal_matrix(heads * d, d_model, seed=1, stream=1, sigma=d_model ** -0.5)
    w_out = synth.normal_matrix(d_model, n_q * d, seed=1, stream=2, sigma=(n_q * d) ** -0.5)
    cache = bdr.alloc_kv_cache(fk, fv, 16, page, n_kv, d)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    block = decode.alloc(fmt_w, torch.from_numpy(w_qkv).cuda(), torch.from_numpy(w_out).cuda(), cache, n_q, n_seqs, 64, dtype=td)
    table = torch.from_numpy(np.random.default_rng(3).permutation(16)[:15].reshape(n_seqs, 5).astype(np.int32)).cuda()
    lengths = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    lines = [[np.zeros((0, n_kv * d), np.float32)] * 2 for _ in range(n_seqs)]  # quantized keys, values by position
    start = lengths.cpu().numpy().copy()
    # what the sequences held before: appended without a rotation
    for s in range(n_seqs):
        t = int(start[s])
        if t:
            kv = H.make_input("normal", t, 2 * n_kv * d, dtype, seed=s).reshape(t, 2 * n_kv, d)
            pos = torch.arange(t, device="cuda")
            bdr.mx_kv_append(cache, A.dev(kv[:, :n_kv], dtype), A.dev(kv[:, n_kv:], dtype), decode.slots_of(table[s:s + 1].expand(t, -1), pos, page))
            lines[s] = [orc.quant_dequant(H.to_orc(f), np.ascontiguousarray(x.reshape(t, -1)), axis=1)[0] for f, x in ((fk, kv[:, :n_kv]), (fv, kv[:, n_kv:]))]
    wq, wo = (orc.quant_dequant(H.to_orc(fmt_w), w, axis=1)[0] for w in (w_qkv, w_out))
    cos, sin = block.cos.cpu().numpy(), block.sin.cpu().numpy()
    for it in range(7):
        h = H.make_input("normal", n_seqs, d_model, dtype, seed=100 + it)
        before = lengths.cpu().numpy().copy()
        out = decode.step(block, H.host_to_device(h, dtype), table, lengths)
        torch.cuda.synchronize()
        assert (lengths.cpu().numpy() == before + 1).all()
        G.check(block.qkv.view(n_seqs, -1), h, wq, d_model, dtype)
        qkv = H.device_to_host_f32(block.qkv).reshape(n_seqs, heads, d)
        rotated = A.rotate(qkv[:, :n_q + n_kv], cos[before], sin[before], False)
        H.assert_bits_equal(H.device_to_host_f32(block.q), A.to_dtype(rotated[:, :n_q], dtype))
        att = H.device_to_host_f32(block.attended).astype(np.float64)
        for s in range(n_seqs):
            new = [orc.quant_dequant(H.to_orc(f), np.ascontiguousarray(x.reshape(1, -1)), axis=1)[0] for f, x in ((fk, rotated[s, n_q:]), (fv, qkv[s, n_q + n_kv:]))]
            lines[s] = [np.concatenate([a, b]) for a, b in zip(lines[s], new)]
            slots = decode.slots_of(table[s:s + 1].expand(len(lines[s][0]), -1), torch.arange(len(lines[s][0]), device="cuda"), page)
            for f, pl, want in ((fk, cache.k, lines[s][0]), (fv, cache.v, lines[s][1])):
                got = torch.empty((len(want), n_kv * d), dtype=torch.float32, device="cuda")
                bdr.bdr_gather_rows(f, pl, 16 * page, slots, got)
                H.assert_bits_equal(got.cpu().numpy(), want)
            k, v = (x.astype(np.float64).reshape(-1, n_kv, d) for x in lines[s])
            q = H.device_to_host_f32(block.q)[s].astype(np.float64).reshape(n_kv, n_q // n_kv, d)
            sc = np.einsum("hgd,thd->hgt", q, k) * d ** -0.5
            w = np.exp(sc - sc.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            want = np.einsum("hgt,thd->hgd", w, v).reshape(n_q, d)
            A_ = np.einsum("hgt,thd->hgd", w, np.abs(v)).reshape(n_q, d)
            # the attention test's bound with its score term for these sizes: |scores| < 32 and sum |q k| / 8 < 64
            dw = 2 * (d / 16 + 16) * 2.0 ** -22 * 64 + 2.0 ** -22 * (4 + 64 + 8)
            assert np.abs(sc).max() < 32 and (np.einsum("hgd,thd->hgt", np.abs(q), np.abs(k)) * d ** -0.5).max() < 64
            bound = 1.1 * A_ * (2 * dw + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -16) + 65 * 2.0 ** -22)
            if dtype == "bf16":
                bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
            assert (np.abs(att[s] - want) <= bound).all()
        G.check(out, att.reshape(n_seqs, -1).astype(np.float32), wo, n_q * d, dtype)
    assert bdr.bdr_device_status() == 0


def test_steps_replayed_from_a_graph_equal_steps_called_one_by_one():
    n_seqs, d_model, n_q, n_kv, d, page = 2, 256, 4, 2, 64, 8
    w_qkv = torch.from_numpy(synth.normal_matrix((n_q + 2 * n_kv) * d, d_model, seed=1, stream=1, sigma=d_model ** -0.5)).cuda()
    w_out = torch.from_numpy(synth.normal_matrix(d_model, n_q * d, seed=1, stream=2, sigma=(n_q * d) ** -0.5)).cuda()
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    tokens = [H.host_to_device(H.make_input("normal", n_seqs, d_model, "bf16", seed=i), "bf16") for i in range(5)]

    def fresh():
        cache = bdr.alloc_kv_cache(bdr.MX6, bdr.MX6, 8, page, n_kv, d)
        return decode.alloc(bdr.MX6, w_qkv, w_out, cache, n_q, n_seqs, 32), torch.tensor([0, 3], dtype=torch.int32, device="cuda")

    def prime(block):   # three tokens in the second sequence's cache
        x = H.host_to_device(H.make_input("normal", 3, 2 * n_kv * d, "bf16", seed=50), "bf16").unflatten(1, (2 * n_kv, d))
        bdr.mx_kv_append(block.cache, x[:, :n_kv], x[:, n_kv:], torch.arange(3, device="cuda") + 4 * page)

    block, lengths = fresh()
    prime(block)
    want = [decode.step(block, t, table, lengths).clone() for t in tokens]
    block, lengths = fresh()
    prime(block)
    h, out = torch.empty_like(tokens[0]), torch.empty_like(tokens[0])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        h.copy_(tokens[0])
        decode.step(block, h, table, lengths, out)            # first calls outside the capture
        side.synchronize()
        assert torch.equal(out, want[0])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            decode.step(block, h, table, lengths, out)
        for t, w in zip(tokens[1:], want[1:]):
            h.copy_(t)
            graph.replay()
            side.synchronize()
            assert torch.equal(out, w)
    assert lengths.tolist() == [5, 8]
