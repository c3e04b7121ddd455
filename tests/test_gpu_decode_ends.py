"""decode.step where a sequence has filled its pages, or has a negative length: NaN and the status word for the former, zeros for the latter, and
nothing changes for the sequences beside them."""
import numpy as np
import pytest
import torch

from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import decode, synth
from tests import helpers as H

pytestmark = pytest.mark.gpu

N_SEQS, D_MODEL, N_Q, N_KV, D, PAGE = 3, 256, 4, 2, 64, 4


def block(n_pos=64):
    w_qkv = torch.from_numpy(synth.normal_matrix((N_Q + 2 * N_KV) * D, D_MODEL, seed=1, stream=1, sigma=D_MODEL ** -0.5)).cuda()
    w_out = torch.from_numpy(synth.normal_matrix(D_MODEL, N_Q * D, seed=1, stream=2, sigma=(N_Q * D) ** -0.5)).cuda()
    cache = bdr.alloc_kv_cache(bdr.MX6, bdr.MX6, 8, PAGE, N_KV, D)
    b = decode.alloc(bdr.MX6, w_qkv, w_out, cache, N_Q, N_SEQS, n_pos)
    kv = H.host_to_device(H.make_input("normal", 8 * PAGE, 2 * N_KV * D, "bf16", seed=9), "bf16").unflatten(1, (2 * N_KV, D))
    bdr.mx_kv_append(cache, kv[:, :N_KV], kv[:, N_KV:], torch.arange(8 * PAGE, device="cuda"))   # every slot holds something
    return b


def h(seed=3):
    return H.host_to_device(H.make_input("normal", N_SEQS, D_MODEL, "bf16", seed=seed), "bf16")


def planes(b):
    return [p.clone() for pl in (b.cache.k, b.cache.v) for p in (pl.exps, pl.micro, pl.elems)]


def test_a_full_sequence_is_reported_and_overwrites_nothing():
    table = torch.tensor([[6, 1], [3, 0], [2, 7]], dtype=torch.int32, device="cuda")
    b = block()
    want = decode.step(b, h(), table, torch.tensor([2, 5, 0], dtype=torch.int32, device="cuda")).clone()
    assert bdr.bdr_device_status() == 0
    for full in (2 * PAGE, 2 * PAGE + 9):
        b = block()
        before = planes(b)
        got = decode.step(b, h(), table, torch.tensor([2, full, 0], dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert bdr.bdr_device_status_reset() == -5
        assert torch.isnan(got[1]).all() and torch.equal(got[[0, 2]], want[[0, 2]])
        changed = [(p != q).any(1).nonzero().flatten().tolist() for p, q in zip(planes(b), before)]
        assert set(sum(changed, [])) == {6 * PAGE + 2, 2 * PAGE}              # the other two sequences' new tokens


def test_a_negative_length_counts_as_an_empty_sequence():
    table = torch.tensor([[6, 1], [3, 0], [2, 7]], dtype=torch.int32, device="cuda")
    want = decode.step(block(), h(), table, torch.tensor([2, 5, 0], dtype=torch.int32, device="cuda")).clone()
    b = block()
    before = planes(b)
    got = decode.step(b, h(), table, torch.tensor([2, -3, 0], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert not got[1].any() and torch.equal(got[[0, 2]], want[[0, 2]])
    changed = [(p != q).any(1).nonzero().flatten().tolist() for p, q in zip(planes(b), before)]
    assert set(sum(changed, [])) == {6 * PAGE + 2, 2 * PAGE}
    bdr.bdr_device_status_reset()
    assert np.isfinite(H.device_to_host_f32(got)).all()


def test_a_negative_length_is_not_an_error():
    table = torch.tensor([[6, 1], [3, 0], [2, 7]], dtype=torch.int32, device="cuda")
    decode.step(block(), h(), table, torch.tensor([2, -3, 0], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert bdr.bdr_device_status_reset() == 0


def test_two_blocks_with_one_tensor_of_lengths():
    table = torch.tensor([[6, 1], [3, 0], [2, 7]], dtype=torch.int32, device="cuda")
    start = torch.tensor([2, 5, 0], dtype=torch.int32, device="cuda")
    pair = lambda: (block(), block())  # noqa: E731
    x, (a, b), la, lb = h(), pair(), start.clone(), start.clone()
    want = [decode.step(b, decode.step(a, x, table, la), table, lb).clone() for _ in range(2)]
    (a, b), lengths = pair(), start.clone()
    got = [decode.step(b, decode.step(a, x, table, lengths, advance=False), table, lengths).clone() for _ in range(2)]
    assert all(torch.equal(g, w) for g, w in zip(got, want)) and lengths.tolist() == [4, 7, 2]
    assert bdr.bdr_device_status() == 0
