"""What decode.step does around the library's calls, which a recorder replaces here."""
import contextlib

import pytest
import torch

from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import decode

N_SEQS, D_MODEL, N_Q, N_KV, D, PAGE = 2, 96, 4, 2, 32, 4


@pytest.fixture
def world(monkeypatch):
    """A block on the CPU, and what happens in a step: (what, in which stream)."""
    now, seen = ["current"], []

    @contextlib.contextmanager
    def stream(s):
        before, now[0] = now[0], s
        yield
        now[0] = before

    def called(name):
        return lambda *a, **kw: seen.append((name, now[0], a))

    empty_like = torch.empty_like
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: now[0])
    monkeypatch.setattr(torch, "empty_like", lambda *a, **kw: seen.append(("empty_like", now[0], a)) or empty_like(*a, **kw))
    for name in ("mx_gemv", "mx_kv_append", "mx_attn_decode"):
        monkeypatch.setattr(bdr, name, called(name))
    cache = bdr.alloc_kv_cache(bdr.MX6, bdr.MX6, 8, PAGE, N_KV, D, device="cpu")
    w = lambda n, k: bdr.alloc_planes(bdr.MX6, n, k, 1, device="cpu")  # noqa: E731
    new = lambda h: torch.zeros((N_SEQS, h, D), dtype=torch.bfloat16)  # noqa: E731
    heads = N_Q + 2 * N_KV
    block = decode.AttentionBlock(bdr.MX6, w(heads * D, D_MODEL), w(D_MODEL, N_Q * D), cache, N_Q, torch.zeros(32, D // 2), torch.zeros(32, D // 2), new(heads), new(N_Q),
                                  new(N_Q), torch.zeros(64, dtype=torch.uint8))
    table = torch.arange(8, dtype=torch.int32).view(2, 4)
    return block, table, torch.tensor([3, 5], dtype=torch.int32), torch.zeros((N_SEQS, D_MODEL), dtype=torch.bfloat16), seen


@pytest.mark.parametrize("stream", [None, "side"])
def test_the_result_is_allocated_on_the_stream_that_writes_it(world, stream):
    block, table, lengths, h, seen = world
    out = decode.step(block, h, table, lengths, stream=stream)
    assert out.shape == h.shape and out.dtype == h.dtype
    assert {s for _, s, _ in seen} == {stream or "current"} and [n for n, _, _ in seen].count("empty_like") == 1
    assert [n for n, _, _ in seen if n != "empty_like"] == ["mx_gemv", "mx_kv_append", "mx_attn_decode", "mx_gemv"]
    assert seen[-1][2][-1] is out


def appended_and_attended(seen):
    by = {n: a for n, _, a in seen}
    return by["mx_kv_append"][3].tolist(), by["mx_kv_append"][4].tolist(), by["mx_attn_decode"][3].tolist()


def test_blocks_of_one_model_share_the_lengths(world):
    block, table, lengths, h, seen = world
    for advance, after in ((False, [3, 5]), (False, [3, 5]), (True, [4, 6])):
        seen.clear()
        decode.step(block, h, table, lengths, advance=advance)
        assert appended_and_attended(seen) == ([3, 5 * PAGE + 1], [3, 5], [4, 6])
        assert lengths.tolist() == after and lengths.dtype == torch.int32


def test_lengths_of_another_type_are_refused_before_anything_is_done(world):
    block, table, lengths, h, seen = world
    wide = lengths.long()
    with pytest.raises(ValueError):
        decode.step(block, h, table, wide)
    assert not seen and wide.tolist() == [3, 5]
