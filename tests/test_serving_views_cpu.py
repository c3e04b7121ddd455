"""The Python boundary of the serving calls and views whose rows share memory (expanded, or strided below a row): the kernels would walk
past such a tensor's end, so the calls refuse it.  A pitch means nothing, and is passed as a whole row, where there is one row at most.
The library call is replaced by a recorder, and CPU tensors say that they are on a GPU."""
import pytest
import torch

from paper_2302_08007_b200 import binding as bdr


class OnGpu(torch.Tensor):
    is_cuda = True


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def calls(monkeypatch):
    seen = []

    class Recorder:
        def __getattr__(self, name):
            return lambda *a: seen.append((name, a)) or 0

    monkeypatch.setattr(bdr, "lib", lambda: Recorder())
    monkeypatch.setattr(bdr, "_stream", lambda stream: None)
    return seen


def planes(lines, cols, bits=5):
    return bdr.Planes(*(t(lines, -(-b // 16) * 16, dtype=torch.uint8) for b in (cols // 16, cols // 16, cols * bits // 8)))


def cache():
    return bdr.KVCache(bdr.MX6, bdr.MX6, planes(32, 64), planes(32, 64), 8, 4, 2, 32)


def overlapping(shape, pitch, dtype=torch.bfloat16):
    rest = [1] * len(shape)
    for i in range(len(shape) - 2, 0, -1):
        rest[i] = rest[i + 1] * shape[i + 1]
    rest[0] = pitch
    return t(4096, dtype=dtype).as_strided(shape, rest)


def test_rows_of_products(calls):
    w = planes(8, 32)
    go = lambda x, y: bdr.mx_gemv(bdr.MX6, w, 8, 32, x, y)  # noqa: E731
    for x, y in ((t(1, 32).expand(4, 32), t(4, 8)), (t(4, 32), t(1, 8).expand(4, 8)), (overlapping((4, 32), 31), t(4, 8)), (t(4, 32), overlapping((4, 8), 7))):
        with pytest.raises(ValueError):
            go(x, y)
    assert not calls
    go(overlapping((1, 32), 0), overlapping((1, 8), 3))
    go(t(4, 48)[:, :32], t(4, 9)[:, 1:])
    go(t(32), t(8))
    go(t(0, 32), t(0, 8))
    assert [(a[6], a[7], a[10]) for _, a in calls] == [(32, 1, 8), (48, 4, 9), (32, 1, 8), (32, 0, 8)]


def test_tokens_of_an_append(calls):
    slots = t(3, dtype=torch.int64)
    good = dict(k=t(3, 2, 32), v=t(3, 2, 32), q=t(3, 4, 32), q_out=t(3, 4, 32), cos=t(5, 16, dtype=torch.float32), sin=t(5, 16, dtype=torch.float32))

    def go(**kw):
        a = {**good, **kw}
        bdr.mx_kv_append(cache(), a["k"], a["v"], slots, slots, a["cos"], a["sin"], q=a["q"], q_out=a["q_out"])

    table = t(1, 16, dtype=torch.float32).expand(5, 16)
    for kw in (dict(k=t(1, 2, 32).expand(3, 2, 32)), dict(v=overlapping((3, 2, 32), 63)), dict(q=t(1, 4, 32).expand(3, 4, 32)), dict(q_out=t(1, 4, 32).expand(3, 4, 32)),
               dict(q_out=overlapping((3, 4, 32), 127)), dict(cos=table, sin=table), dict(cos=overlapping((5, 16), 15, torch.float32), sin=overlapping((5, 16), 15, torch.float32)),
               dict(k=t(3, 1, 32).expand(3, 2, 32)), dict(k=t(3, 2, 1).expand(3, 2, 32))):
        with pytest.raises(ValueError):
            go(**kw)
    assert not calls
    go()
    fused = t(3, 8, 32)
    go(q=fused[:, :4], k=fused[:, 4:6], v=fused[:, 6:])
    a = [x for _, x in calls]
    assert [(x[2], x[4], x[10], x[13]) for x in a] == [(64, 64, 128, 128), (256, 256, 256, 128)]


def test_sequences_of_an_attention(calls):
    good = dict(q=t(3, 4, 32), out=t(3, 4, 32), table=t(3, 5, dtype=torch.int32))
    lengths, ws = t(3, dtype=torch.int32), t(1 << 16, dtype=torch.uint8)

    def go(**kw):
        a = {**good, **kw}
        n = a["q"].shape[0]
        bdr.mx_attn_decode(cache(), a["q"], a["table"], lengths[:n], a["out"], ws)

    for kw in (dict(q=t(1, 4, 32).expand(3, 4, 32)), dict(q=overlapping((3, 4, 32), 64)), dict(out=t(1, 4, 32).expand(3, 4, 32)),
               dict(table=t(1, 5, dtype=torch.int32).expand(3, 5)), dict(table=overlapping((3, 5), 4, torch.int32))):
        with pytest.raises(ValueError):
            go(**kw)
    assert not calls
    go()
    go(table=t(3, 9, dtype=torch.int32)[:, 2:7])
    go(q=overlapping((1, 4, 32), 0), out=overlapping((1, 4, 32), 0), table=overlapping((1, 5), 0, torch.int32))
    a = [x for _, x in calls]
    assert [(x[2], x[7], x[8], x[13]) for x in a] == [(128, 5, 5, 128), (128, 9, 5, 128), (128, 5, 5, 128)]


def test_a_window_wider_than_any_cache_is_no_narrower_one(calls):
    q, table, lengths, ws = t(3, 4, 32), t(3, 5, dtype=torch.int32), t(3, dtype=torch.int32), t(1 << 16, dtype=torch.uint8)
    for window, want in ((0, 0), (7, 7), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 32 + 5, 2 ** 31 - 1), (2 ** 63 - 1, 2 ** 31 - 1), (-1, -1)):
        calls.clear()
        bdr.mx_attn_decode(cache(), q, table, lengths, torch.empty_like(q), ws, window=window)
        assert calls[0][1][11] == want
    with pytest.raises(ValueError):
        bdr.mx_attn_decode(cache(), q, table, lengths, torch.empty_like(q), ws, window=-2 ** 32 + 3)


def test_planes_that_are_not_all_on_a_gpu(calls):
    host = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    q, k, slots, table, lengths, ws = t(3, 4, 32), t(3, 2, 32), t(3, dtype=torch.int64), t(3, 5, dtype=torch.int32), t(3, dtype=torch.int32), t(1 << 16, dtype=torch.uint8)
    for name in ("exps", "micro", "elems"):
        w = planes(8, 32)
        setattr(w, name, host(*getattr(w, name).shape))
        with pytest.raises(ValueError):
            bdr.mx_gemv(bdr.MX6, w, 8, 32, t(4, 32), t(4, 8))
        for which in ("k", "v"):
            c = cache()
            setattr(getattr(c, which), name, host(*getattr(getattr(c, which), name).shape))
            with pytest.raises(ValueError):
                bdr.mx_kv_append(c, k, k, slots)
            with pytest.raises(ValueError):
                bdr.mx_attn_decode(c, q, table, lengths, torch.empty_like(q), ws)
    assert not calls
