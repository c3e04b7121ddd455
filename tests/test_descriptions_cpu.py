"""What the library is told of packed tensors follows the tensors: after a plane, or what a plane lies in, has been replaced, and after a
cache's planes or sizes have, the next call describes the memory that is there now."""
import copy

import pytest
import torch

from paper_2302_08007_b200 import binding as bdr


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def weights(lines=8):
    return bdr.Planes(u8(lines, 16), u8(lines, 16), u8(lines, 32))


def described(p):
    c = p.c()
    return (c.exps, c.micro, c.elems, c.ld_exps, c.ld_micro, c.ld_elems, p.lines())


def now(p):
    t = (p.exps, p.micro, p.elems)
    return tuple(x.data_ptr() for x in t) + tuple(x.stride(0) for x in t) + (min(x.shape[0] for x in t),)


def test_planes_whose_memory_was_exchanged_in_place():
    for change in (lambda t: setattr(t, "data", u8(8, 64)), lambda t: t.set_(u8(9, 48)), lambda t: t.resize_(4096, 32), lambda t: t.resize_(4, 64),
                   lambda t: t.resize_(3, 32)):
        for name in ("exps", "micro", "elems"):
            w = weights()
            described(w)
            change(getattr(w, name))
            assert described(w) == now(w)
    w = weights()
    assert w.c() is w.c()                                                  # and is not made again for nothing


@pytest.fixture
def asked(monkeypatch):
    """What mx_attn_decode_workspace_bytes, as the other calls, tells the library of a cache."""
    class Recorder:
        def mx_attn_decode_workspace_bytes(self, ref, n_seqs, n_q):
            c = bdr._KVCache.from_address(ref)
            seen.append((c.cfg_k.m, c.cfg_v.m, c.k.exps, c.k.elems, c.k.ld_elems, c.v.exps, c.v.elems, c.v.ld_elems, c.n_pages, c.page_size, c.n_kv, c.head_dim))
            return 0

    seen = []
    recorder = Recorder()
    monkeypatch.setattr(bdr, "lib", lambda: recorder)

    def ask(cache):
        bdr.mx_attn_decode_workspace_bytes(cache, 1, 2)
        k, v = cache.k, cache.v
        assert seen.pop() == (cache.cfg_k.m, cache.cfg_v.m, k.exps.data_ptr(), k.elems.data_ptr(), k.elems.stride(0), v.exps.data_ptr(), v.elems.data_ptr(),
                              v.elems.stride(0), cache.n_pages, cache.page_size, cache.n_kv, cache.head_dim)
    return ask


def cache():
    return bdr.KVCache(bdr.MX6, bdr.MX6, weights(), weights(), 2, 4, 1, 32)


def test_a_cache_whose_planes_or_sizes_were_replaced(asked):
    c = cache()
    asked(c)
    c.k, c.v, c.n_pages = weights(64), weights(64), 16                     # a cache that grows
    asked(c)
    c.k.elems = u8(64, 48)
    asked(c)
    c.v.elems.data = u8(64, 64)
    asked(c)
    c.v.exps.resize_(100, 16)
    asked(c)
    c.page_size, c.n_pages = 8, 8
    asked(c)
    c.cfg_v = bdr.MX4
    asked(c)
    c.k = c.v
    asked(c)


def test_replaced_planes_are_checked_like_new_ones(asked):
    c = cache()
    c.n_pages = 3                                                          # twelve slots, planes of eight lines
    with pytest.raises(ValueError):
        asked(c)
    c.k, c.v = weights(12), weights(12)
    asked(c)
    c.v.micro = torch.zeros((12, 16))
    with pytest.raises(ValueError):
        asked(c)


def test_copies_have_a_description_of_their_own(asked):
    c = cache()
    for other in (copy.copy(c), copy.deepcopy(c)):
        asked(other)
        other.n_pages = 1
        asked(other)
        asked(c)
    assert copy.deepcopy(c).k.exps.data_ptr() != c.k.exps.data_ptr() and copy.copy(c).k is c.k
