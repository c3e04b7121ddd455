"""CPU-only checks of the serving operators' boundary: host-side argument validation (no launch happens before it), workspace
sizes, and the Python binding's refusals."""
import ctypes as C

import pytest
import torch

from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import decode

NULL, BAD, UNSUPPORTED, MISALIGNED, SIZE, WORKSPACE = -1, -2, -3, -4, -5, -6
P = 4096                                                       # an aligned address that is never dereferenced: validation fails first


def planes(ld=4096, base=P):
    return bdr._Planes(base, base, base, ld, ld, ld)


def cache(**kw):
    f = dict(cfg_k=bdr.MX6.c(), cfg_v=bdr.MX9.c(), k=planes(), v=planes(), n_pages=8, page_size=16, n_kv=4, head_dim=64)
    f.update(kw)
    return bdr._KVCache(*[f[n] for n in ("cfg_k", "cfg_v", "k", "v", "n_pages", "page_size", "n_kv", "head_dim")])


def gemv(cfg=bdr.MX6, w=None, N=64, K=128, x=P, xdt=1, ldx=128, T=1, y=P, ydt=1, ldy=64):
    c, w = cfg.c(), planes() if w is None else w
    return bdr.lib().mx_gemv(C.addressof(c), C.addressof(w), N, K, x, xdt, ldx, T, y, ydt, ldy, None)


def test_mx_gemv_refusals():
    L = bdr.lib()
    w = planes()
    assert L.mx_gemv(None, C.addressof(w), 64, 128, P, 1, 128, 1, P, 1, 64, None) == NULL
    assert gemv(cfg=bdr.Config(16, 8, 3, 1, 4)) == BAD
    for cfg in (bdr.Config(32, 8, 2, 1, 4), bdr.Config(16, 8, 2, 1, 5), bdr.Config(16, 8, 2, 0, 4), bdr.Config(0, 32, 1, 4, 3, bdr.SCALE_FP32_FP)):
        assert gemv(cfg=cfg) == UNSUPPORTED
    assert gemv(xdt=2) == UNSUPPORTED and gemv(ydt=-1) == UNSUPPORTED
    assert gemv(N=-1) == SIZE and gemv(K=-1) == SIZE and gemv(T=-1) == SIZE and gemv(ldx=127) == SIZE and gemv(ldy=63) == SIZE
    assert gemv(x=None) == NULL and gemv(y=None) == NULL and gemv(w=bdr._Planes(None, P, P, 16, 16, 160)) == NULL
    assert gemv(x=P + 1) == MISALIGNED and gemv(y=P + 1) == MISALIGNED and gemv(w=planes(base=P + 8)) == MISALIGNED and gemv(w=planes(ld=4088)) == MISALIGNED
    assert gemv(w=bdr._Planes(P, P, P, 16, 16, 64)) == SIZE                     # 128 codes of five bits are 80 bytes
    assert gemv(T=0) == 0 and gemv(N=0, ldy=0) == 0                            # nothing to do


def append(c=None, k=P, ldk=256, v=P, ldv=256, dt=1, T=3, slots=P, rot=None, q=None, ldq=0, n_q=0, q_out=None, ldo=0, kd=None, vd=None):
    c = cache() if c is None else c
    return bdr.lib().mx_kv_append(C.addressof(c), k, ldk, v, ldv, dt, T, slots, C.addressof(rot) if rot is not None else None, q, ldq, n_q,
                                  q_out, ldo, kd, vd, None)


def rotation(cos=P, sin=P, pos=P, ld=32, n_pos=10, rot_dim=64, inter=0):
    return bdr._Rotation(cos, sin, pos, ld, n_pos, rot_dim, inter)


@pytest.mark.parametrize("bad,status", [(dict(cfg_k=bdr.Config(16, 8, 2, 1, 5).c()), UNSUPPORTED), (dict(cfg_v=bdr.Config(32, 8, 2, 1, 4).c()), UNSUPPORTED),
                                        (dict(cfg_k=bdr.Config(16, 8, 2, 1, 4, 0, 1).c()), UNSUPPORTED), (dict(cfg_v=bdr.Config(16, 7, 2, 1, 4).c()), BAD),
                                        (dict(n_pages=-1), SIZE), (dict(page_size=0), SIZE), (dict(n_kv=0), SIZE), (dict(head_dim=0), SIZE),
                                        (dict(n_pages=1 << 30), SIZE), (dict(head_dim=72), UNSUPPORTED), (dict(head_dim=272, n_kv=1), UNSUPPORTED),
                                        (dict(k=planes(ld=16)), SIZE), (dict(v=planes(base=P + 4)), MISALIGNED), (dict(k=bdr._Planes(P, None, P, 16, 16, 160)), NULL),
                                        (dict(v=planes(ld=1 << 32)), SIZE)])
def test_cache_descriptions_that_no_call_accepts(bad, status):
    c = cache(**bad)
    assert append(c=c) == status
    assert attend(c=c) == status
    assert bdr.lib().mx_attn_decode_workspace_bytes(C.addressof(c), 2, 8) == 0


def test_mx_kv_append_refusals():
    assert bdr.lib().mx_kv_append(None, P, 256, P, 256, 1, 3, P, None, None, 0, 0, None, 0, None, None, None) == NULL
    assert append(dt=3) == UNSUPPORTED and append(T=-1) == SIZE and append(ldk=255) == SIZE and append(ldv=0) == SIZE
    assert append(k=None) == NULL and append(v=None) == NULL and append(slots=None) == NULL
    assert append(slots=P + 4) == MISALIGNED and append(k=P + 1) == MISALIGNED and append(kd=P + 8) == MISALIGNED and append(vd=P + 2) == MISALIGNED
    for rot, status in ((rotation(rot_dim=63), SIZE), (rotation(rot_dim=66), SIZE), (rotation(rot_dim=-2), SIZE), (rotation(ld=31), SIZE), (rotation(n_pos=-1), SIZE),
                        (rotation(cos=None), NULL), (rotation(pos=None), NULL), (rotation(sin=P + 2), MISALIGNED), (rotation(pos=P + 4), MISALIGNED)):
        assert append(rot=rot) == status
    assert append(q=P, ldq=64, n_q=2, q_out=2 * P, ldo=128) == SIZE and append(q=P, ldq=128, n_q=0, q_out=2 * P, ldo=128) == SIZE
    assert append(q=P, ldq=128, n_q=2, q_out=None, ldo=128) == NULL and append(q=P, ldq=128, n_q=2, q_out=P, ldo=128) == UNSUPPORTED
    assert append(T=0) == 0


def attend(c=None, q=P, ldq=512, dt=1, B=2, n_q=8, table=P, ldt=4, pages=4, lengths=P, scale=0.125, window=0, out=P, ldo=512, lse=None, ws=P, bytes_=1 << 40):
    c = cache() if c is None else c
    return bdr.lib().mx_attn_decode(C.addressof(c), q, ldq, dt, B, n_q, table, ldt, pages, lengths, scale, window, out, ldo, lse, ws, bytes_, None)


def test_mx_attn_decode_refusals():
    assert attend(dt=2) == UNSUPPORTED and attend(n_q=6) == SIZE and attend(n_q=0) == SIZE and attend(B=-1) == SIZE
    assert attend(ldq=511) == SIZE and attend(ldo=511) == SIZE and attend(ldt=3) == SIZE and attend(pages=-1) == SIZE and attend(window=-1) == SIZE
    assert attend(pages=1 << 28, ldt=1 << 28) == SIZE
    assert attend(q=None) == NULL and attend(out=None) == NULL and attend(lengths=None) == NULL and attend(table=None) == NULL
    assert attend(q=P + 1) == MISALIGNED and attend(lengths=P + 2) == MISALIGNED and attend(lse=P + 1) == MISALIGNED and attend(ws=P + 8) == MISALIGNED
    assert attend(ws=None) == WORKSPACE and attend(bytes_=64) == WORKSPACE
    assert attend(scale=float("inf")) == BAD and attend(scale=float("nan")) == BAD
    assert attend(B=0) == 0


def test_workspace_covers_both_query_types_and_grows_with_the_heads():
    c = cache()
    size = lambda n_q: bdr.lib().mx_attn_decode_workspace_bytes(C.addressof(c), 4, n_q)  # noqa: E731
    assert size(8) > 0 and size(8) % 256 == 0 and size(16) > size(8)
    assert size(6) == 0 and size(-4) == 0


def test_the_binding_refuses_what_it_can_see():
    t = lambda *s, d=torch.bfloat16: torch.zeros(s, dtype=d)  # noqa: E731
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    w = bdr.Planes(u8(8, 16), u8(8, 16), u8(8, 32))
    for x, y, n in ((t(1, 30), t(1, 8), 8), (t(1, 32), t(1, 9), 8), (t(2, 32), t(1, 8), 8), (t(1, 32), t(1, 9), 9), (t(32, 4).T[:1], t(1, 8), 8), (t(1, 32), t(1, 8), 8)):
        with pytest.raises(ValueError):
            bdr.mx_gemv(bdr.MX6, w, n, 32, x, y)               # the last one: not on a GPU
    with pytest.raises(ValueError):
        bdr.KVCache(bdr.MX6, bdr.MX6, w, w, 3, 4, 1, 32)       # planes of 8 lines for 12 slots
    c = bdr.KVCache(bdr.MX6, bdr.MX6, w, w, 2, 4, 1, 32)
    with pytest.raises(ValueError):
        bdr.mx_kv_append(c, t(1, 1, 32), t(1, 1, 32), torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError):
        bdr.mx_attn_decode(c, t(1, 2, 32), torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), t(1, 2, 32), u8(64))
    assert bdr.mx_attn_decode_workspace_bytes(c, 1, 2) > 0


def test_a_replaced_plane_is_described_anew():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    w = bdr.Planes(u8(8, 16), u8(8, 16), u8(8, 32))
    assert w.c().ld_elems == 32 and w.lines() == 8 and w.c() is w.c()
    w.elems = u8(6, 48)
    assert w.c().ld_elems == 48 and w.c().elems == w.elems.data_ptr() and w.lines() == 6


def test_slots_of_positions():
    table = torch.tensor([[5, 2, 9], [0, 7, 1]], dtype=torch.int32)
    assert decode.slots_of(table, torch.tensor([4, 11], dtype=torch.int32), 4).tolist() == [8, 7]
    assert decode.slots_of(table, torch.tensor([0, 3]), 4).tolist() == [20, 3]
