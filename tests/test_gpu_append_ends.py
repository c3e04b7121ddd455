"""mx_kv_append at the ends of its tables: positions that no table row has."""
import numpy as np
import pytest
import torch

from paper_2302_08007_b200 import binding as bdr
from tests import helpers as H
from tests.test_gpu_kv_append import dev

pytestmark = pytest.mark.gpu


def prepared(t, n_kv, d, dtype):
    x = H.make_input("normal", t, 3 * n_kv * d, dtype, seed=4).reshape(t, 3 * n_kv, d)
    cache = bdr.alloc_kv_cache(bdr.MX6, bdr.MX9, 2, 4, n_kv, d)
    for pl in (cache.k, cache.v):
        for p in (pl.exps, pl.micro, pl.elems):
            p.fill_(0xA5)
    return cache, [dev(x[:, i * n_kv:(i + 1) * n_kv], dtype) for i in range(3)]


def untouched(cache):
    return [bool((p == 0xA5).all()) for pl in (cache.k, cache.v) for p in (pl.exps, pl.micro, pl.elems)] == [True] * 6


@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("rot", [32, 20])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tables_without_a_row_are_not_read(dtype, rot, interleaved):
    cache, (q, k, v) = prepared(5, 2, 32, dtype)
    q_out, k_dq, v_dq = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    none = torch.empty((0, rot // 2), dtype=torch.float32, device="cuda")
    bdr.mx_kv_append(cache, k, v, torch.arange(5, device="cuda"), torch.arange(5, device="cuda"), none, none, interleaved=interleaved, q=q, q_out=q_out,
                     k_dq=k_dq, v_dq=v_dq)
    torch.cuda.synchronize()
    assert bdr.bdr_device_status_reset() == -5
    assert untouched(cache) and bool(torch.isnan(q_out).all()) and bool(torch.isnan(k_dq).all())
    assert np.isfinite(H.device_to_host_f32(v_dq)).all()


def test_padding_tokens_with_positions_out_of_range_are_not_errors():
    cache, (q, k, v) = prepared(3, 2, 32, "bf16")
    ang = torch.rand((4, 16), device="cuda")
    q_out = torch.empty_like(q)
    bdr.mx_kv_append(cache, k, v, torch.tensor([-1, 6, -7], device="cuda"), torch.tensor([-1, 3, 4], device="cuda"), ang.cos(), ang.sin(), q=q, q_out=q_out)
    torch.cuda.synchronize()
    assert bdr.bdr_device_status_reset() == 0
    assert torch.isnan(q_out).flatten(1).all(1).tolist() == [True, False, True]
    assert (cache.k.elems != 0xA5).any(1).nonzero().flatten().tolist() == [6]
    bdr.mx_kv_append(cache, k, v, torch.tensor([-1, 6, 2], device="cuda"), torch.tensor([-1, 3, 4], device="cuda"), ang.cos(), ang.sin())
    torch.cuda.synchronize()
    assert bdr.bdr_device_status_reset() == -5 and bool((cache.k.elems[2] == 0xA5).all())
