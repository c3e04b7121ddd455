"""mx_gemv of 3-bit codes with 9 to 16 columns on both sides of the limits at which it changes its number of warps: activations that fit in shared
memory beside the rings of both numbers, of one, of neither, with two row tiles per SM and with more.  The bound is that of the operator's
other test."""
import pytest
import torch

from paper_2302_08007_b200 import binding as bdr
from tests import helpers as H
from tests.test_gpu_gemv import check, make, packed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [75, 4736, 4740])
@pytest.mark.parametrize("t,k,dtype", [(16, 4096, "bf16"), (16, 4100, "bf16"), (16, 5632, "bf16"), (16, 5640, "bf16"), (9, 8960, "bf16"), (9, 9730, "bf16"),
                                       (5, 4352, "f32"), (5, 5999, "f32"), (3, 9000, "f32")])
def test_products_around_the_limits(t, k, dtype, n):
    w, x = make(n, k, t, k + n, dtype)
    planes, w_dq = packed(bdr.MX4, w)
    y = torch.empty((t, n), dtype=torch.float32, device="cuda")
    bdr.mx_gemv(bdr.MX4, planes, n, k, H.host_to_device(x, dtype), y)
    check(y, x, w_dq, k, "f32")
    again = bdr.mx_gemv(bdr.MX4, planes, n, k, H.host_to_device(x, dtype), torch.empty_like(y))
    assert torch.equal(again, y)
