"""mx_attn_decode: how exactly the softmax weights and the scores enter, with bounds that a missing part of either would break.

bf16 queries.  The weights enter the second product as two bf16 parts: what is left of a weight after rounding to eight
significant bits twice is at most 2^-16 of it.  The queries are small, so the scores' own errors are, too: with the notation of the
operator's other test (score sums (d / 16 + 16) 2^-22 sum |q k|, exponent 2^-22 (12 + 2 max |score|), sums (n / 16 + 64) 2^-22)
    |error| <= 1.1 A (2 dw + 2^-16 + (n / 16 + 64) 2^-22) + 2^-8 (|result| + that),
where the last term is the rounding of the bf16 result.  Weights held in one bf16 part (2^-8) are ten times above it where a result is
small against A.

fp32 queries.  Queries and weights enter as three parts: the queries exactly, the weights to 2^-24.
  One position: the result is the value itself, and the log-sum is the score.  A score is a sum of d / 32 pieces (one at least); a piece
  is a chain of two instructions on the largest parts, each off by 2^-22 of what it has summed, and adding up to four pieces rounds by 2^-24
  each: 3 2^-22 |scale| sum |q k| for up to 128 elements.  The scale (four roundings on its way to base 2 and back) adds 4 2^-24 |score|.
  Queries in two parts would be 2^-17 sum |q k| off at most, ten times that.
  Two positions: the larger weight is 1 before the division, the other one is off by 2^-22 (the approximate exponential) + the difference
  of two scores' errors + 2^-24 (its three parts); this enters numerator and sum; the product adds 2^-22, the sum, the division, the
  multiplication and the joins of empty partners 4 2^-24:  |error| <= A (2 dw + 2^-22 + 2^-22),  dw = 2^-22 + 2 ds + 2^-24.
  Two parts of the weights would be 2^-17 off."""
import numpy as np
import pytest
import torch

from oracle import oracle as orc
from paper_2302_08007_b200 import binding as bdr
from tests import helpers as H
from tests.test_gpu_attn_decode import Case

pytestmark = pytest.mark.gpu


def exact(c, i):
    """Sequence i in 64 bits: scores and sums of their terms' magnitudes [n_q, n], weights, result, sum w |v|."""
    at, G = c.slots(i), c.n_q // c.n_kv
    k, v = (orc.quant_dequant(H.to_orc(f), np.ascontiguousarray(x[at]), axis=1)[0].astype(np.float64).reshape(-1, c.n_kv, c.d)
            for f, x in ((c.fk, c.keys), (c.fv, c.vals)))
    q = c.q[i].astype(np.float64).reshape(c.n_kv, G, c.d)
    s = np.einsum("hgd,thd->hgt", q, k) * c.scale
    mag = np.einsum("hgd,thd->hgt", np.abs(q), np.abs(k)) * c.scale
    w = np.exp(s - s.max(-1, keepdims=True))
    w /= w.sum(-1, keepdims=True)
    out = np.einsum("hgt,thd->hgd", w, v).reshape(c.n_q, c.d)
    A = np.einsum("hgt,thd->hgd", w, np.abs(v)).reshape(c.n_q, c.d)
    flat = lambda x: x.reshape(c.n_q, -1)  # noqa: E731
    return flat(s), flat(mag), flat(w), out, A


def check_bf16(c, got):
    eps = 2.0 ** -22
    for i, n in enumerate(c.lens):
        s, mag, _, want, A = exact(c, i)
        dw = 2 * (c.d / 16 + 16) * eps * mag.max(-1, keepdims=True) + eps * (12 + 2 * np.abs(s).max(-1, keepdims=True))
        bound = 1.1 * A * (2 * dw + 2.0 ** -16 + (n / 16 + 64) * eps)
        bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        err = np.abs(got[i].astype(np.float64) - want)
        assert (err <= bound).all(), (i, n, int((err > bound).sum()), float((err / bound).max()))


@pytest.mark.parametrize("n_q,n_kv,d", [(8, 2, 128), (16, 4, 64), (24, 2, 128), (4, 1, 256), (5, 5, 80)])
@pytest.mark.parametrize("fk,fv", [(bdr.MX9, bdr.MX9), (bdr.MX6, bdr.MX6), (bdr.MX4, bdr.MX4)], ids=["99", "66", "44"])
def test_weights_of_bf16_queries(fk, fv, n_q, n_kv, d):
    c = Case(fk, fv, [20, 64, 131, 700], n_q, n_kv, d, spread=0.1)
    check_bf16(c, c.call()[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,d", [(8, 2, 128), (16, 4, 64), (8, 8, 16), (6, 3, 48)])
def test_one_position_gives_its_value_and_its_score(n_q, n_kv, d, dtype):
    c = Case(bdr.MX9, bdr.MX6, [1] * 40, n_q, n_kv, d, dtype)
    got, lse = c.call()
    for i in range(40):
        s, mag, _, want, _ = exact(c, i)
        assert np.array_equal(got[i], want.astype(np.float32))           # six bits: exact in either type
        ds = 3 * 2.0 ** -22 * mag[:, 0] + 4 * 2.0 ** -24 * np.abs(s[:, 0])
        if dtype == "bf16":                                              # one chain of d / 16 products, the reference lifted by 2^32
            ds = (d / 16 + 1) * 2.0 ** -22 * mag[:, 0] + 4 * 2.0 ** -24 * np.abs(s[:, 0]) + 2 * 64 * 2.0 ** -24
        assert (np.abs(lse[i] - s[:, 0]) <= ds).all(), (i, float((np.abs(lse[i] - s[:, 0]) / ds).max()))


@pytest.mark.parametrize("n_q,n_kv,d", [(8, 2, 128), (16, 4, 64), (8, 8, 16)])
def test_two_positions_of_32_bit_queries(n_q, n_kv, d):
    c = Case(bdr.MX9, bdr.MX9, [2] * 100, n_q, n_kv, d, "f32", spread=0.1)
    got, _ = c.call()
    for i in range(100):
        s, mag, _, want, A = exact(c, i)
        ds = 3 * 2.0 ** -22 * mag.max(-1, keepdims=True) + 4 * 2.0 ** -24 * np.abs(s).max(-1, keepdims=True)
        bound = A * (2 * (2.0 ** -22 + 2 * ds + 2.0 ** -24) + 2 * 2.0 ** -22)
        err = np.abs(got[i].astype(np.float64) - want)
        assert (err <= bound).all(), (i, int((err > bound).sum()), float((err / bound).max()))
