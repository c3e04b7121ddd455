"""Tie rules of the serving calls: mx_gemv only decodes and takes either, the calls on a cache take ties to even."""
from paper_2302_08007_b200 import binding as bdr
from tests.test_serving_cpu import NULL, UNSUPPORTED, append, attend, cache, gemv


def test_either_tie_rule_of_packed_weights():
    away = bdr.Config(16, 8, 2, 1, 4, bdr.SCALE_POW2, bdr.ROUND_NEAREST_AWAY)
    assert gemv(cfg=away, y=None) == NULL and gemv(cfg=away, T=0) == 0
    assert append(c=cache(cfg_k=away.c())) == UNSUPPORTED and attend(c=cache(cfg_v=away.c())) == UNSUPPORTED
