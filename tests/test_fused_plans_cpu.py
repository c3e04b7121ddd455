"""How the fused operators' calls are shared out, over sizes from one to the largest: host arithmetic, no GPU is used."""
from paper_2302_08007_b200 import binding as bdr


def test_no_part_of_a_vocabulary_is_longer_than_what_it_is_taken_from():
    # 37633 rows, 255 columns and a reduction of 131616: one part of 256 columns was decoded
    assert bdr.bdr_selftest_host() == 0
