"""decode.slots_of at the ends of the page table: nothing is looked up outside it."""
import torch

from paper_2302_08007_b200 import decode


def test_positions_outside_the_page_table():
    table = torch.tensor([[5, 2, 9], [0, 7, 1], [3, 3, 3], [4, 6, 8], [5, 2, 9]], dtype=torch.int32)
    for dtype in (torch.int32, torch.int64):
        got = decode.slots_of(table, torch.tensor([12, -1, 2 ** 31 - 1, -2 ** 31, 11], dtype=dtype), 4).tolist()
        # beyond the table: beyond every cache (n_pages * page_size < 2^31); negative: padding; the last position that the table covers
        assert got[0] >= 2 ** 31 and got[1] < 0 and got[2] >= 2 ** 31 and got[3] < 0 and got[4] == 39


def test_a_page_table_without_pages():
    got = decode.slots_of(torch.zeros((3, 0), dtype=torch.int32), torch.tensor([0, -2, 7], dtype=torch.int32), 16).tolist()
    assert got[0] >= 2 ** 31 and got[1] < 0 and got[2] >= 2 ** 31
