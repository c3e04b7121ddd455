"""How the fused operators' calls are shared out, over sizes from one to the largest: host arithmetic, no GPU is used."""
import itertools
import os
import re

from paper_2302_08007_b200 import binding as bdr
from paper_2302_08007_b200 import head


def test_no_part_of_a_vocabulary_is_longer_than_what_it_is_taken_from():
    # 37633 rows, 255 columns and a reduction of 131616: one part of 256 columns was decoded
    assert bdr.bdr_selftest_host() == 0


def test_sizes_of_workspaces_of_nothing():
    # what the calls accept has a workspace; what they refuse has none
    L = bdr.lib()
    gated = (lambda *s: L.mx_gated_gemm_workspace_bytes(*s), lambda *s: L.mx_gated_gemm_bwd_workspace_bytes(*s, 0), lambda *s: L.mx_gated_gemm_bwd_workspace_bytes(*s, 1))
    entropy = (lambda *s: L.mx_cross_entropy_workspace_bytes(*s), lambda *s: L.mx_cross_entropy_bwd_workspace_bytes(*s, 0),
               lambda *s: L.mx_cross_entropy_bwd_workspace_bytes(*s, 1))
    for m, n, k in itertools.product((0, 1, 256, 1000), (0, 1, 256, 1000), (0, 1, 64, 4096)):
        for query in gated:
            assert (query(m, n, k) > 0) == (k > 0)
        for query in entropy:
            assert (query(m, n, k) > 0) == (n > 0 and k > 0)


def test_buffers_of_no_tokens():
    for cfg in (bdr.MX6, bdr.MX9):
        buf = head.alloc(cfg, 0, 300, 64, device="cpu")
        assert buf.workspace.numel() > 0 and buf.d_weight.shape == (300, 64)


def test_a_reduction_longer_than_the_reencoding_takes_has_no_space_for_it():
    # MX4 / MX6 operands of more than 65535 x 1024 elements a line stay on the bf16 path: the 8-bit one would refuse them half way through the call
    L, most = bdr.lib(), 65535 * 1024
    for query, args in ((L.mx_gated_gemm_bwd_workspace_bytes, (256, 128)), (L.mx_cross_entropy_bwd_workspace_bytes, (256, 256))):
        assert query(*args, most + 1024, 1) < query(*args, most, 1)
        assert query(*args, most, 1) > query(*args, most - 1, 1) + 256 * most


def test_the_lanes_of_a_role_get_one_answer_from_a_wait():
    # The warps of the fused kernels issue with elect.sync: a lane that left its loop alone, because its own polls of a bounded wait ran out, would keep
    # the others waiting for good.  Making a wait run out in the middle of a phase is no test for a GPU, so the source is looked at: only the waits behind
    # a failure, whose answers nobody reads, are each lane's own.
    for name in ("mx_fused_gemm.cuh", "mx_fused_f8.cuh"):
        with open(os.path.join(os.path.dirname(bdr.__file__), "csrc", name)) as f:
            waits = [line.strip() for line in f if re.search(r"\bmbar_wait\w*\(", line)]
        assert len(waits) >= 6
        assert all("mbar_wait_warp(" in w or w.startswith("if (s < stage || turn > 0) mbar_wait(") for w in waits), waits
