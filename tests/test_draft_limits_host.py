"""Bounds and refusals of the drafted-token calls that need no GPU: sizes beyond a launch, scratch, arrays that do not fit."""
import pytest
import torch

from paper_2507_21276_amd import binding as Bd

P = 1 << 20   # an address that no call here may reach: every one of them is refused before its launch


def tree(T, B, max_nodes, h, hk, dh, page=16, ptr=P):
    Bd._check(Bd.lib().lsk_attn_tree(ptr, h * dh, Bd.LS_F16, T, B, max_nodes, h, hk, dh, P, P, P, P, P, P, 4, page, 100, 50, ptr, h * dh,
                                     None, 0, None))


def test_more_workgroups_than_a_launch_counts_are_refused():
    with pytest.raises(Bd.LsError, match="too many"):
        tree(1 << 24, 1 << 22, 256, 4, 4, 64)              # 2^22 requests x 4 key heads x 2 blocks of 128 rows
    with pytest.raises(Bd.LsError, match="too many"):
        tree(1 << 24, 1 << 20, 4, 64, 16, 128)             # 2^24 pairs of one block
    with pytest.raises(Bd.LsError, match="too many"):
        tree(1 << 24, 3, 4, 2, 2, 80)                      # the kernel for any size: a workgroup a row and head
    with pytest.raises(Bd.LsError, match="too many"):
        Bd._check(Bd.lib().lsk_tree_index(P, P, P, (1 << 24) - 1, 1 << 24, 4, P, P, P, P, None))


def test_scratch_of_the_tree_attention_is_bounded():
    need = Bd.lib().lsk_attn_tree_scratch_floats
    row = 32 * (128 + 4)
    for args in ((16384, 64, 32, 32, 128, 256, 131072), (4096, 64, 32, 32, 128, 64, 32768), (65536, 256, 32, 32, 128, 256, 131072),
                 (1, 1, 32, 32, 128, 1, 1 << 20)):
        n = need(*args)
        assert n <= 1 << 28 and n % (args[0] * row) == 0 and n != args[0] * row
    assert need(16384, 64, 32, 32, 128, 256, 131072) == 3 * 16384 * row           # as many parts as fit
    assert need(65536, 256, 32, 32, 128, 256, 131072) == 0                        # one part: no partial results
    assert need(4096, 64, 32, 32, 128, 64, 32768) == 8 * 4096 * row               # within the bound: all of them
    # sizes whose kernel does not split a context
    assert need(8, 1, 8, 8, 256, 8, 4096) == need(8, 1, 8, 8, 80, 8, 4096) == 0 < need(8, 1, 8, 8, 128, 8, 4096)
