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
