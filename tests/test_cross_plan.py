"""The plans of the gradients of attention to other states, by the workspaces they ask for (no
GPU).  dk and dv pass over tiles of 32 positions of one query head of one batch entry, however
few positions the last of them has."""
import pytest

from paper_2606_28560_amd import fibattn as F


def _bytes(B, H, Hkv, T, S, D):
    return F.fibattn_cross_backward_workspace_bytes(B, 1, H, Hkv, T, S, D)


@pytest.mark.parametrize("B,H,Hkv,D", [(64, 8, 8, 64), (64, 16, 4, 128), (96, 8, 1, 64), (7, 4, 2, 32), (200, 1, 1, 128)])
def test_pieces_go_by_tiles_not_by_rows(B, H, Hkv, D):
    # one row of 32 states, so dq has no pieces, and the statistics take as much for 1 position as for 32
    for T0, T1 in ((1, 32), (7, 32), (33, 64), (65, 96)):
        assert _bytes(B, H, Hkv, T0, 32, D) == _bytes(B, H, Hkv, T1, 32, D), (T0, T1)


def test_many_sequences_of_one_token_fill_the_gpu():
    # 64 sequences of one token over 256 shared rows: 64 tiles of queries for each of the 8 problems
    # of 8 tiles of states, 64 workgroups; in one piece three quarters of 256 CUs would be idle
    B, H, S, D = 64, 8, 256, 64
    stats = 4 * 64 * B * H
    k = 4 * H * S * D
    assert _bytes(B, H, H, 1, S, D) >= stats + 2 * 2 * k
