"""Edges of the trunk's entry points that need no GPU: workspaces, sizes, types, what the documentation says."""
import pytest
import torch

from test_tokens_abi import gs, refused  # noqa: F401 (gs: a fixture)
from test_trunk_abi import recur


@pytest.mark.parametrize("n,cols", [(257, 1), (4000, 64), (4000, 129), (400_000, 2048)])
def test_recurrence_workspace_holds_lines_of_its_own(gs, n, cols):
    """Any 16-byte aligned workspace is taken, and the chunks' maps and the groups' states in it start at a line: there is
    room to move up to one."""
    up = lambda b: -(-b // 256) * 256
    chunks, width = -(-n // 128), 126 if cols % 128 == 1 and cols > 1 else 128
    groups, blocks = -(-chunks // 16), -(-cols // width)
    regions = up(chunks * blocks * 64 * 16) + up(groups * blocks * 64 * 16) + up(groups * blocks * 64 * 8) \
        + up((chunks + groups + 32) * blocks * 4)
    assert gs.gs_recurrence_ws_bytes(recur(gs, n=n, cols=cols, ld_x=cols, ld_gate=cols, n_seg=1)) >= regions + 240


def test_recurrence_of_one_chunk_needs_no_workspace(gs):
    assert gs.gs_recurrence_ws_bytes(recur(gs, n=256, n_seg=1)) == 0
