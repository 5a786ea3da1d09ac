"""Edges of the trunk's operators: workspaces at any alignment that is allowed, values near the ends of fp32's range,
infinities, long sums."""
import math

import pytest
import torch

import trunk_refs as ref
from test_tokens_gpu import BF, F32, HF, gen, gs, randn, tk, within  # noqa: F401 (gs, tk: fixtures)
from test_trunk_gpu import starts

pytestmark = pytest.mark.gpu


# -- workspaces ----------------------------------------------------------------------


@pytest.mark.parametrize("at", [0, 16, 64, 112, 240, 256 + 16])
@pytest.mark.parametrize("n,cols,segments", [(300, 5, 1), (9000, 130, 3), (70_000, 257, 1)])
def test_recurrence_in_a_workspace_at_any_alignment(tk, gs, n, cols, segments, at):
    """The bits of a workspace that starts at a line; nothing behind its end is written."""
    g = gen(n + cols)
    x, gate, dy = (randn(g, n, cols, dtype=BF) for _ in range(3))
    gate = gate + 3                                    # states that reach over chunks
    cu = starts([0] + sorted(int(n * (s + 0.37) / segments) for s in range(segments - 1)) + [n])
    want = tk.recurrence(x, gate, cu=cu, keep=True)
    grads = tk.recurrence_backward(dy, x, gate, want.kept, cu=cu)
    r = gs.make_recur(x, gate, cu)
    need = gs.gs_recurrence_ws_bytes(r)
    room = torch.full((at + need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    assert room.data_ptr() % 256 == 0
    ws = room[at:at + need]
    for _ in range(3):
        y, final, kept = torch.empty_like(x), torch.empty_like(want.final), torch.empty_like(want.kept)
        gs.gs_recurrence(r, y, final, kept, ws)
        assert torch.equal(y, want.y) and torch.equal(final, want.final) and torch.equal(kept, want.kept)
        dx, dg = torch.empty_like(x), torch.empty_like(x)
        gs.gs_recurrence_bwd(r, dy, kept, dx, dg, ws=ws)
        assert torch.equal(dx, grads[0]) and torch.equal(dg, grads[1])
    assert bool((room[:at] == 0x5A).all()) and bool((room[at + need:] == 0x5A).all())
