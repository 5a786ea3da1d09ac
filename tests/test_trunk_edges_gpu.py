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


# -- layer norm near the ends of fp32's range ----------------------------------------


@pytest.mark.parametrize("size,eps", [(1e17, 1e-5), (1e18, 1e-5), (1e20, 1e-5), (1e35, 1e-5), (1e25, 0.0), (1e-11, 0.0),
                                      (1e-18, 0.0), (1e-25, 0.0), (1e-35, 0.0), (1e-18, 1e-36), (1e-13, 1e-31)])
@pytest.mark.parametrize("cols", [7, 128, 250, 500, 1001, 1400, 2000, 3000, 9000])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_layer_norm_of_rows_whose_squares_do_not_fit(tk, dtype, cols, size, eps):
    """Beside ordinary rows, with which they share waves: y, dx and the weights' gradients."""
    g = gen(cols)
    x, r, dy, dt = (randn(g, 6, cols) for _ in range(4))
    x[1::2] *= size
    r[1::2] *= size
    x, r, dy, dt = (t.to(dtype) for t in (x, r, dy, dt))
    w, b = 1 + randn(g, cols), randn(g, cols)
    for res in (None, r):
        y, _, bound = ref.layer(x, w, b, eps, res)
        within(tk.layer_norm(x, w, b, eps, residual=res).y, y, bound, "y")
    for extra in (None, dt):
        want, bounds = ref.layer_bwd(dy, x, w, eps, extra)
        for got, v, e, what in zip(tk.layer_norm_backward(dy, x, w, eps, dtotal=extra), want, bounds, ("dx", "dweight", "dbias")):
            within(got, v, e, what)


def test_layer_norm_at_the_end_of_the_range(tk):
    """Differences of the largest numbers are normed; a sum, or a difference, past the range makes its row NaN and no other."""
    x = torch.full((4, 64), 3e38, device="cuda")
    x[0, ::2] *= -1                                    # mean 0
    x[2, 1:] = -1e37                                   # a difference of 3.4e38 and more
    x[2, 0] = 3.4e38
    x[3] = torch.arange(64, device="cuda")
    w, b = torch.ones(64, device="cuda"), torch.zeros(64, device="cuda")
    y = tk.layer_norm(x, w, b).y
    # the reciprocal root is below the normal numbers, 2^-128.2: half a step of 2^-149 is 2^-21.8 of it
    assert float((y[0] - x[0] / 3e38).abs().max()) <= 2.0 ** -20
    assert bool(y[1].isnan().all()) and bool(y[2].isnan().all())
    want, _, bound = ref.layer(x[3:], w, b, 1e-5)
    within(y[3:], want, bound, "an ordinary row")
