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


# -- infinite states --------------------------------------------------------------------


def walked(x, gate, dy, cu, initial, dfinal, reverse):
    """y, final, dx, dgate and dinitial token by token in double, on the CPU."""
    x, gate, dy, initial, dfinal = (t.double().cpu() for t in (x, gate, dy, initial, dfinal))
    a, z = torch.sigmoid(gate), torch.sigmoid(-gate)
    y, before, final, dx, dg, di = (torch.zeros_like(t) for t in (x, x, initial, x, x, initial))
    for s, (lo, hi) in enumerate(zip(cu, cu[1:])):
        order = range(hi - 1, lo - 1, -1) if reverse else range(lo, hi)
        h = initial[s]
        for t in order:
            before[t], h = h, a[t] * h + z[t] * x[t]
            y[t] = h
        final[s], D = h, dfinal[s]
        for t in reversed(order):
            D = D + dy[t]
            dx[t], dg[t], D = z[t] * D, a[t] * z[t] * (before[t] - x[t]) * D, a[t] * D
        di[s] = D
    return y, final, dx, dg, di


def alike(got, want, what):
    """Infinite with the same sign, NaN and finite at the same places."""
    got = got.double().cpu()
    for sort in (torch.isposinf, torch.isneginf, torch.isnan):
        assert torch.equal(sort(got), sort(want)), (what, sort.__name__, int((sort(got) != sort(want)).sum()))


@pytest.mark.parametrize("n,cu", [(40, [0]), (250, [0, 90]), (300, [0, 100]), (9000, [0, 130, 2600, 4096])])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_infinite_states_stay_infinite(tk, n, cu, reverse, dtype):
    """Through runs of gates whose product is 0 in fp32: what they are token by token, and the other channels' bits as they
    are without them."""
    cu = cu + [n]
    g = gen(31 + n)
    x, dy = randn(g, n, 7, dtype=dtype), randn(g, n, 7, dtype=dtype)
    gate = (-8 + 4 * torch.rand(n, 7, generator=g, device="cuda")).to(dtype)
    first, last = randn(g, len(cu) - 1, 7), randn(g, len(cu) - 1, 7)
    clean = tk.recurrence(x, gate, cu=starts(cu), initial=first, reverse=reverse, keep=True)
    grads = tk.recurrence_backward(dy, x, gate, clean.kept, cu=starts(cu), initial=first, dfinal=last, reverse=reverse)
    for lo, hi in zip(cu, cu[1:]):
        near, mid, far = lo + 3, (lo + hi) // 2, hi - 4
        x[far if reverse else near, 1] = dy[near if reverse else far, 1] = math.inf
        x[far if reverse else near, 2] = dy[near if reverse else far, 2] = -math.inf
        x[mid, 2] = dy[mid, 2] = math.inf              # with the infinity of the other sign: NaN from here on
        x[mid, 3] = -math.inf
        dy[mid, 4] = -math.inf
    first[:, 5] = math.inf
    last[:, 6] = -math.inf
    got = tk.recurrence(x, gate, cu=starts(cu), initial=first, reverse=reverse, keep=True)
    back = tk.recurrence_backward(dy, x, gate, got.kept, cu=starts(cu), initial=first, dfinal=last, reverse=reverse)
    want = walked(x, gate, dy, cu, first, last, reverse)
    for a, b, what in zip((got.y, got.final, *back), want, ("y", "final", "dx", "dgate", "dinitial")):
        alike(a, b, what)
    for c in (0, 4, 6):
        assert torch.equal(got.y[:, c], clean.y[:, c]) and torch.equal(got.final[:, c], clean.final[:, c])
    for c in (0, 3, 5):
        assert torch.equal(back[0][:, c], grads[0][:, c]) and torch.equal(back[2][:, c], grads[2][:, c])
    assert torch.equal(back[1][:, 0], grads[1][:, 0])


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("n", [40, 250, 9000])
def test_a_gate_of_zero_leaves_nothing_of_the_state(tk, n, reverse):
    """Of a finite state, whatever the gates around it: exactly 0 where the tokens are; nor of a gradient."""
    g = gen(n)
    gate = -12 * torch.rand(n, 6, generator=g, device="cuda")
    at = n // 3
    gate[at, :3] = -math.inf
    zero, first = torch.zeros(n, 6, device="cuda"), torch.full((1, 6), 1e30, device="cuda")
    r = tk.recurrence(zero, gate, initial=first, reverse=reverse, keep=True)
    behind = slice(0, at + 1) if reverse else slice(at, n)
    assert bool((r.y[behind, :3] == 0).all()) and bool((r.final[0, :3] == 0).all())
    dx, _, di = tk.recurrence_backward(zero, zero, gate, r.kept, initial=first, dfinal=first, reverse=reverse)
    front = slice(at + 1, n) if reverse else slice(0, at)
    assert bool((dx[front, :3] == 0).all()) and bool((di[0, :3] == 0).all())


# -- long sums ---------------------------------------------------------------------------


@pytest.mark.parametrize("tokens,rows,dim", [(400_000, 1, 512), (400_001, 3, 200), (16_000_000, 1, 64), (30_000_000, 2, 5)])
@pytest.mark.parametrize("value", [0.1, 0.7])
def test_embedding_gradient_of_very_many_tokens_a_row(tk, tokens, rows, dim, value):
    """Equal numbers, whose roundings do not cancel: as near as the sums of a few tokens."""
    dout = torch.full((tokens, dim), value, device="cuda")
    ids = (torch.arange(tokens, device="cuda") * rows // tokens).int()
    count = torch.bincount(ids.long(), minlength=rows)[:, None]
    want = (count.double() * float(dout[0, 0]) * 1.5).expand(rows, dim)
    # 64 tokens in fp32, 64 and one of their sums in fp32, those in 64 bits, rounded once, the product with the scale
    bound = (64 + 65 + 2) * ref.F * want
    got = tk.embedding_backward(dout, ids, rows, 1.5)
    within(got, want, bound, "grad")
    unique, n, touched = tk.embedding_rows(dout, ids, rows, 1.5)
    assert int(n) == rows and torch.equal(touched, got)


# -- kept values beside a block's largest -----------------------------------------------


@pytest.mark.parametrize("dtype", [F32, BF])
def test_kept_values_beside_large_ones(tk, dtype):
    """As far off as the documentation says: a 16th, or 2^-10 of the block's power of two; not always a 16th."""
    g = gen(41)
    u = (randn(g, 300, 64) * torch.exp(-14 * torch.rand(300, 64, generator=g, device="cuda"))).to(dtype)
    u[:, 7], u[:, 40] = 448.0 * 2.0 ** -3, -300.0
    r = tk.gated_silu(u, u)
    power = torch.exp2(r.u_scale.double() - 127).repeat_interleave(32, 1)
    top = u.double().abs().view(300, 2, 32).amax(2).repeat_interleave(32, 1)
    assert bool((power <= top / 224).all())
    x, back = u.double().abs(), ref.wide(r.u8, r.u_scale)
    off = (back - u.double()).abs()
    assert bool((off <= torch.maximum(x / 16, power * 2.0 ** -10)).all())
    assert bool((off <= x / 16)[x >= top / 14336].all()) and bool((off > x / 16).any())
    assert bool((back != 0)[x > top / 229376].all()) and bool((back == 0)[x > 0].any())
    # the gradient is that at the kept values
    dh = randn(g, 300, 64, dtype=dtype)
    du, dv, _ = tk.gated_silu_backward(dh, r.u8, r.u_scale, r.v8, r.v_scale)
    want, bounds = ref.silu_bwd(dh, back, back)
    within(du, want[0], bounds[0], "du")
    within(dv, want[1], bounds[1], "dv")


@pytest.mark.parametrize("dtype", [F32, BF])
def test_gated_silu_gradient_far_out(tk, dtype):
    """Against the formula at the kept values, a value a block: on the negative side down to the least numbers, on the
    positive side the factor alone."""
    u = torch.tensor([-1e30, -1e4, -200.0, -120.0, -100.0, -90.0, -75.0, -60.0, 60.0, 75.0, 90.0, 120.0, 1e4, 1e30])
    x, f, d = torch.zeros(14, 32, device="cuda", dtype=dtype), torch.zeros(14, 32, device="cuda", dtype=dtype), torch.ones(14, 32)
    x[:, 0], f[:, 0] = u.to(dtype).cuda(), -3e4
    d = (d * 1.5).to(dtype).cuda()
    r = tk.gated_silu(x, f)
    got = tk.gated_silu_backward(d, r.u8, r.u_scale, r.v8, r.v_scale)
    U, V = ref.wide(r.u8, r.u_scale)[:, 0], ref.wide(r.v8, r.v_scale)[:, 0]
    s, rest = torch.sigmoid(U), torch.sigmoid(-U)
    want = (1.5 * V * (s + U * s * rest), 1.5 * U * s, U * s * V)
    # exp's rounded argument counts where it is not lost beside 1: up to |u| = 104, behind which fp32 holds nothing
    c = torch.where(U < 0, 14 + 2 * U.abs().clamp(max=110), 14.0) * ref.F + ref.UNIT[dtype]
    for t, w, what in zip(got, want, ("du", "dv", "h")):
        within(t[:, 0], w, c * w.abs() + 2.0 ** -147 * 1e5, what)
        assert bool((t[:, 1:] == 0).all()), what
