"""The operators of a linear-cost trunk through the package's functions against plain 64-bit forms: layer norm,
embedding, gated recurrence and the gated SiLU kept in 8 bits.  Every tolerance is a bound derived from the roundings
that the operator makes (trunk_refs), not a measured one."""
import math

import pytest
import torch

import trunk_refs as ref
from test_tokens_gpu import BF, F32, HF, gen, gs, randn, tk, within  # noqa: F401 (gs, tk: fixtures)

pytestmark = pytest.mark.gpu
TYPES = [F32, BF, HF]


def say(*a):
    print(*a, flush=True)


# -- layer norm --------------------------------------------------------------------

LAYERS = [(1, 1), (1, 8), (3, 7), (5, 128), (4, 129), (7, 1024), (9, 1025), (6, 1001), (5, 1536), (3, 2048), (2, 2056),
          (2, 4099), (2, 5000), (3, 8200), (2, 16384), (2, 16381), (0, 64), (515, 72), (1001, 250), (37, 16), (70, 256)]


@pytest.mark.parametrize("rows,cols", LAYERS)
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm(tk, rows, cols, dtype):
    g = gen(rows * 7919 + cols)
    x, r = randn(g, rows, cols, dtype=dtype) * 3 + 2, randn(g, rows, cols, dtype=dtype)
    w, b = 1 + randn(g, cols), randn(g, cols)
    for res, bias in ((None, b), (r, b), (r, None)):
        got = tk.layer_norm(x, w, bias, 1e-5, residual=res)
        y, s, bound = ref.layer(x, w, bias, 1e-5, res)
        within(got.y, y, bound, "y")
        if res is None:
            assert got.total is x
        else:
            assert torch.equal(got.total, (x.float() + r.float()).to(dtype))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_layer_norm_of_special_rows(tk, dtype):
    """A constant row is its bias, a large mean costs the mean's rounding alone, NaN and infinities stay in their row."""
    g = gen(3)
    x = randn(g, 6, 300)
    x[0] = 5.0
    x[1] += 1000.0
    x[2] = 0.0
    x[3, 7] = math.nan
    x[4, 250] = math.inf
    x = x.to(dtype)
    w, b = 1 + randn(g, 300), randn(g, 300)
    got = tk.layer_norm(x, w, b, 1e-5).y
    assert torch.equal(got[0], b.to(dtype)) and torch.equal(got[2], b.to(dtype))
    y, _, bound = ref.layer(x, w, b, 1e-5)
    for row in (1, 5):
        within(got[row], y[row], bound[row], "row")
    assert bool(got[3].isnan().all()) and bool(got[4].isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_strides_and_in_place(tk, gs, dtype):
    g = gen(5)
    wide = randn(g, 33, 1500, dtype=dtype)
    wb = randn(g, 2 * 1500 + 3)
    for off, cols in ((0, 96), (1, 96), (3, 101), (5, 1001), (7, 1400)):
        x, w, b = wide[:, off:off + cols], wb[1:1 + cols], wb[1502:1502 + cols]
        y, _, bound = ref.layer(x, w, b, 1e-5)
        within(tk.layer_norm(x, w, b, 1e-5).y, y, bound, "strided x")
        dx, dw, db = tk.layer_norm_backward(x, wide[:, off + 2:off + 2 + cols], w, 1e-5, dtotal=x)
        want, bounds = ref.layer_bwd(x, wide[:, off + 2:off + 2 + cols], w, 1e-5, x)
        for got, a, e, what in zip((dx, dw, db), want, bounds, ("dx", "dweight", "dbias")):
            within(got, a, e, what)
    x, r, w = randn(g, 40, 259, dtype=dtype), randn(g, 40, 259, dtype=dtype), 1 + randn(g, 259)
    want = tk.layer_norm(x, w, w, 1e-5, residual=r)
    dy = randn(g, 40, 259, dtype=dtype)
    grads = tk.layer_norm_backward(dy, want.total, w, 1e-5, dtotal=r)
    gs.gs_layer_norm(x, w, w, 1e-5, y=x, residual=r.clone(), total=None)
    assert torch.equal(x, want.y)
    dw, db = torch.empty_like(w), torch.empty_like(w)
    ws = torch.empty(gs.gs_layer_norm_bwd_ws_bytes(40, 259), dtype=torch.uint8, device="cuda")
    gs.gs_layer_norm_bwd(dy, want.total, w, 1e-5, dy, dw, None, ws, dtotal=r)
    assert torch.equal(dy, grads[0]) and torch.equal(dw, grads[1])


@pytest.mark.parametrize("rows,cols", [s for s in LAYERS if s[0]] + [(3000, 264), (2100, 2304), (700, 4500)])
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_backward(tk, rows, cols, dtype):
    g = gen(rows * 31 + cols)
    total, dy, dt = (randn(g, rows, cols, dtype=dtype) for _ in range(3))
    total = total + 1
    w = 1 + randn(g, cols)
    for extra in (None, dt):
        got = tk.layer_norm_backward(dy, total, w, 1e-5, dtotal=extra)
        want, bounds = ref.layer_bwd(dy, total, w, 1e-5, extra)
        for a, b, e, what in zip(got, want, bounds, ("dx", "dweight", "dbias")):
            within(a, b, e, what)
        again = tk.layer_norm_backward(dy, total, w, 1e-5, dtotal=extra)
        assert all(torch.equal(a, b) for a, b in zip(again, got))


@pytest.mark.parametrize("rows,cols", [(1, 24), (5, 128), (3, 250), (7, 500), (5, 700), (2, 1400), (3, 2000), (2, 3000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_without_epsilon(tk, rows, cols, dtype):
    """The rows that share a wave with the last ones, or lie behind them, add nothing to the weights' gradients."""
    g = gen(23)
    x, dy, w, b = randn(g, rows, cols, dtype=dtype), randn(g, rows, cols, dtype=dtype), randn(g, cols), randn(g, cols)
    want, _, bound = ref.layer(x, w, b, 0.0)
    within(tk.layer_norm(x, w, b, 0.0).y, want, bound, "y")
    grads, bounds = ref.layer_bwd(dy, x, w, 0.0)
    for got, v, e, what in zip(tk.layer_norm_backward(dy, x, w, 0.0), grads, bounds, ("dx", "dweight", "dbias")):
        within(got, v, e, what)


def test_layer_norm_backward_of_no_rows(tk):
    z = torch.zeros(0, 96, device="cuda")
    dx, dw, db = tk.layer_norm_backward(z, z, torch.ones(96, device="cuda"))
    assert dx.shape == (0, 96) and bool((dw == 0).all()) and bool((db == 0).all())


def test_layer_norm_backward_against_differences(tk):
    g = gen(11)
    x, w, dy, dt = randn(g, 6, 40), 1 + randn(g, 40), randn(g, 6, 40), randn(g, 6, 40)
    dx, dw, db = tk.layer_norm_backward(dy, x, w, 1e-3, dtotal=dt)

    def f(a, v, b):
        return float((ref.layer(a, v, b, 1e-3)[0] * dy.double()).sum() + (a * dt.double()).sum())

    zero = torch.zeros(40, dtype=torch.float64, device="cuda")
    ref.UNIT[torch.float64] = ref.TINY[torch.float64] = 0.0
    for _ in range(4):
        a, v, b, h = randn(g, 6, 40).double(), randn(g, 40).double(), randn(g, 40).double(), 1e-5
        num = (f(x.double() + h * a, w.double() + h * v, zero + h * b)
               - f(x.double() - h * a, w.double() - h * v, zero - h * b)) / (2 * h)
        got = float((dx.double() * a).sum() + (dw.double() * v).sum() + (db.double() * b).sum())
        size = float((dx.double() * a).abs().sum() + (dw.double() * v).abs().sum() + (db.double() * b).abs().sum())
        # the differences' own error (third derivative, h^2) and fp32 gradients
        assert abs(num - got) <= 1e-5 * size


# -- embedding -----------------------------------------------------------------------

EMBEDS = [(1, 1, 1), (5, 3, 7), (37, 10, 64), (300, 1000, 128), (1000, 7, 257), (64, 50, 1000), (9, 4, 4104),
          (3, 2, 16384), (5000, 300, 24), (257, 65, 33)]


@pytest.mark.parametrize("tokens,rows,dim", EMBEDS)
@pytest.mark.parametrize("table,out", [(F32, F32), (F32, BF), (F32, HF), (BF, BF), (HF, HF)])
def test_embedding(tk, tokens, rows, dim, table, out):
    g = gen(tokens + dim)
    t = randn(g, rows, dim, dtype=table)
    ids = torch.randint(-1, rows + 1, (tokens,), generator=g, device="cuda").int()
    ids[0] = rows - 1
    if tokens > 4:
        ids[1], ids[2], ids[3] = -2 ** 31, 2 ** 31 - 1, rows
    for scale in (1.0, -0.3):
        got = tk.embedding(t, ids, scale, out)
        there = (ids >= 0) & (ids < rows)
        want = torch.where(there[:, None], t.float()[ids.long().clamp(0, rows - 1)] * scale, 0.0).to(out)
        assert got.dtype == out and torch.equal(got, want)


def test_embedding_layouts(tk, gs):
    """Columns of wider matrices, at any alignment of an element; rows outside the output stay as they are."""
    g = gen(2)
    big = randn(g, 50, 301)
    ids = torch.randint(0, 50, (90,), generator=g, device="cuda").int()
    for off, dim in ((1, 64), (3, 101), (0, 300)):
        for dtype in (F32, BF):
            out = torch.full((92, 333), 7.0, device="cuda", dtype=dtype)
            gs.gs_embedding(big[:, off:off + dim], ids, 0.5, out[1:91, 5:5 + dim])
            assert torch.equal(out[1:91, 5:5 + dim], (big[:, off:off + dim][ids.long()] * 0.5).to(dtype))
            out[1:91, 5:5 + dim] = 7.0
            assert bool((out == 7.0).all())


def grad_of(dout, ids, rows, scale):
    """(gradient, bound, ids with a token) in double."""
    there = (ids >= 0) & (ids < rows)
    i, d = ids[there].long().cpu(), dout[there].double().cpu()
    want = torch.zeros(rows, dout.shape[1], dtype=torch.float64).index_add_(0, i, d) * scale
    size = torch.zeros(rows, dout.shape[1], dtype=torch.float64).index_add_(0, i, d.abs()) * abs(scale)
    count = torch.bincount(i, minlength=rows)[:, None]
    # a sum of `count` numbers in any order, and the product with the scale
    bound = (count.clamp(min=1) + 1) * ref.F * size + 1e-38
    return want.cuda(), bound.cuda(), torch.unique(i).int().cuda()


GRADS = [  # tokens, rows, dim, ids
    (1, 1, 1, "any"), (1, 100, 8, "any"), (33, 5, 16, "any"), (31, 5, 12, "one"), (100, 1000, 7, "any"),
    (4096, 300, 40, "any"), (4097, 300, 24, "any"), (5000, 1, 64, "any"), (20000, 50, 33, "few"), (9000, 9000, 8, "each"),
    (30000, 2000, 128, "few"), (3000, 1 << 20, 8, "any"), (8000, 1500000, 4, "any"), (700, 40, 1000, "any"),
    (300, 9, 4104, "any"), (64, 1023, 256, "any"), (64, 1024, 256, "any"), (6000, 1025, 20, "runs"), (2000, 64, 96, "none"),
    (1024, 5000, 8, "any"), (1025, 5000, 8, "any"), (2048, 70_000, 8, "runs"), (2049, 5000, 12, "any"), ((1 << 20) + 3, 3000, 8, "few")]


@pytest.mark.parametrize("tokens,rows,dim,how", GRADS)
@pytest.mark.parametrize("dtype", TYPES)
def test_embedding_gradient(tk, tokens, rows, dim, how, dtype):
    g = gen(tokens * 3 + rows + dim)
    say(tokens, rows, dim, how, dtype)
    ids = torch.randint(-1 if how == "any" else 0, rows + (how == "any"), (tokens,), generator=g, device="cuda")
    if how == "one":
        ids[:] = rows // 2
    if how == "few":                                   # most of the tokens in a few rows
        ids = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.9, ids % 3, ids)
    if how == "each":
        ids = torch.randperm(rows, generator=g, device="cuda")[:tokens]
    if how == "runs":
        ids = torch.arange(tokens, device="cuda") // 100
    if how == "none":
        ids[:] = -1
    ids = ids.int()
    dout = randn(g, tokens, dim, dtype=dtype)
    want, bound, unique = grad_of(dout, ids, rows, 1.7)
    got = tk.embedding_backward(dout, ids, rows, 1.7)
    within(got, want, bound, "grad")
    assert torch.equal(tk.embedding_backward(dout, ids, rows, 1.7), got)
    most = min(tokens, rows)
    out = (torch.full((most,), -5, dtype=torch.int32, device="cuda"),
           torch.full((1,), -5, dtype=torch.int32, device="cuda"), torch.full((most, dim), 9.0, device="cuda"))
    u, count, rows_of = tk.embedding_rows(dout, ids, rows, 1.7, out=out)
    n = int(count)
    assert n == unique.numel() and torch.equal(u[:n], unique)
    assert torch.equal(rows_of[:n], got[unique.long()])            # the same sums in the same order
    assert bool((u[n:] == -5).all()) and bool((rows_of[n:] == 9.0).all())


def test_embedding_gradient_of_nothing(tk):
    ids, dout = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, 8, device="cuda")
    assert bool((tk.embedding_backward(dout, ids, 5) == 0).all())
    assert int(tk.embedding_rows(dout, ids, 5)[1]) == 0
    ids, dout = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.ones(3, 8, device="cuda")
    assert tk.embedding_backward(dout, ids, 0).shape == (0, 8)
    assert int(tk.embedding_rows(dout, ids, 0)[1]) == 0
    assert tk.embedding(torch.zeros(0, 8, device="cuda"), ids).tolist() == [[0.0] * 8] * 3
    assert tk.embedding(torch.ones(4, 8, device="cuda"), ids[:0]).shape == (0, 8)


def test_embedding_gradient_keeps_nan_in_its_row(tk):
    g = gen(4)
    ids = torch.randint(0, 20, (500,), generator=g, device="cuda").int()
    dout = randn(g, 500, 40)
    clean = tk.embedding_backward(dout, ids, 20)
    bad = int((ids == 7).nonzero()[0])
    dout[bad, 3] = math.nan
    other = int((ids == -1).sum()) == 0
    got = tk.embedding_backward(dout, ids, 20)
    assert other and bool(got[7, 3].isnan()) and int(got.isnan().sum()) == 1
    got[7, 3] = clean[7, 3]
    assert torch.equal(got, clean)
    ids[bad] = -1                                      # a token of no row
    assert bool(torch.isfinite(tk.embedding_backward(dout, ids, 20)).all())


def test_embedding_gradient_layouts(tk, gs):
    g = gen(6)
    big = randn(g, 700, 303, dtype=BF)
    ids = torch.randint(0, 90, (700,), generator=g, device="cuda").int()
    for off, dim in ((1, 64), (3, 101), (0, 300)):
        dout = big[:, off:off + dim]
        want, bound, _ = grad_of(dout, ids, 90, 1.0)
        grad = torch.full((92, 333), 7.0, device="cuda")
        ws = torch.empty(gs.gs_embedding_bwd_ws_bytes(700, 90, dim), dtype=torch.uint8, device="cuda")
        gs.gs_embedding_bwd(dout, ids, 90, 1.0, grad[1:91, 5:5 + dim], ws)
        within(grad[1:91, 5:5 + dim], want, bound, "grad")
        grad[1:91, 5:5 + dim] = 7.0
        assert bool((grad == 7.0).all())


# -- recurrence ------------------------------------------------------------------------

RUNS = {  # lengths, channels
    "one token": ([1], 1), "one token, many channels": ([1], 300), "steps": ([1] * 40, 130), "steps past a chunk": ([1] * 300, 66),
    "a chunk": ([128], 64), "less": ([127], 128), "more": ([129], 129), "odd": ([77], 33), "kept edges": ([63, 1, 64, 65, 128, 129], 20),
    "long": ([3000], 40), "ragged": ([5, 0, 700, 3, 1, 0, 0, 257, 16, 15, 17], 70), "empty": ([0, 0, 0], 10),
    "empty ends": ([0, 50, 0], 257), "many": ([(i * 7) % 23 for i in range(150)], 18),
    "empties": ([3] + [0] * 200 + [5] + [0] * 70 + [1, 1, 2] + [0] * 130 + [400, 0, 1], 12), "alone": ([100, 0, 156], 66),
    "past alone": ([257], 66), "very many": ([i % 2 for i in range(5000)], 4), "wave edges": ([16, 15, 1, 17, 31, 32, 33], 131),
}


def runs(name, dtype, seed=1):
    lengths, cols = RUNS[name]
    g = gen(seed + cols)
    n = sum(lengths)
    x, gate = randn(g, n, cols, dtype=dtype), (randn(g, n, cols) * 1.5 + 1.5).to(dtype)
    cu = [0] + torch.tensor(lengths).cumsum(0).tolist()
    return g, x, gate, cu, randn(g, len(lengths), cols)


def starts(cu):
    return torch.tensor(cu, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("name", list(RUNS))
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_recurrence(tk, name, reverse, dtype):
    g, x, gate, cu, initial = runs(name, dtype)
    say(name, reverse, dtype)
    for first in (None, initial):
        got = tk.recurrence(x, gate, cu=starts(cu), initial=first, reverse=reverse, keep=True)
        want = ref.recurrence(x, gate, cu, first, reverse)
        for k, t in (("y", got.y), ("final", got.final), ("kept", got.kept)):
            within(t.cpu(), want[k], want["B" + k], k)
        again = tk.recurrence(x, gate, cu=starts(cu), initial=first, reverse=reverse)
        assert again.kept is None and torch.equal(again.y, got.y) and torch.equal(again.final, got.final)


@pytest.mark.parametrize("name", list(RUNS))
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_recurrence_backward(tk, name, reverse, dtype):
    g, x, gate, cu, initial = runs(name, dtype)
    say(name, reverse, dtype)
    dy, dfinal = randn(g, *x.shape, dtype=dtype), randn(g, *initial.shape)
    for first, last in ((None, None), (initial, dfinal)):
        kept = ref.recurrence(x, gate, cu, first, reverse)["kept"].float().cuda()
        got = tk.recurrence_backward(dy, x, gate, kept, cu=starts(cu), initial=first, dfinal=last, reverse=reverse)
        want, bounds = ref.recurrence_bwd(dy, x, gate, cu, first, last, reverse)
        for a, b, e, what in zip(got, want, bounds, ("dx", "dgate", "dinitial")):
            if a is not None:
                within(a.cpu(), b, e, what)
        assert (got[2] is None) == (first is None)
        again = tk.recurrence_backward(dy, x, gate, kept, cu=starts(cu), initial=first, dfinal=last, reverse=reverse)
        assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))


# Lists of many chunks: states that reach over all of them, past 64 looks ahead, segments that start at a chunk's or at
# many chunks' end, next to it and inside.
LONG = {"one": (9_000, [0]), "few": (9_000, [0, 2047, 2048, 4095, 4097, 6144, 8191]), "a place": (2049, [0, 2048]),
        "far": (280_000, [0]), "far, few": (280_000, [0, 130, 2048 * 3 - 1, 2048 * 70, 2048 * 70 + 1, 2048 * 136 + 129])}


def test_the_long_reference_is_the_short_one():
    g = torch.Generator().manual_seed(3)
    x, gate, dy = (torch.randn(60, 3, generator=g) for _ in range(3))
    for reverse in (False, True):
        cu = [0, 7, 8, 30, 60]
        f, (b, e) = ref.recurrence(x, gate, cu, None, reverse), ref.recurrence_bwd(dy, x, gate, cu, None, None, reverse)
        values, bounds = ref.long_recurrence(x, gate, cu, dy, reverse)
        for s, t in zip(values + bounds, (f["y"], b[0], b[1], f["By"], e[0], e[1])):
            assert torch.allclose(s, t, rtol=1e-11, atol=1e-13)


@pytest.mark.parametrize("name", list(LONG))
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_long_recurrence(tk, name, reverse, dtype):
    n, cu = LONG[name]
    cu = cu + [n]
    cols = 3 if n > 10_000 else 130
    g = gen(17)
    say(name, reverse, dtype)
    x, dy = randn(g, n, cols, dtype=dtype), randn(g, n, cols, dtype=dtype)
    gate = (randn(g, n, cols) + 3 * torch.arange(1, cols + 1, device="cuda").clamp(max=4)).to(dtype)
    (y, dx, dg), (By, Bx, Bg) = ref.long_recurrence(x, gate, cu, dy, reverse)
    got = tk.recurrence(x, gate, cu=starts(cu), reverse=reverse, keep=True)
    within(got.y.cpu(), y, By, "y")
    a, b, _ = tk.recurrence_backward(dy, x, gate, got.kept, cu=starts(cu), reverse=reverse)
    within(a.cpu(), dx, Bx, "dx")
    within(b.cpu(), dg, Bg, "dgate")


STEPS = {  # tokens, segments' starts (a number: that many equal segments)
    "one": (1, 1), "each one": (300, 300), "each four": (300, 75), "each five": (300, 60), "many": (5000, 5000),
    "skewed": (251, [0] * 201 + [200] + list(range(201, 252))), "past the ends": (40, [-3] + list(range(0, 37)) + [90] * 5),
    "outside": (50, [7] * 30 + list(range(8, 30)) + [31]), "none": (20, [20] * 41), "in front": (20, [0] * 41),
}


@pytest.mark.parametrize("name", list(STEPS))
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("cols", [1, 2, 131, 600])
@pytest.mark.parametrize("dtype", TYPES)
def test_steps(tk, gs, name, reverse, cols, dtype):
    """Many segments of few tokens: from strided tokens, states in place, tokens outside left alone or zeros."""
    n, cu = STEPS[name]
    segments = cu if isinstance(cu, int) else len(cu) - 1
    g = gen(19)
    say(name, reverse, cols, dtype)
    x, gate = randn(g, n, cols + 3, dtype=dtype)[:, 1:cols + 1], randn(g, n, 2 * cols, dtype=dtype)[:, cols:]
    initial = randn(g, segments, cols)
    at = list(range(0, n + 1, n // segments)) if isinstance(cu, int) else cu
    kw = dict(n_seg=cu) if isinstance(cu, int) else dict(cu=starts(cu))
    want = ref.recurrence(x, gate, at, initial, reverse)
    got = tk.recurrence(x, gate, initial=initial, reverse=reverse, **kw)
    within(got.y.cpu(), want["y"], want["By"], "y")
    within(got.final.cpu(), want["final"], want["Bfinal"], "final")
    state, y = initial.clone(), torch.full((n, cols), 7.0, dtype=dtype, device="cuda")
    r = gs.make_recur(x, gate, None if isinstance(cu, int) else starts(cu), n_seg=segments, initial=state, reverse=reverse)
    ws = torch.empty(max(1, gs.gs_recurrence_ws_bytes(r)), dtype=torch.uint8, device="cuda")
    gs.gs_recurrence(r, y, state, ws=ws)
    inside = torch.zeros(n, dtype=torch.bool, device="cuda")
    inside[min(max(at[0], 0), n):min(max(at[-1], 0), n)] = True
    assert torch.equal(state, got.final) and torch.equal(y[inside], got.y[inside])
    assert bool((y[~inside] == 7.0).all()) and bool((got.y[~inside] == 0).all())
    if name != "skewed":                                   # a segment longer than a wave's tokens is joined from maps
        assert torch.equal(tk.recurrence(x, gate, reverse=reverse, **kw).y,
                           tk.recurrence(x, gate, reverse=reverse, keep=True, **kw).y)


def test_recurrence_of_equal_segments(tk):
    g = gen(8)
    x, gate = randn(g, 6 * 45, 24), randn(g, 6 * 45, 24)
    a = tk.recurrence(x, gate, n_seg=6, keep=True)
    b = tk.recurrence(x, gate, cu=starts(list(range(0, 271, 45))), keep=True)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    dy = randn(g, *x.shape)
    for s, t in zip(tk.recurrence_backward(dy, x, gate, a.kept, n_seg=6),
                    tk.recurrence_backward(dy, x, gate, a.kept, cu=starts(list(range(0, 271, 45))))):
        assert s is t or torch.equal(s, t)


def test_recurrence_step_by_step(tk):
    """A served sequence: one token at a time with its state gives what the whole sequence does."""
    g = gen(9)
    x, gate = randn(g, 5, 20, 48), randn(g, 5, 20, 48)         # sequences, tokens, channels
    whole = tk.recurrence(x.reshape(100, 48), gate.reshape(100, 48), n_seg=5)
    state = torch.zeros(5, 48, device="cuda")
    for t in range(20):
        r = tk.recurrence(x[:, t].contiguous(), gate[:, t].contiguous(), n_seg=5, initial=state)
        state = r.final
        assert torch.equal(r.y, r.final)
        # the same terms with fewer gates between them: the bound of either form
        want = ref.recurrence(x[:, :t + 1].reshape(-1, 48), gate[:, :t + 1].reshape(-1, 48),
                              list(range(0, 5 * (t + 1) + 1, t + 1)))
        within(state.cpu(), want["final"], want["Bfinal"], "state")
    want = ref.recurrence(x.reshape(100, 48), gate.reshape(100, 48), list(range(0, 101, 20)))
    within(whole.final.cpu(), want["final"], want["Bfinal"], "final")


@pytest.mark.parametrize("n,cu", [(50, [5, 20, 44]), (700, [5, 400, 650]), (300, [300, 300]), (300, [0, 0]), (300, [-4, 100, 900])])
@pytest.mark.parametrize("reverse", [False, True])
def test_tokens_outside_every_segment(tk, gs, n, cu, reverse):
    """They reach nothing, whatever they hold, and are left alone by the entry points, zeros from the functions."""
    g = gen(10)
    lo, hi = min(max(cu[0], 0), n), min(cu[-1], n)
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    outside[lo:hi] = False
    x, gate, dy = (randn(g, n, 40) for _ in range(3))
    want = ref.recurrence(x, gate, cu, None, reverse)
    wg, bounds = ref.recurrence_bwd(dy, x, gate, cu, None, None, reverse)
    for t in (x, gate, dy):
        t[outside] = math.nan
    got = tk.recurrence(x, gate, cu=starts(cu), reverse=reverse, keep=True)
    within(got.y.cpu(), want["y"], want["By"], "y")
    within(got.final.cpu(), want["final"], want["Bfinal"], "final")
    within(got.kept.cpu(), want["kept"], want["Bkept"], "kept")
    assert bool((got.y[outside] == 0).all())
    grads = tk.recurrence_backward(dy, x, gate, got.kept, cu=starts(cu), reverse=reverse)
    for a, b, e in zip(grads[:2], wg, bounds):
        within(a.cpu(), b, e, "gradient")
        assert bool((a[outside] == 0).all())
    r = gs.make_recur(x, gate, starts(cu), reverse=reverse)
    y, dx, dg = (torch.full((n, 40), 7.0, device="cuda") for _ in range(3))
    ws = torch.empty(max(1, gs.gs_recurrence_ws_bytes(r)), dtype=torch.uint8, device="cuda")
    gs.gs_recurrence(r, y, ws=ws)
    gs.gs_recurrence_bwd(r, dy, got.kept, dx, dg, ws=ws)
    for t, f in ((y, got.y), (dx, grads[0]), (dg, grads[1])):
        assert bool((t[outside] == 7.0).all()) and torch.equal(t[~outside], f[~outside])


@pytest.mark.parametrize("reverse", [False, True])
def test_nan_stays_in_its_channel_and_segment(tk, reverse):
    g = gen(12)
    cu = [0, 200, 500, 777]
    x, gate, dy = (randn(g, 777, 30) for _ in range(3))
    clean = tk.recurrence(x, gate, cu=starts(cu), reverse=reverse, keep=True)
    grads = tk.recurrence_backward(dy, x, gate, clean.kept, cu=starts(cu), reverse=reverse)
    x2, dy2 = x.clone(), dy.clone()
    x2[333, 7] = math.nan
    dy2[444, 9] = math.inf
    got = tk.recurrence(x2, gate, cu=starts(cu), reverse=reverse, keep=True)
    bad = torch.zeros(777, 30, dtype=torch.bool, device="cuda")
    bad[200:334, 7] = reverse
    bad[333:500, 7] |= not reverse
    bad[333, 7] = True
    assert torch.equal(got.y.isnan(), bad) and torch.equal(got.y[~bad], clean.y[~bad])
    assert int(got.final.isnan().sum()) == 1 and bool(got.final[1, 7].isnan())
    dx, dg, _ = tk.recurrence_backward(dy2, x, gate, clean.kept, cu=starts(cu), reverse=reverse)
    wrong = ~torch.isfinite(dx) | ~torch.isfinite(dg)
    assert bool(wrong[444, 9]) and not bool(wrong[:200].any()) and not bool(wrong[500:].any())
    wrong[:, 9] = False
    assert not bool(wrong.any())
    keep = torch.arange(30, device="cuda") != 9
    assert torch.equal(dx[:, keep], grads[0][:, keep]) and torch.equal(dg[:, keep], grads[1][:, keep])


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", [F32, HF])
def test_nan_stays_in_its_channel_and_segment_of_long_lists(tk, reverse, dtype):
    """Segments of many chunks that start inside one, at its end and at that of many."""
    g = gen(29)
    n, cols = 40_000, 70
    cu = [0, 2048 * 3, 2048 * 7 + 128, 2048 * 9 - 5, n]
    x, gate, dy = (randn(g, n, cols, dtype=dtype) for _ in range(3))
    gate = gate + 8
    clean = tk.recurrence(x, gate, cu=starts(cu), reverse=reverse, keep=True)
    grads = tk.recurrence_backward(dy, x, gate, clean.kept, cu=starts(cu), reverse=reverse)
    bad = torch.zeros(n, cols, dtype=torch.bool, device="cuda")
    x2, gate2, dy2 = x.clone(), gate.clone(), dy.clone()
    for s, (t, c) in enumerate([(5000, 3), (2048 * 4 + 1, 64), (2048 * 8, 3), (20_000, 69)]):
        (x2 if s % 2 else gate2)[t, c] = math.nan
        dy2[t, c + 1 - 2 * (c == 69)] = math.nan
        if reverse:
            bad[cu[s]:t + 1, c] = True
        else:
            bad[t:cu[s + 1], c] = True
    got = tk.recurrence(x2, gate2, cu=starts(cu), reverse=reverse, keep=True)
    assert torch.equal(got.y.isnan(), bad) and torch.equal(got.y[~bad], clean.y[~bad])
    dx, dg, _ = tk.recurrence_backward(dy2, x, gate, clean.kept, cu=starts(cu), reverse=reverse)
    bad[:] = False
    for s, (t, c) in enumerate([(5000, 4), (2048 * 4 + 1, 65), (2048 * 8, 4), (20_000, 68)]):
        if reverse:
            bad[t:cu[s + 1], c] = True
        else:
            bad[cu[s]:t + 1, c] = True
    assert torch.equal(dx.isnan(), bad) and torch.equal(dg.isnan(), bad)
    assert torch.equal(dx[~bad], grads[0][~bad]) and torch.equal(dg[~bad], grads[1][~bad])


def test_gates_at_the_ends(tk):
    """Gates that hold or drop the state entirely, and very large ones."""
    x = torch.arange(1, 301, device="cuda", dtype=F32)[:, None].repeat(1, 6).contiguous()
    gate = torch.tensor([0.0, 1e30, -1e30, math.inf, -math.inf, 60.0], device="cuda").repeat(300, 1).contiguous()
    r = tk.recurrence(x, gate, initial=torch.full((1, 6), 5.0, device="cuda"), keep=True)
    for c, want in ((1, 5.0), (3, 5.0)):
        assert bool((r.y[:, c] == want).all())
    for c in (2, 4):
        assert torch.equal(r.y[:, c], x[:, c])
    # 300 tokens through 1 - a = exp(-60): the state stays, but for 300 * 300 * exp(-60)
    assert bool((r.y[:, 5] == 5.0).all())
    dx, dg, di = tk.recurrence_backward(torch.ones_like(x), x, gate, r.kept, initial=torch.full((1, 6), 5.0, device="cuda"))
    assert torch.equal(di[0, [1, 2, 3, 4]], torch.tensor([300.0, 0.0, 300.0, 0.0], device="cuda"))
    assert bool((dx[:, [1, 3]] == 0).all()) and bool((dx[:, [2, 4]] == 1).all()) and bool((dg[:, 1:5] == 0).all())
    assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dg).all())


def test_small_gates_keep_their_bits(tk):
    """A large state that a gate of 1e-6 lets through by a millionth, and 1 - a of 1e-6."""
    g = -math.log(1e6 - 1)
    x, gate = torch.ones(3, 2, device="cuda"), torch.zeros(3, 2, device="cuda")
    gate[:, 0], gate[:, 1] = g, -g
    first = torch.tensor([[1e6, 0.0]], device="cuda")
    y = tk.recurrence(x, gate, initial=first).y
    want = ref.recurrence(x, gate, [0, 3], first)
    within(y.cpu(), want["y"], want["By"], "y")
    assert abs(float(y[0, 0]) - 2.0) < 1e-4 and abs(float(y[2, 1]) - 3e-6) < 1e-10


@pytest.mark.parametrize("dtype", TYPES)
def test_recurrence_strides(tk, dtype):
    """Gate, x and their gradients as columns of wider matrices at any alignment."""
    g = gen(13)
    wide = randn(g, 400, 500, dtype=dtype)
    cu = [0, 150, 400]
    for off, cols in ((0, 128), (1, 77), (3, 130), (5, 1)):
        x, gate, dy = wide[:, off:off + cols], wide[:, off + 170:off + 170 + cols], wide[:, off + 333:off + 333 + cols]
        got = tk.recurrence(x, gate, cu=starts(cu), keep=True)
        dense = tk.recurrence(x.contiguous(), gate.contiguous(), cu=starts(cu), keep=True)
        assert all(torch.equal(a, b) for a, b in zip(got, dense))
        a = tk.recurrence_backward(dy, x, gate, got.kept, cu=starts(cu))
        b = tk.recurrence_backward(dy.contiguous(), x.contiguous(), gate.contiguous(), got.kept, cu=starts(cu))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_recurrence_backward_against_differences(tk):
    g = gen(14)
    cu = [0, 5, 5, 31]
    x, gate, dy, first, dfinal = randn(g, 31, 6), randn(g, 31, 6), randn(g, 31, 6), randn(g, 3, 6), randn(g, 3, 6)
    ref.UNIT[torch.float64] = ref.TINY[torch.float64] = 0.0
    for reverse in (False, True):
        kept = tk.recurrence(x, gate, cu=starts(cu), initial=first, reverse=reverse, keep=True).kept
        dx, dg, di = (t.double().cpu() for t in tk.recurrence_backward(dy, x, gate, kept, cu=starts(cu), initial=first,
                                                                       dfinal=dfinal, reverse=reverse))

        def f(a, b, c):
            r = ref.recurrence(a, b, cu, c, reverse)
            return float((r["y"] * dy.double().cpu()).sum() + (r["final"] * dfinal.double().cpu()).sum())

        for _ in range(3):
            a, b, c, h = (randn(g, *t.shape).double().cpu() for t in (x, gate, first)), None, None, 1e-5
            a, b, c = a
            X, G, I = (t.double().cpu() for t in (x, gate, first))
            num = (f(X + h * a, G + h * b, I + h * c) - f(X - h * a, G - h * b, I - h * c)) / (2 * h)
            got = float((dx * a).sum() + (dg * b).sum() + (di * c).sum())
            size = float((dx * a).abs().sum() + (dg * b).abs().sum() + (di * c).abs().sum())
            # the differences' own error (third derivative, h^2) and fp32 gradients
            assert abs(num - got) <= 1e-5 * size


# -- gated SiLU -------------------------------------------------------------------------

def near(got, want, bound, what):
    """within(), and infinities where the value is past the type's range (65520 and more round to infinity in fp16)."""
    top = torch.finfo(got.dtype).max
    past = want.abs() - bound > top * (1 + torch.finfo(got.dtype).eps / 4)
    assert torch.equal(got[past].double(), torch.sign(want[past]) * math.inf), what
    fits = want.abs() + bound < top
    within(got[fits], want[fits], bound[fits], what)


SILUS = [(1, 1), (3, 7), (5, 32), (4, 33), (300, 64), (7, 250), (64, 1000), (9, 4099), (2, 20001), (0, 40), (1001, 24)]


@pytest.mark.parametrize("rows,cols", SILUS)
@pytest.mark.parametrize("dtype", TYPES)
def test_gated_silu(tk, rows, cols, dtype):
    g = gen(rows + cols)
    both = randn(g, rows, 2 * cols) * torch.exp(2 * randn(g, rows, 1))
    both = both.to(dtype)
    u = both[:, :cols]
    dh = randn(g, rows, cols, dtype=dtype)
    for v in (None, both[:, cols:]):
        r = tk.gated_silu(u, v)
        h, bound = ref.silu(u, v)
        near(r.h, h, bound, "h")
        for t, q, s in ((u, r.u8, r.u_scale), (v, r.v8, r.v_scale)):
            if t is None:
                assert q is None and s is None
                continue
            want, k = ref.eight(t)
            assert q.dtype == torch.float8_e4m3fn and torch.equal(s, k) and torch.equal(q.double(), want)
        bare = tk.gated_silu(u, v, keep=False)
        assert bare.u8 is None and bare.v8 is None and torch.equal(bare.h, r.h)
        du, dv, again = tk.gated_silu_backward(dh, r.u8, r.u_scale, r.v8, r.v_scale)
        U, V = ref.wide(r.u8, r.u_scale), None if v is None else ref.wide(r.v8, r.v_scale)
        want, bounds = ref.silu_bwd(dh, U, V)
        near(du, want[0], bounds[0], "du")
        near(again, want[2], bounds[2], "h again")
        if v is None:
            assert dv is None
        else:
            near(dv, want[1], bounds[1], "dv")
        without = tk.gated_silu_backward(dh, r.u8, r.u_scale, r.v8, r.v_scale, again=False)
        assert without[2] is None and torch.equal(without[0], du)


@pytest.mark.parametrize("dtype", TYPES)
def test_kept_values_at_the_ends(tk, dtype):
    """Blocks of zeros, tiny and huge values, values at 448's and at rounding's edges, NaN and infinities."""
    top = torch.finfo(dtype).max
    x = torch.zeros(12, 70)
    x[1, 3] = torch.finfo(dtype).tiny
    x[2] = torch.linspace(-448, 448, 70)
    x[3, :32] = torch.tensor([448.0, 449.0] * 16)
    x[4, 0], x[4, 1] = top, 1.0
    x[5] = torch.arange(70) * 0.0625 + 16              # halfway between two e4m3 numbers, both ways
    x[6, 5], x[6, 6] = math.nan, 3.0
    x[7, 40], x[7, 41] = math.inf, -2.0
    x[8] = torch.arange(70) * torch.finfo(dtype).tiny
    x[9] = -x[2]
    x[10, :64] = math.nan
    x[11] = torch.arange(70) * torch.finfo(dtype).smallest_normal * 2.0 ** -6
    x = x.to(dtype).cuda()
    r = tk.gated_silu(x, x)
    for q, s in ((r.u8, r.u_scale), (r.v8, r.v_scale)):
        want, k = ref.eight(x)
        assert torch.equal(s, k)
        assert torch.equal(q.double().nan_to_num(nan=1e9), want.nan_to_num(nan=1e9))
    assert int(r.u_scale[0].max()) == 0 and int(r.u_scale[10, 0]) == 0
    fine = torch.isfinite(x)
    # three bits behind the leading one: a 16th of an element, and half a step of 2^-9 of the scale near zero
    back = ref.wide(r.u8, r.u_scale)
    scale = torch.exp2(r.u_scale.double() - 127).repeat_interleave(32, 1)[:, :70]
    assert bool(((back - x.double()).abs() <= x.double().abs() / 16 + scale * 2.0 ** -10)[fine].all())


def test_gated_silu_far_out(tk):
    u = torch.tensor([[-1e30, -200.0, -90.0, -20.0, 0.0, 20.0, 90.0, 200.0, 1e30]], device="cuda")
    r = tk.gated_silu(u)
    h, bound = ref.silu(u)
    within(r.h, h, bound + 1e-30, "h")
    du, _, again = tk.gated_silu_backward(torch.ones_like(u), r.u8, r.u_scale)
    assert bool(torch.isfinite(du).all()) and bool(torch.isfinite(again).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_silu_strides_and_in_place(tk, gs, dtype):
    g = gen(17)
    wide = randn(g, 60, 700, dtype=dtype)
    for off, cols in ((0, 256), (1, 64), (3, 101), (5, 33)):
        u, v, dh = wide[:, off:off + cols], wide[:, off + 300:off + 300 + cols], wide[:, off + 400:off + 400 + cols]
        want = tk.gated_silu(u.contiguous(), v.contiguous())
        blocks = -(-cols // 32)
        h = torch.full((62, 333), 7.0, dtype=dtype, device="cuda")
        q = torch.full((2, 62, 333), 77, dtype=torch.uint8, device="cuda")
        s = torch.full((2, 62, 50), 77, dtype=torch.uint8, device="cuda")
        at = (slice(1, 61), slice(3, 3 + cols))
        sat = (slice(1, 61), slice(3, 3 + blocks))
        gs.gs_gated_silu(u, v, h[at], q[0][at], s[0][sat], q[1][at], s[1][sat])
        assert torch.equal(h[at], want.h)
        for i, (a, b) in enumerate(((want.u8, want.u_scale), (want.v8, want.v_scale))):
            assert torch.equal(q[i][at], a.view(torch.uint8)) and torch.equal(s[i][sat], b)
        grads = tk.gated_silu_backward(dh.contiguous(), want.u8, want.u_scale, want.v8, want.v_scale)
        d = dh.clone(memory_format=torch.contiguous_format)
        dv, again = torch.empty_like(d), torch.empty_like(d)
        gs.gs_gated_silu_bwd(d, q[0][at], s[0][sat], d, q[1][at], s[1][sat], dv, again)      # du over dh
        assert torch.equal(d, grads[0]) and torch.equal(dv, grads[1]) and torch.equal(again, grads[2])
        h[at], q[0][at], q[1][at], s[0][sat], s[1][sat] = 7.0, 77, 77, 77, 77
        assert bool((h == 7.0).all()) and bool((q == 77).all()) and bool((s == 77).all())


def test_gated_silu_backward_against_differences(tk):
    """Where the inputs are exact in 8 bits, the gradient is that of the forward."""
    g = gen(18)
    u, v = (torch.randint(-15, 16, (6, 64), generator=g, device="cuda").float() / 8 for _ in range(2))
    dh = randn(g, 6, 64)
    r = tk.gated_silu(u, v)
    assert torch.equal(ref.wide(r.u8, r.u_scale), u.double()) and torch.equal(ref.wide(r.v8, r.v_scale), v.double())
    du, dv, h = tk.gated_silu_backward(dh, r.u8, r.u_scale, r.v8, r.v_scale)
    within(h, r.h.double(), 2.0 ** -20 * r.h.double().abs() + 1e-30, "h again")
    f = lambda a, b: float((a * torch.sigmoid(a) * b * dh.double()).sum())
    for _ in range(4):
        a, b, e = randn(g, 6, 64).double(), randn(g, 6, 64).double(), 1e-5
        num = (f(u.double() + e * a, v.double() + e * b) - f(u.double() - e * a, v.double() - e * b)) / (2 * e)
        size = float((du.double() * a).abs().sum() + (dv.double() * b).abs().sum())
        assert abs(num - float((du.double() * a).sum() + (dv.double() * b).sum())) <= 1e-5 * size
