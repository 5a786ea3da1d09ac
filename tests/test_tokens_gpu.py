"""The token operators through the package's functions against plain 64-bit
forms.  Every tolerance is a bound derived from the roundings that the operator
makes (token_refs), not a measured one."""
import math

import pytest
import torch

import token_refs as ref

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def tk():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2607_19893_amd import tokens
    return tokens


@pytest.fixture(scope="module")
def gs():
    from paper_2607_19893_amd import gsmi
    return gsmi


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def within(got, want, bound, what):
    err = (got.double() - want).abs()
    assert bool(torch.isfinite(got.double()).all()), what
    bad = err > bound
    assert not bool(bad.any()), "%s: %d elements off, worst %g of its bound" % (
        what, int(bad.sum()), float((err / bound.clamp(min=1e-300)).max()))


# -- norm ------------------------------------------------------------------------

NORMS = [(1, 1), (1, 8), (3, 7), (5, 128), (4, 129), (7, 1024), (9, 1025), (6, 1160), (5, 1536), (3, 2048), (2, 2056),
         (2, 4099), (2, 5000), (3, 8200), (2, 16384), (0, 64), (515, 72), (1001, 250), (37, 16), (70, 256)]


@pytest.mark.parametrize("rows,cols", NORMS)
@pytest.mark.parametrize("dtype", [F32, BF, HF])
def test_norm(tk, rows, cols, dtype):
    g = gen(rows * 7919 + cols)
    x, r = randn(g, rows, cols, dtype=dtype) * 3, randn(g, rows, cols, dtype=dtype)
    w = 1 + randn(g, cols)
    u = ref.UNIT[dtype]
    for res in (None, r):
        got = tk.rms_norm(x, w, 1e-6, residual=res)
        y, s = ref.norm(x, w, 1e-6, res)
        # fp32: the sum, the squares' sum (relative, all positive), root, reciprocal and three products
        within(got.y, y, (u + (cols / 64 + 40) * 2.0 ** -24) * y.abs() + 4 * ref.TINY[dtype], "y")
        if res is not None:
            assert torch.equal(got.total, (x.float() + r.float()).to(dtype))
        else:
            assert got.total is x
        e = tk.rms_norm(x, w, 1e-6, residual=res, eight_bit=True)
        assert e.q.dtype == torch.float8_e4m3fn and e.scale.shape == (rows, -(-cols // 128)) and e.y is None
        if rows:
            top = torch.stack([b.abs().amax(1) for b in y.split(128, 1)], 1)
            within(e.scale, top / 448, 1e-5 * top / 448 + 1e-38, "scale")
            at = torch.arange(cols, device="cuda") // 128
            v = y / e.scale.double()[:, at]
            step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
            within(e.q.float(), v, step * 0.5 * (1 + 1e-3) + 1e-4 * v.abs(), "q")


def test_norm_special_rows(tk):
    x = torch.zeros(5, 300, device="cuda")
    x[1] = 1e-30
    x[2, :128] = 5.0
    x[3, 7] = math.nan
    x[4, 200] = math.inf
    w = torch.ones(300, device="cuda")
    r = tk.rms_norm(x, w, 0.0 + 1e-12)
    assert bool((r.y[0] == 0).all()) and bool(torch.isfinite(r.y[:3]).all())
    assert bool(r.y[3].isnan().all()) and bool(r.y[4, 200].isnan())
    e = tk.rms_norm(x, w, 1e-12, eight_bit=True)
    assert bool((e.scale[0] == 1).all()) and bool((e.q[0].float() == 0).all())
    assert bool((e.scale[2, 1:] == 1).all()) and float(e.q[2, 0].float()) == 448.0
    assert bool(e.q[3].float().isnan().all())


@pytest.mark.parametrize("dtype", [F32, BF])
def test_norm_strides_and_in_place(tk, gs, dtype):
    g = gen(5)
    wide = randn(g, 33, 200, dtype=dtype)
    for off, cols in ((0, 96), (1, 96), (3, 101)):
        x, w = wide[:, off:off + cols], 1 + randn(g, cols)
        y, _ = ref.norm(x, w, 1e-5)
        u = ref.UNIT[dtype]
        within(tk.rms_norm(x, w, 1e-5).y, y, (u + 1e-5) * y.abs() + 1e-38, "strided x")
    x, r, w = randn(g, 40, 256, dtype=dtype), randn(g, 40, 256, dtype=dtype), 1 + randn(g, 256)
    want = tk.rms_norm(x, w, 1e-5, residual=r)
    gs.gs_rms_norm(x, w, 1e-5, y=x, residual=r, total=r)
    assert torch.equal(x, want.y) and torch.equal(r, want.total)


@pytest.mark.parametrize("rows,cols", [s for s in NORMS if s[0]] + [(3000, 264), (2100, 2304)])
@pytest.mark.parametrize("dtype", [F32, BF, HF])
def test_norm_backward(tk, rows, cols, dtype):
    g = gen(rows * 31 + cols)
    total, dy, dt = (randn(g, rows, cols, dtype=dtype) for _ in range(3))
    w = 1 + randn(g, cols)
    u = ref.UNIT[dtype]
    for extra in (None, dt):
        dx, dw = tk.rms_norm_backward(dy, total, w, 1e-6, dtotal=extra)
        rx, rw, size = ref.norm_bwd(dy, total, w, 1e-6, extra)
        r = 1.0 / torch.sqrt(total.double().pow(2).mean(1, keepdim=True) + 1e-6)
        n = total.double() * r
        gw = dy.double() * w.double()
        # fp32 sums of |g n| terms behind the mean, products of a few factors
        part = r * (gw.abs() + n.abs() * (gw * n).abs().mean(1, keepdim=True))
        within(dx, rx, u * rx.abs() + (cols / 64 + 40) * 2.0 ** -24 * part + 2.0 ** -23 * rx.abs() + 4 * ref.TINY[dtype], "dx")
        adds = rows / min(512, -(-rows // 4)) + 100
        within(dw, rw, (adds + cols / 64 + 40) * 2.0 ** -24 * size + 1e-38, "dweight")
        again = tk.rms_norm_backward(dy, total, w, 1e-6, dtotal=extra)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


def test_norm_backward_of_no_rows(tk):
    z = torch.zeros(0, 96, device="cuda")
    dx, dw = tk.rms_norm_backward(z, z, torch.ones(96, device="cuda"))
    assert dx.shape == (0, 96) and bool((dw == 0).all())


def test_norm_backward_against_differences(tk):
    g = gen(11)
    x, w, dy, dt = randn(g, 6, 40), 1 + randn(g, 40), randn(g, 6, 40), randn(g, 6, 40)
    dx, dw = tk.rms_norm_backward(dy, x, w, 1e-3, dtotal=dt)
    f = lambda a, b: float((ref.norm(a, b, 1e-3)[0] * dy.double()).sum() + (a * dt.double()).sum())
    for _ in range(4):
        a, b, h = randn(g, 6, 40).double(), randn(g, 40).double(), 1e-5
        num = (f(x.double() + h * a, w.double() + h * b) - f(x.double() - h * a, w.double() - h * b)) / (2 * h)
        got = float((dx.double() * a).sum() + (dw.double() * b).sum())
        # the differences' own error (third derivative, h^2) and fp32 gradients
        size = float((dx.double() * a).abs().sum() + (dw.double() * b).abs().sum())
        assert abs(num - got) <= 1e-5 * size


# -- rotary -----------------------------------------------------------------------

ROTARY = [  # tokens, heads, dim, axis_pairs
    (1, (1,), 2, [1]), (5, (3, 1), 64, [32]), (37, (8, 2), 128, [64]), (130, (4, 4), 64, [8, 8, 8]),
    (17, (2, 1), 80, [13, 13, 13]), (9, (5,), 66, [10, 0, 23]), (300, (6, 3), 32, [4, 4]), (4, (2, 2), 512, [256]),
    (1100, (16, 4), 96, [20]), (6, (2,), 16, [0]), (2, (3,), 7, [3]),
]


def turn_bound(size, y, dtype, amplitude):
    # the reduced angle in fp32 (pi 2^-24), sine and cosine, two products and a sum; then the type's rounding
    return 8 * 2.0 ** -24 * abs(amplitude) * size + ref.UNIT[dtype] * y.abs() + ref.TINY[dtype]


@pytest.mark.parametrize("tokens,heads,dim,axis_pairs", ROTARY)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF, HF])
def test_rotary(tk, tokens, heads, dim, axis_pairs, interleaved, dtype):
    g = gen(tokens + dim)
    xs = [randn(g, tokens, h, dim, dtype=dtype) for h in heads]
    pairs = sum(axis_pairs)
    pos = randn(g, tokens, len(axis_pairs)) * 500
    pos[0] = 16777215.0                                # the largest odd whole number of fp32
    freq = torch.rand(pairs, generator=g, device="cuda")
    for inverse, amplitude in ((False, 1.0), (True, 1.25)):
        got = tk.rotary(xs, pos, freq, axis_pairs, interleaved=interleaved, inverse=inverse, amplitude=amplitude)
        for x, y in zip(xs, got):
            want, size = ref.rotary(x, pos, freq, axis_pairs, interleaved, inverse, amplitude)
            within(y, want, turn_bound(size, want, dtype, amplitude), "turned")
            assert torch.equal(y[..., 2 * pairs:], x[..., 2 * pairs:])
    there = tk.rotary([x.clone() for x in xs], pos, freq, axis_pairs, interleaved=interleaved, inverse=True,
                      amplitude=1.25, inplace=True)
    assert all(torch.equal(a, b) for a, b in zip(there, got))


def test_rotary_layouts(tk):
    """Columns of one projection, heads before tokens, rows that are not aligned."""
    g = gen(3)
    freq = torch.rand(24, generator=g, device="cuda")
    pos = randn(g, 50, 1) * 40
    qkv = randn(g, 50, 12, 64, dtype=BF)
    byhead = randn(g, 6, 50, 64, dtype=BF).transpose(0, 1)
    odd = randn(g, 50 * 3 * 65 + 1, dtype=BF)[1:].view(50, 3, 65)[..., :64]
    for xs in ((qkv[:, :8], qkv[:, 8:10]), (byhead,), (odd, qkv[:, 3:5])):
        for x, y in zip(xs, tk.rotary(xs, pos, freq, [24])):
            want, size = ref.rotary(x, pos, freq, [24], False)
            within(y, want, turn_bound(size, want, BF, 1.0), "layout")


def test_rotary_there_and_back(tk):
    g = gen(9)
    x, pos = randn(g, 64, 4, 64), randn(g, 64, 1) * 1000
    freq = torch.rand(32, generator=g, device="cuda")
    (y,) = tk.rotary(x, pos, freq, [32])
    (z,) = tk.rotary(y, pos, freq, [32], inverse=True)
    size = x.abs()[..., :32] + x.abs()[..., 32:]
    within(z, x.double(), 16 * 2.0 ** -24 * 2 * torch.cat((size, size), -1).double(), "back")
    # the gradient is the turn back: <turn(x), y> = <x, turn back(y)>
    a, b = randn(g, 64, 4, 64), randn(g, 64, 4, 64)
    left = float((tk.rotary(a, pos, freq, [32])[0].double() * b).sum())
    right = float((a.double() * tk.rotary(b, pos, freq, [32], inverse=True)[0]).sum())
    assert abs(left - right) <= 1e-5 * float((a.double() * b).abs().sum())


# -- attention ----------------------------------------------------------------------

def case(nq, nk=None, heads=2, kv=None, dim=64, left=-1, right=-1, off=0.0, dtype=BF):
    return dict(nq=nq, nk=list(nq) if nk is None else nk, heads=heads, kv=kv or heads, dim=dim, left=left, right=right,
                off=off, dtype=dtype, scale=dim ** -0.5)


CASES = {
    "one by one": case([1], [1], 1, dim=8),
    "one by many": case([1], [700], 4, 1, dim=128),
    "one by many, parts": case([1], [6000], 8, 2, dim=128),
    "many by one": case([300], [1], 2, dim=32),
    "tile edges": case([31, 32, 33, 63, 64, 65, 127, 128, 129], heads=2, dim=64),
    "tile edges ordered": case([31, 32, 33, 63, 64, 65, 127, 128, 129], heads=2, dim=32, right=0),
    "no keys, no rows": case([5, 0, 70, 3], [9, 40, 0, 0], 2, dim=64),
    "all empty": case([4, 4], [0, 0], 2, dim=64),
    "more rows than keys, ordered": case([200, 40], [70, 3], 2, dim=64, right=0),
    "window": case([333, 50], heads=4, kv=2, dim=96, left=40, right=0),
    "window both ways": case([257], [300], 3, 1, dim=80, left=17, right=5, off=0.4),
    "window ahead only": case([100], [180], 2, dim=40, right=30),
    "window behind only": case([150, 20], [90, 160], 2, dim=64, left=12),
    "masked": case([140, 80], [150, 64], 4, 4, dim=64, off=0.5, dtype=HF),
    "all keys off but one segment's": case([50, 50, 50], heads=2, dim=64, off="but the first"),
    "groups of three": case([45, 130], heads=6, kv=2, dim=24, right=0),
    "groups of five": case([77], [200], heads=5, kv=1, dim=64, dtype=HF),
    "groups of twelve, few": case([2, 1, 3], [900, 1, 64], heads=12, kv=1, dim=128, off=0.2),
    "few, long parts": case([1, 2, 1], [3000, 1500, 10], heads=8, kv=8, dim=64, off=0.1),
    "few, ordered": case([7, 4], [2200, 30], heads=4, kv=4, dim=96, right=0),
    "few, window": case([3, 3], [4000, 70], heads=4, kv=2, dim=128, left=1000, right=20),
    "two rows, more parts than lanes": case([2], [60000], heads=2, kv=1, dim=32, off=0.1),
    "few, but for one segment": case([100, 1, 1, 0, 1, 1], [700, 300, 0, 50, 9, 2000], heads=1, dim=64, left=900, right=0),
    "few, 70 segments": case([(i * 5) % 4 for i in range(70)], [(i * 37) % 900 for i in range(70)], 4, 1, dim=64, off=0.1),
    "wide rows split over the keys": case([40], [5000], heads=2, kv=1, dim=64, dtype=HF),
    "rows split for dk": case([2500], [130], heads=4, kv=1, dim=128),
    "dim 16": case([90], heads=2, dim=16, dtype=HF),
    "dim 112 ordered": case([190], heads=2, dim=112, right=0),
    "65 segments": case([(i * 7) % 23 for i in range(65)], heads=2, dim=32),
    "300 segments": case([(i * 11) % 19 for i in range(300)], [(i * 5) % 31 for i in range(300)], 2, 1, dim=64, right=0),
    "64 segments": case([(i * 13) % 40 for i in range(64)], heads=1, dim=64),
}


def inputs(c, seed=1):
    g = gen(seed)
    q = randn(g, sum(c["nq"]), c["heads"], c["dim"], dtype=c["dtype"])
    k, v = (randn(g, sum(c["nk"]), c["kv"], c["dim"], dtype=c["dtype"]) for _ in range(2))
    on = None
    if c["off"] == "but the first":
        on = torch.zeros(k.shape[0], dtype=torch.uint8, device="cuda")
        on[:c["nk"][0]] = 1
    elif c["off"]:
        on = (torch.rand(k.shape[0], generator=g, device="cuda") >= c["off"]).to(torch.uint8)
    return g, q, k, v, on


def cu(n):
    return torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda()


def how(c, on):
    return dict(cu_q=cu(c["nq"]), cu_k=cu(c["nk"]), key_on=on, scale=c["scale"], left=c["left"], right=c["right"])


def check_forward(got, want):
    (out, lse), (o, L, bound) = got, want
    within(out, o, bound, "out")
    empty = L == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    assert bool((out[empty] == 0).all())
    d = (lse.double() - L)[~empty].abs()
    # fp32 products (the scores, up to a few tens) and sums
    assert bool((d <= 2e-5 * (1 + L[~empty].abs())).all()), float(d.max())


@pytest.mark.parametrize("name", list(CASES))
def test_attention(tk, name):
    c = CASES[name]
    g, q, k, v, on = inputs(c)
    kw = how(c, on)
    out, lse = tk.attention(q, k, v, **kw)
    check_forward((out, lse), ref.attention(q, k, v, c, on))
    again = tk.attention(q, k, v, **kw)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("name", list(CASES))
def test_attention_backward(tk, name):
    c = CASES[name]
    g, q, k, v, on = inputs(c)
    dout = randn(g, *q.shape, dtype=c["dtype"])
    o, L, _ = ref.attention(q, k, v, c, on)
    out, lse = o.to(c["dtype"]), L.float()
    kw = how(c, on)
    got = tk.attention_backward(dout, q, k, v, out, lse, **kw)
    want, bounds = ref.attention(q, k, v, c, on, lse, out, dout)
    for a, b, e, what in zip(got, want, bounds, ("dq", "dk", "dv")):
        within(a, b, e, what)
    again = tk.attention_backward(dout, q, k, v, out, lse, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_attention_backward_against_differences(tk):
    c = case([9, 5], [12, 5], 4, 2, dim=16, right=0, off=0.2, dtype=HF)
    g, q, k, v, on = inputs(c)
    dout = randn(g, *q.shape, dtype=HF)
    o, L, _ = ref.attention(q, k, v, c, on)
    got = tk.attention_backward(dout, q, k, v, o.to(HF), L.float(), **how(c, on))
    _, bounds = ref.attention(q, k, v, c, on, L.float(), o.to(HF), dout)
    h = 1e-5

    def f(a, b, d):
        r = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        for q0, q1, k0, k1 in ref.segments(c):
            m = ref.seen(q1 - q0, k1 - k0, c["left"], c["right"], on[k0:k1] != 0)
            for head in range(4):
                s = torch.where(m, a[q0:q1, head] @ b[k0:k1, head // 2].T * c["scale"], -1e300)
                p = torch.softmax(s, 1) * m.any(1, keepdim=True)
                r[q0:q1, head] = torch.where(m, p, 0.0) @ d[k0:k1, head // 2]
        return float((r * dout.double()).sum())

    for i in range(3):
        dirs = [randn(g, *t.shape).double() for t in (q, k, v)]
        plus = f(*(t.double() + h * d for t, d in zip((q, k, v), dirs)))
        minus = f(*(t.double() - h * d for t, d in zip((q, k, v), dirs)))
        num = (plus - minus) / (2 * h)
        mine = sum(float((a.double() * d).sum()) for a, d in zip(got, dirs))
        # the gradients' own bounds, and out's rounding where delta reads it
        room = sum(float((e * d.abs()).sum()) for e, d in zip(bounds, dirs))
        size = sum(float((a.double() * d).abs().sum()) for a, d in zip(got, dirs))
        assert abs(num - mine) <= room + 2.0 ** -10 * size


def test_attention_layouts(tk):
    """Columns of one projection, heads before rows, a padded row stride, segments of equal length without cu."""
    c = case([96, 96, 96], heads=6, kv=2, dim=64, right=0)
    g = gen(2)
    qkv = randn(g, 288, 10, 64, dtype=BF)
    byhead = [randn(g, h, 288, 64, dtype=BF).transpose(0, 1) for h in (6, 2, 2)]
    padded = [randn(g, 288, h * 64 + 24, dtype=BF)[:, :h * 64].view(288, h, 64) for h in (6, 2, 2)]
    for q, k, v in ((qkv[:, :6], qkv[:, 6:8], qkv[:, 8:]), byhead, padded):
        kw = dict(scale=c["scale"], right=0)
        out, lse = tk.attention(q, k, v, n_seg=3, **kw)
        check_forward((out, lse), ref.attention(q, k, v, c))
        same = tk.attention(q, k, v, cu_q=cu(c["nq"]), cu_k=cu(c["nk"]), **kw)
        assert torch.equal(same[0], out) and torch.equal(same[1], lse)
        dout = randn(g, 288, 6, 80, dtype=BF)[..., :64]
        got = tk.attention_backward(dout, q, k, v, out, lse, n_seg=3, **kw)
        want, bounds = ref.attention(q, k, v, c, None, lse, out, dout)
        for a, b, e, what in zip(got, want, bounds, ("dq", "dk", "dv")):
            within(a, b, e, what)


@pytest.mark.parametrize("stride", [0, 8, 260, 1 << 30, 1 << 31])
@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 300), (50, 1), (300, 1)])
def test_attention_of_a_single_row_with_any_row_stride(tk, nq, nk, stride):
    """A tensor of one row may carry any row stride: it has no next row."""
    c = case([nq], [nk], 4, 2, dim=64)
    g, q, k, v, _ = inputs(c)
    dout = randn(g, *q.shape, dtype=BF)

    def odd(t):
        return t.as_strided(t.shape, (stride, 64, 1)) if t.shape[0] == 1 else t

    kw = dict(scale=c["scale"])
    out, lse = tk.attention(odd(q), odd(k), odd(v), **kw)
    check_forward((out, lse), ref.attention(q, k, v, c))
    got = tk.attention_backward(odd(dout), odd(q), odd(k), odd(v), odd(out), lse, **kw)
    want, bounds = ref.attention(q, k, v, c, None, lse, out, dout)
    for a, b, e, what in zip(got, want, bounds, ("dq", "dk", "dv")):
        within(a, b, e, what)


@pytest.mark.parametrize("nq,nk", [([40, 200], [90, 70]), ([2, 1], [900, 1300])])
def test_nan_in_places_that_nothing_admits(tk, nq, nk):
    """Keys that are off, rows that admit no key, and what lies beside the segments."""
    c = case(nq, nk, 2, dim=64, off=0.3, right=0)
    g, q, k, v, on = inputs(c)
    on[nk[0]:] = 0                                     # the last segment admits nothing
    dout = randn(g, *q.shape, dtype=BF)
    kw = how(c, on)
    clean = tk.attention(q, k, v, **kw)
    cleaned = tk.attention_backward(dout, q, k, v, *clean, **kw)
    for bad in (math.nan, math.inf, -math.inf):
        k2, v2, q2, d2 = k.clone(), v.clone(), q.clone(), dout.clone()
        k2[on == 0] = bad
        v2[on == 0] = bad
        q2[nq[0]:] = bad
        d2[nq[0]:] = bad
        out, lse = tk.attention(q2, k2, v2, **kw)
        assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])
        got = tk.attention_backward(d2, q2, k2, v2, out, lse, **kw)
        for a, b in zip(got, cleaned):
            assert torch.equal(a, b)
        assert bool((got[0][nq[0]:] == 0).all()) and bool((got[1][on == 0] == 0).all())


def test_neighbouring_segments_do_not_meet(tk):
    """NaN tokens of one segment stay in it (their rows lie in the same tiles)."""
    c = case([30, 41, 50], heads=2, dim=64)
    g, q, k, v, _ = inputs(c)
    dout = randn(g, *q.shape, dtype=BF)
    kw = how(c, None)
    clean = tk.attention(q, k, v, **kw)
    cleaned = tk.attention_backward(dout, q, k, v, *clean, **kw)
    k2, v2, q2 = k.clone(), v.clone(), q.clone()
    for t in (k2, v2, q2):
        t[30:71] = math.nan
    out, lse = tk.attention(q2, k2, v2, **kw)
    got = tk.attention_backward(dout, q2, k2, v2, out, lse, **kw)
    keep = torch.ones(121, dtype=torch.bool, device="cuda")
    keep[30:71] = False
    assert bool(out[30:71].isnan().all()) and torch.equal(out[keep], clean[0][keep])
    for a, b in zip(got, cleaned):
        assert torch.equal(a[keep], b[keep])


def test_rows_outside_every_segment_stay(tk, gs):
    c = case([20, 30], heads=1, dim=64)
    g, q, k, v, _ = inputs(c)
    out, lse = torch.full_like(q, 7.0), torch.full((50, 1), 7.0, device="cuda")
    starts = torch.tensor([5, 20, 44], dtype=torch.int32, device="cuda")
    a = gs.make_attn(q, k, v, 0.125, cu_q=starts, cu_k=starts)
    n = gs.gs_attention_ws_bytes(a)
    gs.gs_attention(a, out, lse, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
    assert bool((out[:5] == 7).all()) and bool((out[44:] == 7).all()) and bool((lse[44:] == 7).all())
    want = tk.attention(q[5:20].clone(), k[5:20].clone(), v[5:20].clone(), scale=0.125)
    assert torch.equal(out[5:20], want[0])


@pytest.mark.parametrize("rows", [40, 2])
def test_rows_outside_every_segment_stay_where_keys_are_cut(tk, gs, rows):
    c = case([rows + 10], [5000], heads=2, kv=1, dim=64)
    g, q, k, v, _ = inputs(c)
    out, lse = torch.full_like(q, 7.0), torch.full((rows + 10, 2), 7.0, device="cuda")
    cu_q, cu_k = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([5, 5 + rows], [3, 4990]))
    a = gs.make_attn(q, k, v, 0.125, cu_q=cu_q, cu_k=cu_k)
    gs.gs_attention(a, out, lse, torch.full((gs.gs_attention_ws_bytes(a),), 64, dtype=torch.uint8, device="cuda"))
    for t in (out, lse):
        assert bool((t[:5] == 7).all()) and bool((t[5 + rows:] == 7).all()) and bool((t[5:5 + rows] != 7).all())


def test_keys_outside_every_segment_stay_where_rows_are_cut(tk, gs):
    c = case([2500], [130], heads=2, kv=1, dim=64)
    g, q, k, v, _ = inputs(c)
    out, lse = tk.attention(q, k, v)
    dq, dk, dv = (torch.full_like(t, 7.0) for t in (q, k, v))
    cu_q, cu_k = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([5, 2400], [3, 120]))
    a = gs.make_attn(q, k, v, 0.125, cu_q=cu_q, cu_k=cu_k)
    n = gs.gs_attention_ws_bytes(a, True)
    gs.gs_attention_bwd(a, out, lse, torch.ones_like(q), dq, dk, dv, torch.full((n,), 64, dtype=torch.uint8, device="cuda"))
    for t, lo, hi in ((dq, 5, 2400), (dk, 3, 120), (dv, 3, 120)):
        assert bool((t[:lo] == 7).all()) and bool((t[hi:] == 7).all()) and bool((t[lo:hi] != 7).any(-1).all())


def test_offsets_past_32_bits(tk):
    """Keys and values whose rows lie 2^20 elements apart: the last is past 2^32 bytes and 2^31 elements."""
    n, ld = 2100, 1 << 20
    big = torch.empty(n * ld, dtype=BF, device="cuda")
    g = gen(4)
    k, v = (big[o:].as_strided((n, 1, 64), (ld, 64, 1)) for o in (0, 64))
    k.copy_(randn(g, n, 1, 64, dtype=BF))
    v.copy_(randn(g, n, 1, 64, dtype=BF))
    for nq in (3, 200):
        c = case([nq], [n], 1, dim=64)
        q, dout = randn(g, nq, 1, 64, dtype=BF), randn(g, nq, 1, 64, dtype=BF)
        kc, vc = k.contiguous(), v.contiguous()
        got, want = tk.attention(q, k, v), tk.attention(q, kc, vc)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        check_forward(got, ref.attention(q, kc, vc, c))
        mine = tk.attention_backward(dout, q, k, v, *got)
        same = tk.attention_backward(dout, q, kc, vc, *got)
        assert all(torch.equal(a, b) for a, b in zip(mine, same))


def test_large_scores(tk):
    """Scores far apart: the running maximum carries them, one key takes all."""
    c = case([70], [300], 2, dim=64)
    g, q, k, v, _ = inputs(c)
    q = (q.float() * 30).to(BF)
    got = tk.attention(q, k, v, scale=c["scale"])
    check_forward(got, ref.attention(q, k, v, c))


@pytest.mark.parametrize("nq", [40, 2])
@pytest.mark.parametrize("rise", [4.0, -40.0, 40.0, 400.0])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_rising_scores(tk, nq, rise, dtype):
    """Scores that climb (or fall) along the keys: the maximum that the sums stand against is passed by a little, again
    and again, or by much in a few keys."""
    c = case([nq], [900], 2, dim=64, dtype=dtype)
    g, q, k, v, _ = inputs(c)
    q[..., 0] = 8.0
    k[..., 0] = (torch.arange(900, device="cuda") * (rise / 900))[:, None].to(dtype)
    got = tk.attention(q, k, v, scale=c["scale"])
    check_forward(got, ref.attention(q, k, v, c))


def test_other_stream_and_graph(tk):
    c = case([100, 30], heads=4, kv=2, dim=64, right=0)
    g, q, k, v, _ = inputs(c)
    kw = how(c, None)
    want = tk.attention(q, k, v, **kw)
    dout = randn(g, *q.shape, dtype=BF)
    grads = tk.attention_backward(dout, q, k, v, *want, **kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = tk.attention(q, k, v, **kw)
        more = tk.attention_backward(dout, q, k, v, *got, **kw)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and all(torch.equal(a, b) for a, b in zip(more, grads))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o2, l2 = tk.attention(q, k, v, **kw)
        g2 = tk.attention_backward(dout, q, k, v, o2, l2, **kw)
        n2 = tk.rms_norm(q.view(130, -1), torch.ones(256, device="cuda"))
    for i in range(3):
        q.copy_(randn(g, *q.shape, dtype=BF))
        graph.replay()
        want = tk.attention(q, k, v, **kw)
        grads = tk.attention_backward(dout, q, k, v, *want, **kw)
        y = tk.rms_norm(q.view(130, -1), torch.ones(256, device="cuda")).y
        torch.cuda.synchronize()
        assert torch.equal(o2, want[0]) and all(torch.equal(a, b) for a, b in zip(g2, grads))
        assert torch.equal(n2.y, y)


def test_autograd(tk):
    """The autograd forms give what the functions give, and sum a shared input's gradients."""
    g = gen(6)
    x = randn(g, 60, 128, dtype=BF).requires_grad_()
    res = randn(g, 60, 128, dtype=BF).requires_grad_()
    w = (1 + randn(g, 128)).requires_grad_()
    y, total = tk.RmsNorm.apply(x, res, w, 1e-6)
    pos, freq = randn(g, 60, 3) * 9, torch.rand(9, generator=g, device="cuda")
    q, k = tk.Rotary.apply(y.view(60, 4, 32), y.view(60, 4, 32)[:, :2], pos, freq, (3, 3, 3), False, 1.0)
    out, lse = tk.Attention.apply(q, k, total.view(60, 4, 32)[:, 2:], dict(right=0))
    d = randn(g, 60, 4, 32, dtype=BF)
    out.backward(d)
    dq, dk, dv = tk.attention_backward(d, q.detach(), k.detach(), total.detach().view(60, 4, 32)[:, 2:], out.detach(),
                                       lse, right=0)
    dq, dk = tk.rotary((dq, dk), pos, freq, (3, 3, 3), inverse=True)
    dy = dq.clone()
    dy[:, :2] += dk
    dt = torch.zeros_like(dq)
    dt[:, 2:] += dv
    dx, dw = tk.rms_norm_backward(dy.view(60, 128), total.detach(), w.detach(), 1e-6, dtotal=dt.view(60, 128))
    assert torch.equal(x.grad, dx) and torch.equal(res.grad, dx) and torch.equal(w.grad, dw)


def test_refusals(tk, gs):
    t = torch.zeros(8, 2, 64, dtype=BF, device="cuda")
    with pytest.raises(ValueError):
        tk.attention(t, t, t.float())
    with pytest.raises(ValueError):
        tk.attention(t.cpu(), t, t)
    with pytest.raises(gs.GsmiError):
        tk.attention(t.float(), t.float(), t.float())              # 16-bit types only
    with pytest.raises(gs.GsmiError):
        tk.attention(t, t[:, :1], t[:, :1], scale=0.0)
    with pytest.raises(gs.GsmiError):
        tk.attention(t, t, t, n_seg=3)                             # 3 does not divide 8
    with pytest.raises(ValueError):
        tk.attention(t, t, t, cu_q=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        tk.attention(t, t, t, key_on=torch.ones(7, dtype=torch.uint8, device="cuda"))
    odd = torch.zeros(8 * 2 * 64 + 1, dtype=BF, device="cuda")[1:].view(8, 2, 64)
    with pytest.raises(gs.GsmiError):
        tk.attention(t, odd, t)                                    # keys not 16-byte aligned
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    with pytest.raises(ValueError):
        tk.rms_norm(x, w[:32])
    with pytest.raises(ValueError):
        tk.rms_norm(x, w, residual=x.to(BF))
    with pytest.raises(gs.GsmiError):
        tk.rms_norm(x, w, eps=-1.0)
    with pytest.raises(ValueError):
        tk.rms_norm(x.to(torch.float64), w)
    with pytest.raises(ValueError):
        tk.rotary(t, torch.zeros(7, 1, device="cuda"), torch.zeros(4, device="cuda"), [4])
    with pytest.raises(gs.GsmiError):
        tk.rotary(t, torch.zeros(8, 1, device="cuda"), torch.zeros(40, device="cuda"), [40])
