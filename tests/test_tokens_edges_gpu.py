"""The token operators at the ends of their numbers' ranges and of their layouts: tiny and special rows of the 8-bit
norm, rows outside every segment, large scores, heads and rows whose strides mean nothing, very many rows."""
import math

import pytest
import torch

import token_refs as ref
from test_tokens_gpu import BF, F32, HF, case, cu, gen, gs, inputs, randn, tk, within  # noqa: F401 (gs, tk: fixtures)

pytestmark = pytest.mark.gpu
LEAST = 2.0 ** -126                                    # least scale of a block


def check_8bit(e, y):
    """q and scale against y in double: the scale is max|y| / 448, at least 2^-126, 1 for zeros; q the nearest."""
    rows, cols = y.shape
    top = torch.stack([b.abs().amax(1) for b in y.split(128, 1)], 1)
    want = torch.where(top > 0, (top / 448).clamp(min=LEAST), torch.ones_like(top))
    # fp32: the squares' sum, root, reciprocal and two products
    within(e.scale, want, (cols / 64 + 40) * 2.0 ** -24 * want, "scale")
    v = y / e.scale.double()[:, torch.arange(cols, device="cuda") // 128]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    # half a step, and the scale's and the norm's own roundings (a few 2^-24 of v each)
    within(e.q.float(), v, step * 0.5 * (1 + 1e-3) + 1e-4 * v.abs(), "q")


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("weights", ["ones", "some", "tiny block"])
def test_norm_8bit_of_tiny_values(tk, dtype, weights):
    """Values whose quotient 448 / max|s w| or 1 / scale is past the largest fp32 number."""
    g = gen(21)
    cols = 300
    x = randn(g, 8, cols)
    x[0] *= 1e-37
    x[1] *= 0.1
    x[1, 128:256] *= 1e-39
    x[1, 140:150] = 0.0
    x[1, 256:] *= 1e-37
    x[2] *= 1e-30
    x[3] *= 1e-41
    x[4] *= 1e-3
    x[4, 128:256] *= 2e-35
    x[5] *= 1e15
    x[5, 128:256] *= 1e-53
    x[6, 128:] = 0.0
    x[7] *= 1e-37
    x[7, 1:] = 0.0
    x = x.to(dtype)
    w = torch.ones(cols, device="cuda")
    if weights != "ones":
        w = 1 + 0.2 * randn(g, cols)
    if weights == "tiny block":
        w[128:256] *= 1e-37
    for res in (None, x.flip(1).contiguous()):
        y, _ = ref.norm(x, w, 1e-6, res)
        check_8bit(tk.rms_norm(x, w, 1e-6, residual=res, eight_bit=True), y)


def test_norm_8bit_without_eps(tk):
    """Nothing added to the squares' mean: rows of any size give the same quotients."""
    g = gen(22)
    x = randn(g, 5, 200) * torch.tensor([1e-17, 1e-10, 1.0, 1e10, 1e17], device="cuda")[:, None]
    w = 1 + 0.2 * randn(g, 200)
    y, _ = ref.norm(x, w, 0.0)
    check_8bit(tk.rms_norm(x, w, 0.0, eight_bit=True), y)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_norm_8bit_of_special_rows(tk, dtype):
    """NaN, infinities and sums past the range: the scale is that of the block's numbers, 1 where none is left."""
    g = gen(23)
    x = randn(g, 5, 300)
    x[1, 7] = math.nan                                 # y is NaN throughout
    x[2, 200] = math.inf                               # y is NaN there and 0 elsewhere
    x[3, 0] = 1e25                                     # the squares' sum is infinite: y is 0
    x[4] = 0.0
    x = x.to(dtype)
    w = torch.ones(300, device="cuda")
    e = tk.rms_norm(x, w, 1e-6, eight_bit=True)
    q = e.q.float()
    assert bool((e.scale[1:] == 1).all())
    assert bool(q[1].isnan().all()) and bool((q[3:] == 0).all())
    assert torch.equal(q[2].isnan(), torch.arange(300, device="cuda") == 200) and float(q[2].nan_to_num().abs().max()) == 0
    clean = tk.rms_norm(x[:1], w, 1e-6, eight_bit=True)
    assert torch.equal(clean.q[0].float(), q[0]) and torch.equal(clean.scale[0], e.scale[0])
    # without eps a row of zeros is 0 / 0
    z = tk.rms_norm(x[4:], w, 0.0, eight_bit=True)
    assert bool((z.scale == 1).all()) and bool(z.q.float().isnan().all())
    # a weight: NaN stays with its column, an infinity takes its block
    for bad in (math.nan, math.inf):
        w2 = w.clone()
        w2[130] = bad
        e = tk.rms_norm(x[:1], w2, 1e-6, eight_bit=True)
        q = e.q.float()[0]
        others = torch.arange(300, device="cuda") // 128 != 1
        assert torch.equal(q[others], clean.q[0].float()[others])
        assert torch.equal(e.scale[0, ::2], clean.scale[0, ::2])
        if bad == math.inf:
            assert float(e.scale[0, 1]) == math.inf and bool(q[128:256].isnan().all())
        else:
            assert bool(q[130].isnan()) and int(q.isnan().sum()) == 1
            w2[130] = 0.0
            without = tk.rms_norm(x[:1], w2, 1e-6, eight_bit=True)
            assert torch.equal(e.scale, without.scale)
            keep = torch.arange(300, device="cuda") != 130
            assert torch.equal(q[keep], without.q.float()[0][keep])


@pytest.mark.parametrize("heads,nq,nk,starts_q,starts_k", [
    (2, 50, 60, [5, 20, 44], [3, 30, 51]), (2, 50, 5000, [5, 45], [3, 4990]), (2, 12, 5000, [5, 7], [3, 4990]),
    (4, 2500, 130, [5, 2400], [3, 120]), (1, 300, 400, [7] + list(range(7, 270, 3)), [9] + list(range(9, 360, 4))[:88]),
    (2, 40, 40, [0, 0, 0], [0, 0, 0]), (2, 40, 40, [40, 40], [40, 40])])
def test_rows_outside_every_segment_are_zeros(tk, heads, nq, nk, starts_q, starts_k):
    """A buffer at capacity whose count is on the device: the rows past it are no one's, and no one's gradient."""
    c = case([nq], [nk], heads, 1, dim=64)
    g, q, k, v, _ = inputs(c)
    dout = randn(g, *q.shape, dtype=BF)
    cu_q, cu_k = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (starts_q, starts_k))
    assert len(starts_q) == len(starts_k)
    on = torch.ones(nk, dtype=torch.uint8, device="cuda")
    for flags in (None, on):
        junk = [torch.full((1 << 20,), 7.0, device="cuda") for _ in range(8)]     # what fresh outputs may hold
        junk += [torch.full((n,), 7.0, dtype=t, device="cuda") for n, t in
                 [(q.numel(), BF), (k.numel(), BF), (nq * heads, F32)] for _ in range(4)]
        del junk
        out, lse = tk.attention(q, k, v, cu_q, cu_k, key_on=flags)
        dq, dk, dv = tk.attention_backward(dout, q, k, v, out, lse, cu_q, cu_k, key_on=flags)
        for t, (lo, hi) in ((out, (starts_q[0], starts_q[-1])), (dq, (starts_q[0], starts_q[-1])),
                            (dk, (starts_k[0], starts_k[-1])), (dv, (starts_k[0], starts_k[-1]))):
            assert bool((t[:lo] == 0).all()) and bool((t[hi:] == 0).all())
            assert bool((t[lo:hi] != 0).any(-1).all())
        lo, hi = starts_q[0], starts_q[-1]
        assert bool((lse[:lo] == -math.inf).all()) and bool((lse[hi:] == -math.inf).all())
        assert bool(torch.isfinite(lse[lo:hi]).all())


def test_rotary_in_place_is_seen_by_autograd(tk):
    g = gen(31)
    x, w = randn(g, 20, 2, 64), randn(g, 20, 2, 64).requires_grad_()
    pos, freq = randn(g, 20, 1), torch.rand(32, generator=g, device="cuda")
    before = x._version
    y = (x * w).sum()                                  # saves x
    (z,) = tk.rotary(x, pos, freq, [32], inplace=True)
    assert z is x and x._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.mark.parametrize("stride", [0, 3, 1 << 40])
@pytest.mark.parametrize("nq,nk", [(150, 150), (3, 900)])
def test_attention_of_a_single_head_with_any_head_stride(tk, nq, nk, stride):
    """A tensor of one head may carry any head stride: it has no next head."""
    c = case([nq], [nk], 1, dim=64)
    g, q, k, v, _ = inputs(c)
    dout = randn(g, *q.shape, dtype=BF)
    want = tk.attention(q, k, v)
    grads = tk.attention_backward(dout, q, k, v, *want)
    q, k, v, dout, out = (t.as_strided(t.shape, (64, stride, 1)) for t in (q, k, v, dout, want[0]))
    got = tk.attention(q, k, v)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all(torch.equal(a, b) for a, b in zip(tk.attention_backward(dout, q, k, v, out, want[1]), grads))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_large_equal_scores_beside_rising_ones(tk, dtype):
    """Rows whose scores are all the same large number, in a wave with one whose maximum rises at every step: what they
    have summed keeps its weight.  Values are +1 in the first half and -1 in the second, so the mean is 0."""
    n, heads = 8192, 8
    q = torch.zeros(n, heads, 64, dtype=dtype, device="cuda")
    k, v = (torch.zeros(n, heads, 64, dtype=dtype, device="cuda") for _ in range(2))
    q[..., 0] = 64.0
    q[::32, :, 0] = 0.0
    q[::32, :, 1] = 64.0
    k[..., 0] = 508.0                                  # 32512 scale log2(e) lies between two fp32 numbers
    k[..., 1] = (torch.arange(n, device="cuda") // 64).to(dtype)[:, None]       # 8 a step: 11.5 powers of two
    v[:n // 2], v[n // 2:] = 1.0, -1.0
    out, lse = tk.attention(q, k, v, scale=0.125)
    flat = torch.arange(n, device="cuda") % 32 != 0
    # one rounding of each probability and of the result, fp32 sums (as in token_refs.attention)
    room = ref.UNIT[dtype] + 2e-5
    assert float(out[flat].float().abs().max()) <= room, float(out[flat].float().abs().max())
    s = 8.0 * float(k[0, 0, 0])
    assert float((lse[flat].double() - (s + math.log(n))).abs().max()) <= 2e-5 * (1 + s)


@pytest.mark.parametrize("rows,cols,dtype", [((1 << 23) + 5, 8, BF), ((1 << 27) + 3, 4, F32)])
def test_norm_of_very_many_rows(tk, rows, cols, dtype):
    """More rows than a launch of one thread group a row holds."""
    g = gen(41)
    x = torch.empty(rows, cols, dtype=dtype, device="cuda").normal_(generator=g)
    w = 1 + randn(g, cols)
    y = tk.rms_norm(x, w, 1e-6).y
    e = tk.rms_norm(x, w, 1e-6, eight_bit=True)
    edge = [0, 1, (1 << 22) - 1, 1 << 22, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, rows // 2, rows - 2, rows - 1]
    at = torch.cat((torch.tensor(edge, device="cuda"),
                    torch.randint(0, rows, (4000,), generator=g, device="cuda")))
    want, _ = ref.norm(x[at], w, 1e-6)
    within(y[at], want, (ref.UNIT[dtype] + 41 * 2.0 ** -24) * want.abs() + 4 * ref.TINY[dtype], "y")
    few = tk.rms_norm(x[at], w, 1e-6, eight_bit=True)
    assert torch.equal(e.q[at].float(), few.q.float()) and torch.equal(e.scale[at], few.scale)


def test_rotary_of_very_many_tokens(tk):
    """More workgroups than a launch holds: 2^27 tokens of one head of 512, 137 GB turned in place."""
    n, dim, slab = (1 << 27) + 9, 512, 1 << 20
    if torch.cuda.mem_get_info()[0] < (n * dim * 2) * 5 // 4:
        torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < (n * dim * 2) * 5 // 4:
        pytest.skip("needs 172 GB of free memory")
    g = gen(43)
    x = torch.empty(n, 1, dim, dtype=BF, device="cuda")
    some = randn(g, slab, 1, dim, dtype=BF)
    for first in range(0, n, slab):
        x[first:first + slab].copy_(some[:min(slab, n - first)])
    pos = torch.rand(n, 1, generator=g, device="cuda") * 100
    freq = torch.rand(dim // 2, generator=g, device="cuda")
    edge = [e + d for e in (0, 1 << 25, 1 << 26, 3 << 25, 1 << 27) for d in (-1, 0, 1) if 0 <= e + d < n] + [n - 1]
    at = torch.cat((torch.tensor(edge, device="cuda"), torch.randint(0, n, (2000,), generator=g, device="cuda")))
    before = x[at]
    tk.rotary(x, pos, freq, [dim // 2], inplace=True)
    want = tk.rotary(before, pos[at], freq, [dim // 2])[0]
    assert torch.equal(x[at], want)
    del x, pos
    torch.cuda.empty_cache()


@pytest.mark.parametrize("cols", [1, 40, 128, 200, 256, 1000, 1536, 2048, 2500, 8200, 16384])
@pytest.mark.parametrize("dtype", [F32, BF, HF])
def test_norm_8bit_of_tiny_blocks_at_every_width(tk, cols, dtype):
    """Rows that share a wave, a row a wave and a row a workgroup: tiny and zero blocks get their numbers and leave the
    bits of the rows beside them as they are."""
    g = gen(24 + cols)
    x = randn(g, 37, cols)
    w = 1 + 0.2 * randn(g, cols)
    tiny = torch.arange(37, device="cuda") % 3 == 1
    block = torch.arange(cols, device="cuda") // 128 % 2 == (1 if cols > 128 else 0)
    alone = tk.rms_norm(x[~tiny].to(dtype), w, 1e-6, eight_bit=True)
    small = 6e-8 if dtype == HF else 1e-38
    x[tiny] = torch.where(block, x[tiny] * small, x[tiny])
    x[1] = 0.0
    x[4] = 0.0
    x[4, cols // 2] = small
    x = x.to(dtype)
    e = tk.rms_norm(x, w, 1e-6, eight_bit=True)
    check_8bit(e, ref.norm(x, w, 1e-6)[0])
    assert torch.equal(e.q[~tiny].float(), alone.q.float()) and torch.equal(e.scale[~tiny], alone.scale)
