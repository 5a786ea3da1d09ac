"""Plain 64-bit forms of the layer norm, the embedding, the gated recurrence and the kept gated SiLU, with the error
bounds that fp32 arithmetic and one rounding to the operators' types give for each output element."""
import torch

from token_refs import TINY, UNIT

F = 2.0 ** -24                                         # half a step of fp32, relative


def layer(x, weight, bias, eps, residual=None):
    """(y, total, bound of y) in double."""
    s = x.double() if residual is None else x.double() + residual.double()
    n, rho, En, _ = _normed(s, eps)
    w, b = weight.double(), torch.zeros_like(weight.double()) if bias is None else bias.double()
    y = n * w + b
    # n's error, the product and the sum with the bias, the rounding to the type
    bound = En * w.abs() + 3 * F * ((n * w).abs() + b.abs()) + UNIT[x.dtype] * y.abs() + 4 * TINY[x.dtype]
    return y, s, bound


def _normed(s, eps):
    """(n, rho, bound of n's error, bound of rho's relative error)."""
    cols = s.shape[1]
    adds = cols / 64 + 40                              # of a sum over the row: in a lane, then over the lanes
    m = s.mean(1, keepdim=True)
    d = s - m
    var = (d * d).mean(1, keepdim=True)
    rho = 1 / torch.sqrt(var + eps)
    # the sum with the residual, the mean's sum, the difference
    Ed = F * (s.abs() + d.abs() + adds * s.abs().mean(1, keepdim=True))
    # half the variance's relative error; root, reciprocal and product
    Er = 0.5 * (2 * (d.abs() * Ed).mean(1, keepdim=True) + (Ed * Ed).mean(1, keepdim=True) + adds * F * var) * rho ** 2 + 6 * F
    n = d * rho
    return n, rho, rho * Ed * (1 + Er) + n.abs() * (Er + F), Er


def layer_bwd(dy, total, weight, eps, dtotal=None):
    """((dx, dweight, dbias), bounds) in double."""
    s, g0, w = total.double(), dy.double(), weight.double()
    rows, cols = s.shape
    adds = cols / 64 + 40
    n, rho, En, Er = _normed(s, eps)
    g = g0 * w
    mg, mgn = g.mean(1, keepdim=True), (g * n).mean(1, keepdim=True)
    inner = g - mg - n * mgn
    dx = rho * inner + (0 if dtotal is None else dtotal.double())
    Emg = (adds + 2) * F * g.abs().mean(1, keepdim=True)
    # the sum is over g (s - m), multiplied by rho behind it
    Emgn = (adds + 4) * F * (g * n).abs().mean(1, keepdim=True) + (g.abs() * En).mean(1, keepdim=True)
    size = g.abs() + mg.abs() + (n * mgn).abs()
    bdx = rho * (Emg + En * mgn.abs() + (n.abs() + En) * Emgn + 4 * F * size + Er * inner.abs()) \
        + (UNIT[total.dtype] + 2 * F) * dx.abs() + 2 * F * (rho * inner).abs() + 4 * TINY[total.dtype]
    walk = rows / min(512, -(-rows // 4)) + 100         # a workgroup's rows, then the partial rows
    bdw = walk * F * (g0 * n).abs().sum(0) + (g0.abs() * En).sum(0) + 1e-38
    bdb = walk * F * g0.abs().sum(0) + 1e-38
    return (dx, (g0 * n).sum(0), g0.sum(0)), (bdx, bdw, bdb)


def layout(n, cu, reverse):
    """(order, first, last, segment): tokens in the recurrence's order, with what each is in its segment (-1: none)."""
    seg = torch.full((n,), -1, dtype=torch.long)
    first, last = torch.zeros(n, dtype=torch.bool), torch.zeros(n, dtype=torch.bool)
    at = [min(max(c, 0), n) for c in cu]
    for s in range(len(at) - 1):
        if at[s] < at[s + 1]:
            seg[at[s]:at[s + 1]] = s
            first[at[s + 1] - 1 if reverse else at[s]] = True
            last[at[s] if reverse else at[s + 1] - 1] = True
    order = torch.arange(n)
    if reverse:
        order = order.flip(0)
    return order, first, last, seg


def _gates(g):
    g = g.double().cpu()
    # exp's argument is rounded in fp32 and its function is two units off, the reciprocal and the difference one each
    return torch.sigmoid(g), torch.sigmoid(-g), (8 + 2 * (float(g.abs().max()) if g.numel() else 0.0)) * F


def recurrence(x, gate, cu, initial=None, reverse=False):
    """dict of y, final, kept (CPU, double) and their bounds, and of what the gradient needs."""
    n, cols = x.shape
    order, first, last, seg = layout(n, cu, reverse)
    a, z, c = _gates(gate)
    xd = x.double().cpu()
    h0 = torch.zeros(len(cu) - 1, cols, dtype=torch.float64) if initial is None else initial.double().cpu()
    y, By = torch.zeros(n, cols, dtype=torch.float64), torch.zeros(n, cols, dtype=torch.float64)
    before, Bbefore = torch.zeros_like(y), torch.zeros_like(y)
    final, Bfinal = h0.clone(), torch.zeros_like(h0)
    kept = torch.zeros(-(-n // 64), cols, dtype=torch.float64)
    Bkept = torch.zeros_like(kept)
    h = size = far = torch.zeros(cols, dtype=torch.float64)
    for p in range(n):
        t = int(order[p])
        if seg[t] < 0:
            continue
        if first[t]:
            h, size, far = h0[seg[t]], h0[seg[t]].abs(), torch.zeros(cols, dtype=torch.float64)
        elif p % 64 == 0:
            kept[p // 64], Bkept[p // 64] = h, c * (size + far)
        before[t], Bbefore[t] = h, c * (size + far) * (not first[t])
        h = a[t] * h + z[t] * xd[t]
        # the sum of the terms' sizes, and of the sizes times the gates that each has passed: every gate brings its own
        # relative error
        far = a[t] * (far + size)
        size = a[t] * size + z[t] * xd[t].abs()
        y[t], By[t] = h, c * (size + far)
        if last[t]:
            final[seg[t]], Bfinal[seg[t]] = h, c * (size + far)
    out = dict(y=y, final=final, kept=kept, before=before, Bbefore=Bbefore)
    out["By"] = By + UNIT[x.dtype] * y.abs() + TINY[x.dtype]
    out["Bfinal"], out["Bkept"] = Bfinal + 1e-38, Bkept + 1e-38
    return out


def recurrence_bwd(dy, x, gate, cu, initial=None, dfinal=None, reverse=False):
    """((dx, dgate, dinitial), bounds) on the CPU in double."""
    n, cols = x.shape
    order, first, last, seg = layout(n, cu, reverse)
    f = recurrence(x, gate, cu, initial, reverse)
    a, z, c = _gates(gate)
    xd, dyd = x.double().cpu(), dy.double().cpu()
    zero = torch.zeros(len(cu) - 1, cols, dtype=torch.float64)
    df = zero if dfinal is None else dfinal.double().cpu()
    dx, dg, di = torch.zeros_like(xd), torch.zeros_like(xd), df.clone()
    bx, bg, bi = torch.zeros_like(xd), torch.zeros_like(xd), torch.zeros_like(zero)
    carry = size = far = torch.zeros(cols, dtype=torch.float64)
    for p in range(n - 1, -1, -1):
        t = int(order[p])
        s = int(seg[t])
        if s < 0:
            continue
        if last[t]:
            carry, size, far = df[s], df[s].abs(), torch.zeros(cols, dtype=torch.float64)
        D, sD = dyd[t] + carry, dyd[t].abs() + size
        eD = c * (sD + far)
        e = f["before"][t] - xd[t]
        dx[t], dg[t] = z[t] * D, a[t] * z[t] * e * D
        bx[t] = z[t] * (eD + c * D.abs())
        bg[t] = a[t] * z[t] * (f["Bbefore"][t] * (D.abs() + eD) + e.abs() * eD
                               + c * (f["before"][t].abs() + xd[t].abs()) * D.abs())
        far = a[t] * (far + sD)
        carry, size = a[t] * D, a[t] * sD
        if first[t]:
            di[s], bi[s] = carry, c * (size + far)
    u, tiny = UNIT[x.dtype], TINY[x.dtype]
    return (dx, dg, di), (bx + u * dx.abs() + tiny, bg + u * dg.abs() + tiny, bi + 1e-38)


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis in double, by doubling."""
    a, b = a.clone(), b.clone()
    d = 1
    while d < len(a):
        b[d:] = b[d:] + a[d:] * b[:-d]
        a[d:] = a[d:] * a[:-d]
        d *= 2
    return b


def long_recurrence(x, gate, cu, dy, reverse=False):
    """((y, dx, dgate), bounds) as the two above give them, for lists of which cu's segments hold every token."""
    a, z, c = _gates(gate)
    xd, dyd = x.double().cpu(), dy.double().cpu()
    if reverse:
        n = len(xd)
        (y, dx, dg), b = long_recurrence(x.flip(0), gate.flip(0), [n - v for v in cu][::-1], dy.flip(0))
        return tuple(t.flip(0) for t in (y, dx, dg)), tuple(t.flip(0) for t in b)
    first = torch.zeros(len(xd), 1, dtype=torch.float64)
    first[torch.tensor([v for v in cu if v < len(xd)])] = 1
    last = first.roll(-1, 0)
    behind = lambda t: t.roll(1, 0) * (1 - first)          # of the token in front
    ahead = lambda t: t.roll(-1, 0) * (1 - last)
    A = a * (1 - first)
    h, size = _scan(A, z * xd), _scan(A, z * xd.abs())
    far = _scan(A, A * behind(size))
    back = lambda p, q: _scan(p.flip(0), q.flip(0)).flip(0)
    P = ahead(a)
    D, sD = back(P, dyd), back(P, dyd.abs())
    eD = c * (sD + back(P, P * ahead(sD)))
    e = behind(h) - xd
    dx, dg = z * D, a * z * e * D
    bx = z * (eD + c * D.abs())
    bg = a * z * (behind(c * (size + far)) * (D.abs() + eD) + e.abs() * eD + c * (behind(h).abs() + xd.abs()) * D.abs())
    u, tiny = UNIT[x.dtype], TINY[x.dtype]
    return (h, dx, dg), (c * (size + far) + u * h.abs() + tiny, bx + u * dx.abs() + tiny, bg + u * dg.abs() + tiny)


def eight(u):
    """(rows in e4m3, scale bytes) on u's device: exact quotients by the least power of two, one rounding."""
    rows, cols = u.shape
    blocks = -(-cols // 32)
    w = torch.zeros(rows, blocks * 32, dtype=torch.float64, device=u.device)
    w[:, :cols] = u.double()
    w = w.view(rows, blocks, 32)
    top = torch.where(torch.isfinite(w), w.abs(), 0.0).amax(2) if rows else w.new_zeros(rows, blocks)
    m, e = torch.frexp(top)                            # 448 is 7/8 of 2^9
    k = torch.where(top == 0, -127, torch.where(m > 0.875, e - 8, e - 9).clamp(min=-127))
    v = w / torch.exp2(k.double())[:, :, None]
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    q = torch.where(torch.isfinite(v), torch.round(v / step) * step, torch.nan)
    return q.view(rows, blocks * 32)[:, :cols], (k + 127).to(torch.uint8)


def wide(q, scale):
    return q.double() * torch.exp2(scale.double() - 127).repeat_interleave(32, 1)[:, :q.shape[1]]


def silu(u, v=None):
    """(h, bound) in double."""
    a = u.double()
    h = a * torch.sigmoid(a) * (1 if v is None else v.double())
    # exp's rounded argument and its function, twice, the sum, the reciprocal, four products; below the normal numbers
    # a product is off by half of 2^-149, times the factors behind it
    return h, (UNIT[u.dtype] + (12 + 2 * a.abs()) * F) * h.abs() + 4 * TINY[u.dtype] + 2.0 ** -147 * (1 + (0 if v is None else v.double().abs()))


def silu_bwd(dh, u, v=None):
    """((du, dv, h), bounds) in double, at u and v in double."""
    unit, tiny = UNIT[dh.dtype], TINY[dh.dtype]
    d, s, r = dh.double(), torch.sigmoid(u), torch.sigmoid(-u)
    f = 1 if v is None else v
    du, dv, h = d * f * (s + u * s * r), d * u * s, u * s * f
    c = (14 + 2 * u.abs()) * F
    floor = 4 * tiny + 2.0 ** -147 * (1 + d.abs() + (1 + u.abs()) * (0 if v is None else v.abs()) + (1 + u.abs()) * (d * f).abs())
    bu = unit * du.abs() + c * (d * f).abs() * (s + (u * s * r).abs()) + floor
    return (du, dv, h), (bu, (unit + c) * dv.abs() + floor, (unit + c) * h.abs() + floor)
