"""Plain 64-bit forms of the token operators (torch, double), with the error
bounds that rounding to the operators' types gives for each output element."""
import math

import torch

# largest relative error of rounding to nearest
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# largest absolute error below the type's normal range
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


def norm(x, weight, eps, residual=None):
    """(y, total) in double."""
    s = x.double() if residual is None else x.double() + residual.double()
    return s * weight.double() / torch.sqrt(s.pow(2).mean(1, keepdim=True) + eps), s


def norm_bwd(dy, total, weight, eps, dtotal=None):
    """(dx, dweight, sum |dy n|) in double."""
    x, g = total.double(), dy.double()
    r = 1.0 / torch.sqrt(x.pow(2).mean(1, keepdim=True) + eps)
    n, gw = x * r, g * weight.double()
    dx = r * (gw - n * (gw * n).mean(1, keepdim=True))
    if dtotal is not None:
        dx = dx + dtotal.double()
    return dx, (g * n).sum(0), (g * n).abs().sum(0)


def rotary(x, pos, freq, axis_pairs, interleaved, inverse=False, amplitude=1.0):
    """(turned, |a| + |b| of every element's pair)."""
    pairs = sum(axis_pairs)
    axis = torch.repeat_interleave(torch.arange(len(axis_pairs)), torch.tensor(axis_pairs)).to(pos.device)
    t = pos.double()[:, axis] * freq.double() * (-1 if inverse else 1)
    c, s = amplitude * torch.cos(t)[:, None], amplitude * torch.sin(t)[:, None]
    y, size = x.double().clone(), x.double().abs()
    ia = torch.arange(pairs) * 2 if interleaved else torch.arange(pairs)
    ib = ia + 1 if interleaved else ia + pairs
    a, b = x.double()[..., ia], x.double()[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return y, size


def segments(case):
    """(q0, q1, k0, k1) of every segment."""
    q = [0] + torch.tensor(case["nq"]).cumsum(0).tolist()
    k = [0] + torch.tensor(case["nk"]).cumsum(0).tolist()
    return [(q[i], q[i + 1], k[i], k[i + 1]) for i in range(len(case["nq"]))]


def seen(nq, nk, left, right, on):
    place = torch.arange(nq)[:, None] + nk - nq
    key = torch.arange(nk)[None]
    m = torch.ones(nq, nk, dtype=torch.bool)
    if left >= 0:
        m &= key >= place - left
    if right >= 0:
        m &= key <= place + right
    return m.to(on.device) & on[None]


def attention(q, k, v, case, on=None, lse=None, out=None, dout=None):
    """The forward (out, lse, and |P| |v| for the bound), or with lse, out and
    dout the gradients, each with the bound of its elements' error."""
    u, tiny = UNIT[q.dtype], TINY[q.dtype]
    scale, group = case["scale"], q.shape[1] // k.shape[1]
    z = lambda like: torch.zeros(like.shape, dtype=torch.float64, device=q.device)
    o, L, ob = z(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device), z(q)
    dq, dk, dv, bq, bk, bv = z(q), z(k), z(k), z(q), z(k), z(k)
    for q0, q1, k0, k1 in segments(case):
        if q1 == q0:
            continue
        flags = torch.ones(k1 - k0, dtype=torch.bool, device=q.device) if on is None else on[k0:k1] != 0
        m = seen(q1 - q0, k1 - k0, case["left"], case["right"], flags)
        some = m.any(1)
        for h in range(q.shape[1]):
            a, b, c = (t.double() for t in (q[q0:q1, h], k[k0:k1, h // group], v[k0:k1, h // group]))
            # what no row or key admits reaches nothing, whatever it holds
            a = torch.where(some[:, None], a, 0.0)
            b, c = torch.where(flags[:, None], b, 0.0), torch.where(flags[:, None], c, 0.0)
            s = torch.where(m, a @ b.T * scale, torch.full((), -math.inf, dtype=torch.float64, device=q.device))
            if lse is None:
                top = torch.where(some, s.amax(1) if k1 > k0 else torch.zeros_like(s.sum(1)), 0.0)[:, None]
                e = torch.exp(s - top)
                t = e.sum(1, keepdim=True)
                p = e / torch.where(t > 0, t, 1.0)
                o[q0:q1, h] = p @ c
                L[q0:q1, h] = torch.where(some, (top + torch.log(t))[:, 0], -math.inf)
                # one rounding of each probability (against the running maximum, at most 1), one of the result,
                # fp32 sums and exponentials
                ob[q0:q1, h] = (u + 2e-5) * (p @ c.abs()) + u * (p @ c).abs() + 2 * tiny * (1 + m.double() @ c.abs())
                continue
            p = torch.where(m, torch.exp(s - torch.where(some, lse[q0:q1, h].double(), 0.0)[:, None]), 0.0)
            d = torch.where(some[:, None], dout[q0:q1, h].double(), 0.0)
            delta = (d * torch.where(some[:, None], out[q0:q1, h].double(), 0.0)).sum(1, keepdim=True)
            dp = d @ c.T
            ds = p * (dp - delta)
            dq[q0:q1, h] = scale * (ds @ b)
            dk[k0:k1, h // group] += scale * (ds.T @ a)
            dv[k0:k1, h // group] += p.T @ d
            # one rounding of p and of ds, one of the result; ds itself from fp32 sums of |d||c| and |d||out| terms
            sd = p * (d.abs() @ c.abs().T + (d.abs() * out[q0:q1, h].double().abs().nan_to_num()).sum(1, keepdim=True))
            es = u * ds.abs() + 2e-5 * sd + tiny * m
            bq[q0:q1, h] = scale * (es @ b.abs()) + u * dq[q0:q1, h].abs() + tiny
            bk[k0:k1, h // group] += scale * (es.T @ a.abs())
            bv[k0:k1, h // group] += ((u + 2e-5) * p + tiny * m).T @ d.abs()
    if lse is None:
        return o, L, ob
    bk, bv = bk + u * dk.abs() + tiny, bv + u * dv.abs() + tiny
    return (dq, dk, dv), (bq, bk, bv)
