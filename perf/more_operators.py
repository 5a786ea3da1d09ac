"""The operators of a trunk whose cost is linear in the tokens, as cases that can be timed and compared: the layer norm
with the residual's addition (forward, backward), the embedding's lookup and its gradient, the gated linear recurrence
over ragged segments (forward, backward) and the gated SiLU whose inputs are kept in 8 bits (forward, backward).

A case is a dict of plain values.  prepare() makes what a program holds before the call, run() is one pass: elementary
torch operations in 32 bits (sums over tokens in 64) where `own` is false, the package's entry points where it is true.
exact() gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5
KEPT = 64          # tokens between the states that a recurrence leaves for its gradient
BLOCK = 32         # columns that share a scale byte of the kept values
TOP = 448.0        # largest e4m3 value


def listed():
    return [
        # the tokens of a view's few regions between two layers: the call itself is the time
        dict(name="layer-few-tokens", kind="layer", rows=5, cols=768, type="f16", residual=True),
        # a large view's tokens, with a width that fills no whole 16-byte piece
        dict(name="layer-odd-width", kind="layer", rows=60_001, cols=1001, type="bf16", residual=True),
        # the training pass, fp32 tokens as the pool's rows are
        dict(name="layer-backward", kind="layer_bwd", rows=24_000, cols=768, type="f32", residual=True),
        # every primitive of a large view looks up the vector of its cell; a few cells hold most of them
        dict(name="cells-lookup", kind="embed", tokens=400_000, rows=32_768, dim=256, skew=2.0, table="f32",
             type="bf16"),
        # the way back: thousands of tokens sum into one cell's row, others have one or none
        dict(name="cells-gradient", kind="embed_grad", tokens=300_001, rows=20_000, dim=256, skew=4.0, touched=False,
             type="bf16"),
        # a large table of which a view touches a part: the rows that the sparse optimizer steps
        dict(name="cells-gradient-touched", kind="embed_grad", tokens=120_000, rows=2_000_000, dim=64, skew=1.0,
             touched=True, type="f32"),
        # one new token of many sequences, the state read and written: the call itself is most of the time
        dict(name="recur-step", kind="recur", least=1, most=1, segments=160, spread=1, cols=2048, reverse=False,
             initial=True, keep=False, type="bf16"),
        # the regions of a scene against their order, fp32
        dict(name="recur-regions-back", kind="recur", least=40, most=1600, segments=40, spread=2, cols=512,
             reverse=True, initial=False, keep=False, type="f32"),
        # one long ordered run of tokens in training
        dict(name="recur-long", kind="recur", least=131_072, most=131_072, segments=1, spread=3, cols=1024,
             reverse=False, initial=False, keep=True, type="bf16"),
        # its gradient, ragged, with states
        dict(name="recur-backward", kind="recur_bwd", least=3, most=60_000, segments=9, spread=4, cols=768,
             reverse=False, initial=True, type="bf16"),
        # the MLP's activation of a large view in training
        dict(name="gate-keep", kind="gate", rows=40_000, cols=2048, gated=True, type="bf16"),
        # and its gradient from what was kept, with the product's operand again
        dict(name="gate-backward", kind="gate_bwd", rows=40_000, cols=2048, gated=True, again=True, type="bf16"),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["layer", "layer_bwd", "embed", "embed_grad", "embed_grad", "recur", "recur", "recur_bwd",
                       "recur_bwd", "gate", "gate_bwd"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("layer", "layer_bwd"):
        cols = rng.choice([8 * _between(rng, 1, 300), _between(rng, 8, 2400)])
        return dict(kind=kind, rows=_between(rng, 1, max(2, min(100_000, 60_000_000 // cols))), cols=cols, type=t,
                    residual=rng.random() < 0.7)
    if kind in ("embed", "embed_grad"):
        dim = rng.choice([8 * _between(rng, 1, 128), _between(rng, 1, 1000)])
        c = dict(kind=kind, tokens=_between(rng, 1, min(400_000, 80_000_000 // dim)),
                 rows=_between(rng, 1, min(2_000_000, 120_000_000 // dim)), dim=dim, skew=rng.choice([1.0, 2.0, 4.0]),
                 type=t)
        if kind == "embed":
            c["table"] = rng.choice(["f32", t])
        else:
            c["touched"] = rng.random() < 0.5
        return c
    if kind in ("recur", "recur_bwd"):
        cols = rng.choice([64 * _between(rng, 1, 32), _between(rng, 1, 2000)])
        segments = _between(rng, 1, 300)
        most = max(1, min(100_000, 60_000_000 // (cols * segments)))
        most = _between(rng, 1, max(2, most))
        c = dict(kind=kind, least=max(1, most // rng.choice([1, 5, 100])), most=most, segments=segments,
                 spread=rng.randint(0, 1 << 20), cols=cols, reverse=rng.random() < 0.4, initial=rng.random() < 0.5,
                 type=t)
        if kind == "recur":
            c["keep"] = rng.random() < 0.5
        return c
    cols = rng.choice([32 * _between(rng, 1, 200), _between(rng, 1, 5000)])
    c = dict(kind=kind, rows=_between(rng, 1, max(2, min(100_000, 60_000_000 // cols))), cols=cols,
             gated=rng.random() < 0.7, type=t)
    if kind == "gate_bwd":
        c["again"] = rng.random() < 0.7
    return c


# -- inputs --------------------------------------------------------------------


def _lengths(case):
    """Segment lengths, spread over the case's range on a log scale, the first the longest."""
    lo, hi = case["least"], case["most"]
    if lo == hi:
        return [hi] * case["segments"]
    g = torch.Generator()
    g.manual_seed(case["spread"])
    u = torch.rand(case["segments"], generator=g).tolist()
    n = [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * t))) for t in u]
    return [hi] + n[1:]


def _starts(n):
    return torch.tensor([0] + n, dtype=torch.int64).cumsum(0).to(torch.int32).to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    t = TYPES[case["type"]]
    kind = case["kind"]

    def normal(*shape, dtype=t, scale=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device=DEV) * scale + mean).to(dtype)

    s = dict(case=case)
    if kind in ("layer", "layer_bwd"):
        rows, cols = case["rows"], case["cols"]
        # some channels are larger than the others and few have mean 0, as trained tokens have them
        spread = torch.exp(torch.randn(cols, generator=g, device=DEV) * 0.7)
        shift = torch.randn(cols, generator=g, device=DEV) * 0.5
        s["weight"] = 1.0 + 0.2 * torch.randn(cols, generator=g, device=DEV)
        s["bias"] = 0.1 * torch.randn(cols, generator=g, device=DEV)
        s["x"] = (normal(rows, cols, dtype=torch.float32) * spread + shift).to(t)
        if kind == "layer":
            s["residual"] = (normal(rows, cols, dtype=torch.float32) * spread).to(t) if case["residual"] else None
        else:
            s["dy"] = normal(rows, cols, scale=0.1)
            s["dtotal"] = normal(rows, cols, scale=0.1) if case["residual"] else None
        return s
    if kind in ("embed", "embed_grad"):
        n, rows, dim = case["tokens"], case["rows"], case["dim"]
        u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
        s["ids"] = (u.pow(case["skew"]) * rows).long().clamp_(max=rows - 1).to(torch.int32)
        s["scale"] = math.sqrt(dim)
        if kind == "embed":
            s["table"] = normal(rows, dim, dtype=TYPES[case["table"]], scale=1.0 / s["scale"])
        else:
            s["dout"] = normal(n, dim, scale=0.1)
            if case["touched"]:                # the optimizer's buffers
                most = min(n, rows)
                s["unique"] = torch.full((most,), -1, dtype=torch.int32, device=DEV)
                s["count"] = torch.zeros(1, dtype=torch.int32, device=DEV)
                s["grad"] = torch.zeros(most, dim, device=DEV)
        return s
    if kind in ("recur", "recur_bwd"):
        lengths = _lengths(case)
        n, cols, segments = sum(lengths), case["cols"], case["segments"]
        s["n"], s["longest"], s["cu"] = n, max(lengths), _starts(lengths)
        s["x"] = normal(n, cols)
        s["gate"] = normal(n, cols, scale=1.5, mean=1.5)           # most of the state is held for some tokens
        s["initial"] = normal(segments, cols, dtype=torch.float32) if case["initial"] else None
        if kind == "recur_bwd":
            s["dy"] = normal(n, cols, scale=0.1)
            s["dfinal"] = normal(segments, cols, dtype=torch.float32, scale=0.1) if case["initial"] else None
            # what the forward left: the states in front of every KEPT tokens
            s["kept"] = _plain_recur(dict(s, case=dict(case, keep=True)))["kept"]
        return s
    rows, cols = case["rows"], case["cols"]
    # columns of one projection
    both = normal(rows, cols * (2 if case["gated"] else 1))
    u, v = both[:, :cols], both[:, cols:] if case["gated"] else None
    if kind == "gate":
        s["u"], s["v"] = u, v
        return s
    s["dh"] = normal(rows, cols, scale=0.1)
    s["u8"], s["u_scale"] = _plain_eight(u)
    s["v8"], s["v_scale"] = _plain_eight(v) if case["gated"] else (None, None)
    return s


# -- plain forms ---------------------------------------------------------------


def _plain_layer(s):
    total = s["x"].float()
    if s["residual"] is not None:
        total = total + s["residual"].float()
    d = total - total.mean(1, keepdim=True)
    y = d * torch.rsqrt((d * d).mean(1, keepdim=True) + EPS) * s["weight"] + s["bias"]
    out = {"y": y.to(s["x"].dtype)}
    if s["residual"] is not None:
        out["total"] = total.to(s["x"].dtype)
    return out


def _plain_layer_bwd(s):
    x, dy = s["x"].float(), s["dy"].float()
    d = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    n = d * r
    gw = dy * s["weight"]
    dx = r * (gw - gw.mean(1, keepdim=True) - n * (gw * n).mean(1, keepdim=True))
    if s["dtotal"] is not None:
        dx = dx + s["dtotal"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * n).sum(0), "dbias": dy.sum(0)}


def _plain_embed(s):
    return {"out": (s["table"].float()[s["ids"].long()] * s["scale"]).to(TYPES[s["case"]["type"]])}


def _plain_embed_grad(s):
    """Tokens sorted by their row, running sums in 64 bits, and each row's share as the difference at its ends."""
    c = s["case"]
    ids, order = torch.sort(s["ids"].long(), stable=True)
    rows, counts = torch.unique_consecutive(ids, return_counts=True)
    upto = torch.cumsum(s["dout"][order].double().T.contiguous(), 1)[:, counts.cumsum(0) - 1]
    sums = ((upto - torch.cat((torch.zeros_like(upto[:, :1]), upto[:, :-1]), 1)) * s["scale"]).float().T
    if not c["touched"]:
        grad = torch.zeros(c["rows"], c["dim"], device=DEV)
        grad[rows] = sums
        return {"grad": grad}
    count = torch.zeros_like(s["count"]) + rows.numel()
    unique, grad = torch.full_like(s["unique"], -1), torch.zeros_like(s["grad"])
    unique[:rows.numel()] = rows.to(torch.int32)
    grad[:rows.numel()] = sums
    return {"unique": unique, "count": count, "grad": grad}


def _layout(s):
    """Tokens in the recurrence's order: each one's segment, and which are a segment's first; the ends of all."""
    c = s["case"]
    cu = s["cu"].long()
    n = s["n"]
    at = torch.arange(n, device=DEV)
    seg = torch.searchsorted(cu, at, right=True) - 1
    first, last = cu[seg] == at, cu[seg + 1] == at + 1
    if c["reverse"]:
        return seg.flip(0), last.flip(0), first.flip(0)
    return seg, first, last


def _turned(t, c):
    return t.flip(0) if c["reverse"] else t


def _scan(A, B, longest):
    """h_t = A_t h_(t-1) + B_t along the first dimension, where A is 0 at every start: joined over 1, 2, 4, ... tokens."""
    d = 1
    while d < longest:
        B = torch.cat((B[:d], B[d:] + A[d:] * B[:-d]))
        A = torch.cat((A[:d], A[d:] * A[:-d]))
        d *= 2
    return B


def _plain_recur(s):
    c = s["case"]
    seg, first, last = _layout(s)
    x, g = _turned(s["x"].float(), c), _turned(s["gate"].float(), c)
    a, z = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    b = z * x
    if s["initial"] is not None:
        b = torch.where(first[:, None], b + a * s["initial"][seg], b)
    h = _scan(torch.where(first[:, None], 0.0, a), b, s["longest"])
    out = {"y": _turned(h, c).to(s["x"].dtype), "final": torch.zeros(c["segments"], c["cols"], device=DEV)}
    out["final"][seg[last]] = h[last]
    if c["keep"]:
        before = torch.cat((torch.zeros_like(h[:1]), h[:-1]))[::KEPT]
        out["kept"] = torch.where(first[::KEPT, None], 0.0, before)
    return out


def _plain_recur_bwd(s):
    c = s["case"]
    seg, first, last = _layout(s)
    x, g, dy = (_turned(s[k].float(), c) for k in ("x", "gate", "dy"))
    a, z = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    b = z * x
    if s["initial"] is not None:
        b = torch.where(first[:, None], b + a * s["initial"][seg], b)
    h = _scan(torch.where(first[:, None], 0.0, a), b, s["longest"])
    before = torch.cat((torch.zeros_like(h[:1]), h[:-1]))
    start = s["initial"][seg] if s["initial"] is not None else torch.zeros_like(before)
    before = torch.where(first[:, None], start, before)
    if s["dfinal"] is not None:
        dy = torch.where(last[:, None], dy + s["dfinal"][seg], dy)
    # D_t = dy_t + a_(t+1) D_(t+1), from the other end
    after = torch.cat((a[1:], torch.zeros_like(a[:1])))
    D = _scan(torch.where(last[:, None], 0.0, after).flip(0), dy.flip(0), s["longest"]).flip(0)
    out = {"dx": _turned(D * z, c).to(s["x"].dtype),
           "dgate": _turned(D * (before - x) * a * z, c).to(s["x"].dtype)}
    if s["initial"] is not None:
        out["dinitial"] = torch.zeros(c["segments"], c["cols"], device=DEV)
        out["dinitial"][seg[first]] = (a * D)[first]
    return out


def _plain_eight(u):
    """(rows in 8 bits, scale bytes): a block's power of two is the least that brings its largest value to 448."""
    rows, cols = u.shape
    blocks = -(-cols // BLOCK)
    wide = torch.zeros(rows, blocks * BLOCK, device=DEV)
    wide[:, :cols] = u.float()
    wide = wide.view(rows, blocks, BLOCK)
    m, e = torch.frexp(wide.abs().amax(2))     # m in [1/2, 1): 448 is 7/8 2^9
    k = torch.where(m > 0.875, e - 8, e - 9)
    k = torch.where(m == 0, -127, k).clamp(min=-127)
    q = torch.ldexp(wide, -k[:, :, None]).view(rows, blocks * BLOCK)[:, :cols]
    return q.to(torch.float8_e4m3fn), (k + 127).to(torch.uint8)


def _plain_wide(q, scale):
    k = scale.int().repeat_interleave(BLOCK, 1)[:, :q.shape[1]] - 127
    return torch.ldexp(q.float(), k)


def _plain_gate(s):
    u = s["u"].float()
    h = u / (1 + torch.exp(-u))
    if s["v"] is not None:
        h = h * s["v"].float()
    out = {"h": h.to(s["u"].dtype)}
    out["u8"], out["u_scale"] = _plain_eight(s["u"])
    if s["v"] is not None:
        out["v8"], out["v_scale"] = _plain_eight(s["v"])
    return out


def _plain_gate_bwd(s):
    dh, u = s["dh"].float(), _plain_wide(s["u8"], s["u_scale"])
    p = 1 / (1 + torch.exp(-u))
    t = s["dh"].dtype
    d = p * (1 + u * (1 - p))
    if s["v8"] is None:
        out = {"du": (dh * d).to(t)}
        if s["case"]["again"]:
            out["h"] = (u * p).to(t)
        return out
    v = _plain_wide(s["v8"], s["v_scale"])
    out = {"du": (dh * v * d).to(t), "dv": (dh * u * p).to(t)}
    if s["case"]["again"]:
        out["h"] = (u * p * v).to(t)
    return out


# -- one pass ------------------------------------------------------------------


def _own(s):
    from paper_2607_19893_amd import tokens

    c = s["case"]
    kind = c["kind"]
    if kind == "layer":
        r = tokens.layer_norm(s["x"], s["weight"], s["bias"], EPS, residual=s["residual"])
        return {"y": r.y, "total": r.total} if s["residual"] is not None else {"y": r.y}
    if kind == "layer_bwd":
        dx, dw, db = tokens.layer_norm_backward(s["dy"], s["x"], s["weight"], EPS, dtotal=s["dtotal"])
        return {"dx": dx, "dweight": dw, "dbias": db}
    if kind == "embed":
        return {"out": tokens.embedding(s["table"], s["ids"], scale=s["scale"], dtype=TYPES[c["type"]])}
    if kind == "embed_grad":
        if c["touched"]:
            unique, count, grad = tokens.embedding_rows(s["dout"], s["ids"], c["rows"], scale=s["scale"],
                                                        out=(s["unique"], s["count"], s["grad"]))
            return {"unique": unique, "count": count, "grad": grad}
        return {"grad": tokens.embedding_backward(s["dout"], s["ids"], c["rows"], scale=s["scale"])}
    if kind == "recur":
        r = tokens.recurrence(s["x"], s["gate"], cu=s["cu"], initial=s["initial"], reverse=c["reverse"],
                              keep=c["keep"])
        return {"y": r.y, "final": r.final, "kept": r.kept} if c["keep"] else {"y": r.y, "final": r.final}
    if kind == "recur_bwd":
        dx, dgate, dinitial = tokens.recurrence_backward(s["dy"], s["x"], s["gate"], s["kept"], cu=s["cu"],
                                                         initial=s["initial"], dfinal=s["dfinal"],
                                                         reverse=c["reverse"])
        out = {"dx": dx, "dgate": dgate}
        return dict(out, dinitial=dinitial) if s["initial"] is not None else out
    if kind == "gate":
        r = tokens.gated_silu(s["u"], s["v"])
        out = {"h": r.h, "u8": r.u8, "u_scale": r.u_scale}
        return dict(out, v8=r.v8, v_scale=r.v_scale) if c["gated"] else out
    du, dv, h = tokens.gated_silu_backward(s["dh"], s["u8"], s["u_scale"], s["v8"], s["v_scale"], again=c["again"])
    out = {"du": du}
    if c["gated"]:
        out["dv"] = dv
    return dict(out, h=h) if c["again"] else out


def run(state):
    if own:
        return _own(state)
    return {"layer": _plain_layer, "layer_bwd": _plain_layer_bwd, "embed": _plain_embed,
            "embed_grad": _plain_embed_grad, "recur": _plain_recur, "recur_bwd": _plain_recur_bwd,
            "gate": _plain_gate, "gate_bwd": _plain_gate_bwd}[state["case"]["kind"]](state)


# -- what a pass cannot do without ----------------------------------------------


def _touched(case):
    """Rows of the table that the tokens are expected to reach."""
    edge = torch.arange(case["rows"] + 1, dtype=torch.float64) / case["rows"]
    p = edge.pow(1.0 / case["skew"]).diff()
    return float((1 - torch.exp(case["tokens"] * torch.log1p(-p.clamp(max=1 - 1e-12)))).sum())


def work(case):
    e = BYTES[case["type"]]
    kind = case["kind"]
    if kind == "layer":
        n = case["rows"] * case["cols"]
        return {"bytes": n * e * (4 if case["residual"] else 2) + 8 * case["cols"], "flops": 8.0 * n}
    if kind == "layer_bwd":
        n = case["rows"] * case["cols"]
        return {"bytes": n * e * (4 if case["residual"] else 3) + 12 * case["cols"], "flops": 14.0 * n}
    if kind == "embed":
        n = case["tokens"] * case["dim"]
        return {"bytes": n * e + 4 * case["tokens"] + _touched(case) * case["dim"] * BYTES[case["table"]],
                "flops": 1.0 * n}
    if kind == "embed_grad":
        n = case["tokens"] * case["dim"]
        out = _touched(case) * (4 * case["dim"] + 4) if case["touched"] else 4 * case["rows"] * case["dim"]
        return {"bytes": n * e + 4 * case["tokens"] + out, "flops": 1.0 * n}
    if kind in ("recur", "recur_bwd"):
        tokens = sum(_lengths(case))
        n, states = tokens * case["cols"], 4 * case["segments"] * case["cols"]
        kept = 4 * -(-tokens // KEPT) * case["cols"]
        if kind == "recur":
            return {"bytes": 3 * n * e + states * (2 if case["initial"] else 1) + (kept if case["keep"] else 0),
                    "flops": 8.0 * n}
        return {"bytes": 5 * n * e + states * (3 if case["initial"] else 0) + kept, "flops": 18.0 * n}
    n = case["rows"] * case["cols"]
    parts = 2 if case["gated"] else 1
    eight = parts * (n + case["rows"] * -(-case["cols"] // BLOCK))
    if kind == "gate":
        return {"bytes": (parts + 1) * n * e + eight, "flops": 8.0 * n}
    return {"bytes": (1 + parts + (1 if case["again"] else 0)) * n * e + eight, "flops": 12.0 * n}


# -- the definitions in 64 bits ----------------------------------------------------


def _exact_layer(s):
    total = s["x"].double()
    if s["residual"] is not None:
        total = total + s["residual"].double()
    var, mean = torch.var_mean(total, 1, correction=0, keepdim=True)
    y = (total - mean) / torch.sqrt(var + EPS) * s["weight"].double() + s["bias"].double()
    return {"y": y, "total": total} if s["residual"] is not None else {"y": y}


def _exact_layer_bwd(s):
    x, dy, w = s["x"].double(), s["dy"].double(), s["weight"].double()
    cols = x.shape[1]
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    rms = torch.sqrt(var + EPS)
    g = dy * w
    dx = g / rms - g.sum(1, keepdim=True) / (cols * rms)
    dx -= (x - mean) * (g * (x - mean)).sum(1, keepdim=True) / (cols * rms ** 3)
    if s["dtotal"] is not None:
        dx += s["dtotal"].double()
    return {"dx": dx, "dweight": (dy * (x - mean) / rms).sum(0), "dbias": dy.sum(0)}


def _exact_embed(s):
    return {"out": torch.index_select(s["table"], 0, s["ids"].long()).double() * s["scale"]}


def _exact_embed_grad(s):
    """Rows of few tokens one place of theirs at a time, the others row by row."""
    c = s["case"]
    ids = s["ids"].long()
    order = torch.sort(ids, stable=True).indices
    rows, counts = torch.unique_consecutive(ids[order], return_counts=True)
    ends = counts.cumsum(0)
    sums = torch.zeros(rows.numel(), c["dim"], dtype=torch.float64, device=DEV)
    small = counts <= 64
    for j in range(int(counts[small].max()) if bool(small.any()) else 0):
        at = torch.nonzero(small & (counts > j)).squeeze(1)
        sums[at] += s["dout"][order[(ends - counts)[at] + j]].double()
    for i in torch.nonzero(~small).squeeze(1).tolist():
        sums[i] = s["dout"][order[int(ends[i] - counts[i]):int(ends[i])]].double().sum(0)
    sums *= s["scale"]
    if not c["touched"]:
        grad = torch.zeros(c["rows"], c["dim"], dtype=torch.float64, device=DEV)
        grad[rows] = sums
        return {"grad": grad}
    grad = torch.zeros(s["grad"].shape, dtype=torch.float64, device=DEV)
    grad[:rows.numel()] = sums
    return {"unique": None, "count": None, "grad": grad}


def _exact_states(a, b, reset):
    """h_t = a_t h_(t-1) + b_t (b_t alone where reset): runs of tokens side by side, one token at a time, then run by run."""
    n, cols = a.shape
    per = max(1, int(math.sqrt(n)))
    runs = -(-n // per)
    more = runs * per - n
    a = torch.cat((a.masked_fill(reset[:, None], 0.0), a.new_zeros(more, cols))).view(runs, per, cols)
    b = torch.cat((b, b.new_zeros(more, cols))).view(runs, per, cols).clone()
    held = a.clone()
    for i in range(1, per):
        b[:, i] += a[:, i] * b[:, i - 1]
        held[:, i] *= held[:, i - 1]
    carry = torch.zeros_like(b[0, 0])
    for r in range(runs):
        b[r] += held[r] * carry
        carry = b[r, -1]
    return b.view(runs * per, cols)[:n]


def _exact_recur(s):
    c = s["case"]
    n, cols = s["n"], c["cols"]
    cu = s["cu"].tolist()
    order = torch.arange(n, device=DEV)
    if c["reverse"]:
        order = order.flip(0)
        heads, tails = [cu[i + 1] - 1 for i in range(len(cu) - 1)], cu[:-1]
    else:
        heads, tails = cu[:-1], [cu[i + 1] - 1 for i in range(len(cu) - 1)]
    place = torch.empty(n, dtype=torch.int64, device=DEV)
    place[order] = torch.arange(n, device=DEV)
    heads, tails = place[torch.tensor(heads, device=DEV)], place[torch.tensor(tails, device=DEV)]
    g, x = s["gate"].double()[order], s["x"].double()[order]
    a, z = torch.sigmoid(g), torch.sigmoid(-g)
    del g
    reset = torch.zeros(n, dtype=torch.bool, device=DEV)
    reset[heads] = True
    h0 = s["initial"].double() if s["initial"] is not None else torch.zeros(c["segments"], cols, dtype=torch.float64,
                                                                            device=DEV)
    b = z * x
    b[heads] += a[heads] * h0
    h = _exact_states(a, b, reset)
    if c["kind"] == "recur":
        out = {"y": h[place], "final": h[tails]}
        if c["keep"]:
            kept = torch.zeros(-(-n // KEPT), cols, dtype=torch.float64, device=DEV)
            for i in range(1, kept.shape[0]):
                if not bool(reset[i * KEPT]):
                    kept[i] = h[i * KEPT - 1]
            out["kept"] = kept
        return out
    before = torch.roll(h, 1, 0)
    before[heads] = h0
    del h, b
    dy = s["dy"].double()[order]
    if s["dfinal"] is not None:
        dy[tails] += s["dfinal"].double()
    ends = torch.zeros(n, dtype=torch.bool, device=DEV)
    ends[tails] = True
    D = _exact_states(torch.roll(a, -1, 0).flip(0), dy.flip(0), ends.flip(0)).flip(0)
    out = {"dx": (z * D)[place], "dgate": (a * z * (before - x) * D)[place]}
    return dict(out, dinitial=(a * D)[heads]) if s["initial"] is not None else out


def _exact_eight(u):
    """e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6, ties to the even step."""
    parts = []
    for block in u.double().split(BLOCK, 1):
        top = block.abs().amax(1, keepdim=True)
        k = torch.ceil(torch.log2(top / TOP)).clamp(min=-127)
        k = torch.where(torch.exp2(k - 1) * TOP >= top, k - 1, k).clamp(min=-127)      # the logarithm's own rounding
        k = torch.where(torch.exp2(k) * TOP < top, k + 1, k)
        v = block / torch.exp2(k)
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        parts.append(torch.round(v / step) * step)
    return torch.cat(parts, 1)


def _exact_gate(s):
    u = s["u"].double()
    h = u * torch.sigmoid(u)
    out = {"u8": _exact_eight(s["u"]), "u_scale": None}
    if s["v"] is not None:
        h = h * s["v"].double()
        out.update(v8=_exact_eight(s["v"]), v_scale=None)
    return dict(out, h=h)


def _exact_gate_bwd(s):
    c = s["case"]

    def wide(q, scale):
        return q.double() * torch.exp2(scale.double() - 127).repeat_interleave(BLOCK, 1)[:, :q.shape[1]]

    u, dh = wide(s["u8"], s["u_scale"]), s["dh"].double()
    v = wide(s["v8"], s["v_scale"]) if c["gated"] else torch.ones_like(u)
    p, m = torch.sigmoid(u), torch.sigmoid(-u)
    out = {"du": dh * v * (p + u * p * m)}
    if c["gated"]:
        out["dv"] = dh * u * p
    return dict(out, h=u * p * v) if c["again"] else out


def exact(case, seed):
    s = prepare(case, seed)
    return {"layer": _exact_layer, "layer_bwd": _exact_layer_bwd, "embed": _exact_embed,
            "embed_grad": _exact_embed_grad, "recur": _exact_recur, "recur_bwd": _exact_recur,
            "gate": _exact_gate, "gate_bwd": _exact_gate_bwd}[case["kind"]](s)
