"""The token operators as cases that can be timed and compared: the norm with
the residual's addition (forward, into 8 bits, backward), the rotation by
position, and attention over ragged segments (forward, few rows over many
keys, backward).

A case is a dict of plain values.  prepare() makes what a program holds before
the call, run() is one pass: elementary torch operations in 32 bits where
`own` is false, the package's entry points where it is true.  exact() gives the
same outputs from the definitions in 64 bits, one segment and head at a time.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6
BLOCK = 128        # columns that share a scale of the 8-bit output
TOP = 448.0        # largest e4m3 value


def listed():
    return [
        # the tokens of one view's few regions between two layers: the call itself is the time
        dict(name="norm-few-tokens", kind="norm", rows=7, cols=1024, type="bf16", residual=True, bits=16),
        # a partition's tokens as they are published to a replica: rows in 8 bits with their scales
        dict(name="norm-publish-8bit", kind="norm", rows=50_001, cols=1536, type="bf16", residual=True, bits=8),
        # the training pass through the same norm, fp32 tokens and weights as the pool's rows have
        dict(name="norm-backward-f32", kind="norm_bwd", rows=20_000, cols=768, type="f32", residual=True),
        # and in 16 bits, with a width that is no power of two
        dict(name="norm-backward-bf16", kind="norm_bwd", rows=60_000, cols=1160, type="bf16", residual=True),
        # primitives rotated by their place in the scene: three axes, three quarters of each head
        dict(name="rotary-places", kind="rotary", tokens=50_000, heads=8, kv_heads=8, dim=64, rot=48, axes=3,
             interleaved=False, inverse=False, reach=300.0, type="f32"),
        # the gradient's rotation back, a long sequence, key heads shared
        dict(name="rotary-long-back", kind="rotary", tokens=32_768, heads=32, kv_heads=8, dim=128, rot=128, axes=1,
             interleaved=True, inverse=True, reach=131072.0, type="bf16"),
        # one new token over everything that was seen
        dict(name="attend-one-token", kind="attend", q_least=1, q_most=1, k_least=32_768, k_most=32_768,
             segments=1, spread=1, heads=32, kv_heads=8, dim=128, left=-1, right=-1, masked=0.0, type="bf16"),
        # a few view tokens read the tokens of their region, some of them switched off, one region all
        dict(name="attend-views-regions", kind="attend", q_least=1, q_most=16, k_least=900, k_most=9000,
             segments=24, spread=2, heads=16, kv_heads=16, dim=64, left=-1, right=-1, masked=0.2, type="bf16"),
        # the regions of a scene, each attending to itself
        dict(name="attend-regions", kind="attend", q_least=40, q_most=1600, segments=40, spread=3, heads=8, kv_heads=8,
             dim=64, left=-1, right=-1, masked=0.0, type="f16"),
        # one long ordered run of tokens, each sees what is before it
        dict(name="attend-long-ordered", kind="attend", q_least=8192, q_most=8192, segments=1, spread=4, heads=16,
             kv_heads=4, dim=128, left=-1, right=0, masked=0.0, type="bf16"),
        # the training pass through small regions
        dict(name="attend-backward-regions", kind="attend_bwd", q_least=3, q_most=1500, segments=24, spread=5, heads=8,
             kv_heads=8, dim=64, left=-1, right=-1, masked=0.1, type="bf16"),
        # and through the long run
        dict(name="attend-backward-long", kind="attend_bwd", q_least=8192, q_most=8192, segments=1, spread=6, heads=16,
             kv_heads=4, dim=128, left=-1, right=0, masked=0.0, type="bf16"),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "rotary", "attend", "attend", "attend_bwd", "attend_bwd"])
    if kind in ("norm", "norm_bwd"):
        cols = 8 * _between(rng, 8, 300)
        rows = _between(rng, 1, max(2, min(100_000, 70_000_000 // cols)))
        c = dict(kind=kind, rows=rows, cols=cols, type=rng.choice(["bf16", "f16", "f32"]), residual=rng.random() < 0.7)
        if kind == "norm":
            c["bits"] = rng.choice([16, 16, 8])
        return c
    if kind == "rotary":
        dim = rng.choice([32, 64, 80, 128])
        axes = rng.choice([1, 3])
        rot = rng.choice([dim, dim // 2]) // (2 * axes) * (2 * axes)
        kv = rng.choice([1, 2, 4, 8])
        kind_type = rng.choice(["bf16", "f16", "f32"])
        reach = float(_between(rng, 10, 300 if kind_type == "f32" else 30_000))
        return dict(kind=kind, tokens=_between(rng, 1, 40_000), heads=kv * rng.choice([1, 2, 4]), kv_heads=kv, dim=dim,
                    rot=rot, axes=axes, interleaved=rng.random() < 0.5, inverse=rng.random() < 0.5, reach=reach,
                    type=kind_type)
    segments = _between(rng, 1, 40)
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4])
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128])
    most = int(math.sqrt(8192 * 8192 * 16 * 128 / 4 / (segments * heads * dim)))     # a quarter of the long run's work
    top = _between(rng, 16, max(17, min(8192, most)))
    c = dict(kind=kind, q_least=max(1, top // rng.choice([1, 4, 40])), q_most=top, segments=segments,
             spread=rng.randint(0, 1 << 20), heads=heads, kv_heads=kv, dim=dim, left=-1, right=-1,
             masked=rng.choice([0.0, 0.0, 0.3]), type=rng.choice(["bf16", "bf16", "f16"]))
    form = rng.choice(["self", "ordered", "window", "few"] if kind == "attend" else ["self", "ordered", "window"])
    if form == "ordered":
        c["right"] = 0
    if form == "window":
        c["left"], c["right"] = _between(rng, 4, 1000), rng.choice([0, 0, 50])
    if form == "few":
        c["q_least"], c["q_most"] = 1, rng.randint(1, 16)
        c["k_least"], c["k_most"] = max(1, top // 4), min(20_000, 4 * top)
    return c


# -- inputs --------------------------------------------------------------------


def _lengths(case):
    """Segment lengths (queries, keys): spread over the case's range on a log scale, the first the longest."""
    g = torch.Generator()
    g.manual_seed(case["spread"])

    def some(lo, hi):
        if lo == hi:
            return [hi] * case["segments"]
        u = torch.rand(case["segments"], generator=g).tolist()
        n = [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * t))) for t in u]
        n[0] = hi
        return n

    nq = some(case["q_least"], case["q_most"])
    return nq, (some(case["k_least"], case["k_most"]) if "k_most" in case else list(nq))      # else each to itself


def _starts(n):
    t = torch.tensor([0] + n, dtype=torch.int64).cumsum(0)
    return t.to(torch.int32).to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    t = TYPES[case["type"]]

    def normal(*shape, dtype=t, scale=1.0):
        return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)

    s = dict(case=case)
    if case["kind"] in ("norm", "norm_bwd"):
        rows, cols = case["rows"], case["cols"]
        # some channels are much larger than the others, as trained tokens have them
        spread = torch.exp(torch.randn(cols, generator=g, device=DEV) * 0.7)
        s["weight"] = 1.0 + 0.2 * torch.randn(cols, generator=g, device=DEV)
        s["x"] = (normal(rows, cols, dtype=torch.float32) * spread).to(t)
        if case["kind"] == "norm":
            s["residual"] = (normal(rows, cols, dtype=torch.float32) * spread).to(t) if case["residual"] else None
        else:
            s["dy"] = normal(rows, cols, scale=0.1)
            s["dtotal"] = normal(rows, cols, scale=0.1) if case["residual"] else None
        return s
    if case["kind"] == "rotary":
        n, axes, pairs = case["tokens"], case["axes"], case["rot"] // 2
        per = pairs // axes
        s["q"], s["k"] = normal(n, case["heads"], case["dim"]), normal(n, case["kv_heads"], case["dim"])
        if axes == 1:
            s["pos"] = torch.randint(0, int(case["reach"]), (n, 1), generator=g, device=DEV).float()
        else:
            s["pos"] = (torch.rand(n, axes, generator=g, device=DEV) - 0.5) * case["reach"]
        f = torch.arange(per, dtype=torch.float64) / per
        s["freq"] = (10000.0 ** -f).repeat(axes).float().to(DEV)
        s["per_axis"] = [per] * axes
        return s
    nq, nk = _lengths(case)
    s["longest"] = (max(nq), max(nk))
    s["cu_q"], s["cu_k"] = _starts(nq), _starts(nk)
    Q, K = sum(nq), sum(nk)
    s["q"] = normal(Q, case["heads"], case["dim"])
    s["k"], s["v"] = normal(K, case["kv_heads"], case["dim"]), normal(K, case["kv_heads"], case["dim"])
    s["key_on"] = None
    if case["masked"]:
        on = torch.rand(K, generator=g, device=DEV) >= case["masked"]
        if len(nk) > 1:                       # the last region's tokens are all off
            on[K - nk[-1]:] = False
        s["key_on"] = on.to(torch.uint8)
    s["scale"] = 1.0 / math.sqrt(case["dim"])
    if case["kind"] == "attend_bwd":
        s["dout"] = normal(Q, case["heads"], case["dim"])
        # what the forward left: its result and the rows' log sums
        st = dict(s, case=dict(case, kind="attend"))
        s["out"], s["lse"] = _plain_attend(st)
        del st
    return s


# -- plain forms ---------------------------------------------------------------


def _plain_norm(s):
    c = s["case"]
    total = s["x"].float()
    if s["residual"] is not None:
        total = total + s["residual"].float()
    y = total * torch.rsqrt((total * total).mean(1, keepdim=True) + EPS) * s["weight"]
    out = {}
    if s["residual"] is not None:
        out["total"] = total.to(s["x"].dtype)
    if c["bits"] == 8:
        rows, cols = y.shape
        blocks = -(-cols // BLOCK)
        wide = torch.zeros(rows, blocks * BLOCK, device=DEV)
        wide[:, :cols] = y
        wide = wide.view(rows, blocks, BLOCK)
        top = wide.abs().amax(2)
        scale = torch.where(top > 0, top / TOP, torch.ones_like(top))
        q = (wide / scale[:, :, None]).clamp(-TOP, TOP).view(rows, blocks * BLOCK)[:, :cols]
        out["q"], out["scale"] = q.to(torch.float8_e4m3fn), scale
    else:
        out["y"] = y.to(s["x"].dtype)
    return out


def _plain_norm_bwd(s):
    x, dy = s["x"].float(), s["dy"].float()
    r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    n = x * r
    gw = dy * s["weight"]
    dx = r * (gw - n * (gw * n).mean(1, keepdim=True))
    if s["dtotal"] is not None:
        dx = dx + s["dtotal"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * n).sum(0)}


def _plain_turn(x, angle, interleaved):
    pairs = angle.shape[1]
    f = x.float()
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    part = f[..., :2 * pairs]
    if interleaved:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = part[..., :pairs], part[..., pairs:]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, f[..., 2 * pairs:]), -1).to(x.dtype)


def _plain_rotary(s):
    c = s["case"]
    axis = torch.arange(c["axes"], device=DEV).repeat_interleave(s["per_axis"][0])
    angle = s["pos"][:, axis] * s["freq"]
    if c["inverse"]:
        angle = -angle
    return {"q": _plain_turn(s["q"], angle, c["interleaved"]), "k": _plain_turn(s["k"], angle, c["interleaved"])}


def _padded(cu, longest):
    """[segments, longest] row ids of a padded layout and which of them are there."""
    at = torch.arange(longest, device=DEV)
    there = at < (cu[1:] - cu[:-1])[:, None]
    return torch.where(there, cu[:-1, None] + at, 0).long(), there


def _scores(s):
    """Padded fp32 operands, scores with -inf at what is not admitted, and the layout."""
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    iq, onq = _padded(s["cu_q"], s["longest"][0])
    ik, onk = _padded(s["cu_k"], s["longest"][1])
    q = s["q"].float()[iq].transpose(1, 2).contiguous()                                   # [S, H, Lq, D]
    k = s["k"].float()[ik].transpose(1, 2).repeat_interleave(group, 1).contiguous()
    v = s["v"].float()[ik].transpose(1, 2).repeat_interleave(group, 1).contiguous()
    # keys by their distance from the query, the last query on the last key
    nq, nk = s["cu_q"][1:] - s["cu_q"][:-1], s["cu_k"][1:] - s["cu_k"][:-1]
    rows = torch.arange(iq.shape[1], device=DEV)[None, :, None] + (nk - nq)[:, None, None]
    ahead = torch.arange(ik.shape[1], device=DEV)[None, None, :] - rows
    seen = onk[:, None, :] & onq[:, :, None]
    if s["key_on"] is not None:
        seen = seen & (s["key_on"][ik] != 0)[:, None, :]
    if c["left"] >= 0:
        seen = seen & (ahead >= -c["left"])
    if c["right"] >= 0:
        seen = seen & (ahead <= c["right"])
    z = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    z = torch.where(seen[:, None], z, torch.full_like(z, -math.inf))
    return q, k, v, z, (iq, onq, ik, onk)


def _plain_attend(s):
    q, k, v, z, (iq, onq, ik, onk) = _scores(s)
    top = z.amax(3, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total)).squeeze(3)
    out = torch.empty_like(s["q"])
    rows = iq[onq]
    out[rows] = o.transpose(1, 2)[onq].to(s["q"].dtype)
    lses = torch.empty(s["q"].shape[:2], device=DEV)
    lses[rows] = lse.transpose(1, 2)[onq]
    return out, lses


def _plain_attend_bwd(s):
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    q, k, v, z, (iq, onq, ik, onk) = _scores(s)
    keep = onq[:, None, :, None]
    lse = s["lse"][iq].transpose(1, 2)[..., None]
    p = torch.where(z == -math.inf, torch.zeros_like(z), torch.exp(z - lse))
    del z
    do = torch.where(keep, s["dout"].float()[iq].transpose(1, 2), 0.0).contiguous()
    delta = (do * s["out"].float()[iq].transpose(1, 2)).sum(3, keepdim=True)
    ds = p * (torch.matmul(do, v.transpose(2, 3).contiguous()) - delta) * s["scale"]
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    outs = []
    for t, like, i, on, shared in ((dq, s["q"], iq, onq, 1), (dk, s["k"], ik, onk, group),
                                   (dv, s["v"], ik, onk, group)):
        t = t.view(t.shape[0], t.shape[1] // shared, shared, *t.shape[2:]).sum(2).transpose(1, 2)
        flat = torch.empty_like(like)
        flat[i[on]] = t[on].to(like.dtype)
        outs.append(flat)
    return {"dq": outs[0], "dk": outs[1], "dv": outs[2]}


# -- one pass ------------------------------------------------------------------


def _own(s):
    from paper_2607_19893_amd import tokens

    c = s["case"]
    if c["kind"] == "norm":
        r = tokens.rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], eight_bit=c["bits"] == 8)
        out = {"total": r.total} if s["residual"] is not None else {}
        if c["bits"] == 8:
            return dict(out, q=r.q, scale=r.scale)
        return dict(out, y=r.y)
    if c["kind"] == "norm_bwd":
        dx, dw = tokens.rms_norm_backward(s["dy"], s["x"], s["weight"], EPS, dtotal=s["dtotal"])
        return {"dx": dx, "dweight": dw}
    if c["kind"] == "rotary":
        q, k = tokens.rotary((s["q"], s["k"]), s["pos"], s["freq"], s["per_axis"], interleaved=c["interleaved"],
                             inverse=c["inverse"])
        return {"q": q, "k": k}
    how = dict(cu_q=s["cu_q"], cu_k=s["cu_k"], key_on=s["key_on"], scale=s["scale"], left=c["left"], right=c["right"])
    if c["kind"] == "attend":
        out, lse = tokens.attention(s["q"], s["k"], s["v"], **how)
        return {"out": out, "lse": lse}
    dq, dk, dv = tokens.attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], **how)
    return {"dq": dq, "dk": dk, "dv": dv}


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "attend":
        out, lse = _plain_attend(state)
        return {"out": out, "lse": lse}
    return {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "rotary": _plain_rotary,
            "attend_bwd": _plain_attend_bwd}[kind](state)


# -- what a pass cannot do without ----------------------------------------------


def _admitted(case, nq, nk):
    """(query, key) pairs inside the windows, summed over the segments, less the share that is switched off."""
    pairs = 0
    for a, b in zip(nq, nk):
        if case["left"] < 0 and case["right"] < 0:
            pairs += a * b
            continue
        i = torch.arange(a, dtype=torch.int64) + b - a
        hi = torch.clamp(i + case["right"], max=b - 1) if case["right"] >= 0 else torch.full_like(i, b - 1)
        lo = torch.clamp(i - case["left"], min=0) if case["left"] >= 0 else torch.zeros_like(i)
        pairs += int(torch.clamp(hi - lo + 1, min=0).sum())
    return pairs * (1.0 - case["masked"])


def work(case):
    e = BYTES[case["type"]]
    if case["kind"] == "norm":
        n = case["rows"] * case["cols"]
        out = n * (1 + 4 / BLOCK) if case["bits"] == 8 else n * e
        return {"bytes": n * e * (3 if case["residual"] else 1) + out + 4 * case["cols"], "flops": 5.0 * n}
    if case["kind"] == "norm_bwd":
        n = case["rows"] * case["cols"]
        return {"bytes": n * e * (4 if case["residual"] else 3) + 8 * case["cols"], "flops": 10.0 * n}
    if case["kind"] == "rotary":
        n = case["tokens"] * (case["heads"] + case["kv_heads"])
        return {"bytes": 2 * n * case["dim"] * e + 4 * case["tokens"] * case["axes"], "flops": 3.0 * n * case["rot"]}
    nq, nk = _lengths(case)
    rows, keys = sum(nq) * case["heads"], sum(nk) * case["kv_heads"]
    pairs = _admitted(case, nq, nk) * case["heads"]
    if case["kind"] == "attend":
        return {"bytes": (2 * rows + 2 * keys) * case["dim"] * e + 4 * rows, "flops": 4.0 * pairs * case["dim"]}
    return {"bytes": (4 * rows + 4 * keys) * case["dim"] * e + 4 * rows, "flops": 10.0 * pairs * case["dim"]}


# -- the definitions in 64 bits ----------------------------------------------------


def _exact_norm(s):
    c = s["case"]
    total = s["x"].double()
    if s["residual"] is not None:
        total = total + s["residual"].double()
    y = s["weight"].double() * total / torch.sqrt(total.pow(2).sum(1, keepdim=True) / c["cols"] + EPS)
    out = {"total": total} if s["residual"] is not None else {}
    if c["bits"] != 8:
        return dict(out, y=y)
    scale = torch.stack([b.abs().max(1).values / TOP for b in y.split(BLOCK, 1)], 1)
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    v = y / scale[:, torch.arange(c["cols"], device=DEV) // BLOCK]
    # e4m3: three bits behind the leading one, steps of 2^-9 below 2^-6, ties to the even step
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return dict(out, q=torch.round(v / step) * step, scale=scale)


def _exact_norm_bwd(s):
    x, dy, w = s["x"].double(), s["dy"].double(), s["weight"].double()
    d = x.shape[1]
    rms = torch.sqrt(x.pow(2).sum(1, keepdim=True) / d + EPS)
    dx = dy * w / rms - x * (dy * w * x).sum(1, keepdim=True) / (d * rms ** 3)
    if s["dtotal"] is not None:
        dx = dx + s["dtotal"].double()
    return {"dx": dx, "dweight": (dy * x / rms).sum(0)}


def _exact_rotary(s):
    c = s["case"]
    pairs = c["rot"] // 2
    got = {}
    for name in ("q", "k"):
        x = s[name].double()
        y = x.clone()
        for j in range(pairs):
            t = s["pos"][:, j // s["per_axis"][0]].double() * s["freq"][j].double() * (-1 if c["inverse"] else 1)
            i, k = (2 * j, 2 * j + 1) if c["interleaved"] else (j, j + pairs)
            turn = torch.polar(torch.ones_like(t), t)[:, None] * torch.complex(x[..., i], x[..., k])
            y[..., i], y[..., k] = turn.real, turn.imag
        got[name] = y
    return got


def _exact_attend(s):
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    backward = c["kind"] == "attend_bwd"
    shape = tuple(s["q"].shape)
    out, dq, lse, dk, dv = (torch.zeros(n, dtype=torch.float64, device=DEV)
                            for n in (shape, shape, shape[:2], s["k"].shape, s["k"].shape))
    cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
    for n in range(c["segments"]):
        q0, q1, k0, k1 = cq[n], cq[n + 1], ck[n], ck[n + 1]
        place = torch.arange(q1 - q0, device=DEV)[:, None] + (k1 - k0) - (q1 - q0)
        key = torch.arange(k1 - k0, device=DEV)[None]
        off = torch.zeros(q1 - q0, k1 - k0, dtype=torch.bool, device=DEV)
        if c["left"] >= 0:
            off |= key < place - c["left"]
        if c["right"] >= 0:
            off |= key > place + c["right"]
        if s["key_on"] is not None:
            off |= s["key_on"][None, k0:k1] == 0
        for h in range(c["heads"]):
            q, k, v = s["q"][q0:q1, h].double(), s["k"][k0:k1, h // group].double(), s["v"][k0:k1, h // group].double()
            z = (q @ k.T * s["scale"]).masked_fill_(off, -math.inf)
            if not backward:
                total = torch.logsumexp(z, 1)
                lse[q0:q1, h] = total
                out[q0:q1, h] = torch.nan_to_num(torch.exp(z - total[:, None]), nan=0.0) @ v
                continue
            p = torch.nan_to_num(torch.exp(z - s["lse"][q0:q1, h, None].double()), nan=0.0)
            do = s["dout"][q0:q1, h].double()
            dz = p * (do @ v.T - (do * s["out"][q0:q1, h].double()).sum(1, keepdim=True)) * s["scale"]
            dq[q0:q1, h] = dz @ k
            dk[k0:k1, h // group] += dz.T @ q
            dv[k0:k1, h // group] += p.T @ do
    return {"dq": dq, "dk": dk, "dv": dv} if backward else {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_bwd": _exact_norm_bwd, "rotary": _exact_rotary, "attend": _exact_attend,
            "attend_bwd": _exact_attend}[case["kind"]](s)
