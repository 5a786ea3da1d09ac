"""The trunk's operators as programs run them: under autograd together, in captured graphs, on streams of their own,
with the framework's optimizer, and on lists past 2^31 elements."""
import math

import pytest
import torch

import trunk_refs as ref
from test_tokens_gpu import BF, F32, HF, gen, gs, randn, tk, within  # noqa: F401 (gs, tk: fixtures)
from test_trunk_gpu import starts

pytestmark = pytest.mark.gpu


def block(tk, w, ids, cu, scale=1.5):
    """One block of the operators over tokens in fp32; w: the weights."""
    x = tk.Embedding.apply(w["table"], ids, scale, None)
    y, total = tk.LayerNorm.apply(x, w["place"], w["w1"], w["b1"], 1e-5)
    h, final = tk.Recurrence.apply(y, y @ w["gate"], w["first"], dict(cu=cu))
    z, total = tk.LayerNorm.apply(h, total, w["w2"], None, 1e-5)
    return tk.GatedProjection.apply(z @ w["up"], w["down"]) + tk.GatedSilu.apply(total, h), final


def weights(g, cols=40, tokens=230):
    return {k: v.requires_grad_() for k, v in dict(
        table=randn(g, 17, cols), place=randn(g, tokens, cols), w1=1 + 0.1 * randn(g, cols), b1=randn(g, cols),
        gate=randn(g, cols, cols) * cols ** -0.5, first=randn(g, 3, cols), w2=1 + 0.1 * randn(g, cols),
        up=randn(g, cols, 2 * 24) * cols ** -0.5, down=randn(g, 24, cols) * 24 ** -0.5).items()}


def plain_block(w, ids, cu, kept):
    """The same in double with torch's autograd; kept: the values that 8 bits hold, in place of u and v."""
    norm = lambda x, a, b: torch.nn.functional.layer_norm(x, x.shape[1:], a, b, 1e-5)
    x = 1.5 * w["table"][ids.long()] + w["place"]
    y = norm(x, w["w1"], w["b1"])
    a = torch.sigmoid(y @ w["gate"])
    out = []
    for s in range(len(cu) - 1):
        h = w["first"][s]
        for t in range(cu[s], cu[s + 1]):
            h = a[t] * h + (1 - a[t]) * y[t]
            out.append(h)
    h = torch.stack(out)
    final = torch.stack([out[e - 1] if e > b else w["first"][i] for i, (b, e) in enumerate(zip(cu, cu[1:]))])
    total = x + h
    z = norm(total, w["w2"], None)
    u, v = (z @ w["up"]).split(24, 1)
    return kept(u, v) @ w["down"] + kept(total, h), final


def test_a_block_under_autograd(tk):
    """The operators one after the other: their gradients reach every weight, through the last states too.

    The kept values are exact where the plain form's gradient is taken at them: its silu reads u and v through a
    function whose value is silu(u) * v and whose gradient is that at the kept values."""
    g = gen(1)
    w = weights(g)
    cu = [0, 100, 100, 230]
    ids = torch.randint(0, 17, (230,), generator=g, device="cuda").int()
    out, final = block(tk, w, ids, starts(cu))
    d, df = randn(g, *out.shape), randn(g, *final.shape)
    torch.autograd.backward((out, final), (d, df))

    class Kept(torch.autograd.Function):
        @staticmethod
        def forward(ctx, u, v):
            pairs = [ref.wide(*ref.eight(t.float())) for t in (u, v)]
            ctx.save_for_backward(*pairs)
            return torch.nn.functional.silu(u) * v

        @staticmethod
        def backward(ctx, dh):
            (du, dv, _), _ = ref.silu_bwd(dh, *ctx.saved_tensors)
            return du, dv

    ref.UNIT[torch.float64] = ref.TINY[torch.float64] = 0.0
    p = {k: v.detach().double().requires_grad_() for k, v in w.items()}
    want, wf = plain_block(p, ids, cu, Kept.apply)
    torch.autograd.backward((want, wf), (d.double(), df.double()))
    near = lambda a, b: float((a.double() - b).norm() / b.norm())
    assert near(out.detach(), want.detach()) < 1e-5 and near(final.detach(), wf.detach()) < 1e-5
    for k in w:
        # `down`'s gradient is formed with silu(u') v' of the kept values: a 16th of u and of v off at most
        limit = 2 * 2.0 ** -4 if k == "down" else 1e-3     # the rest: fp32, and a kept value in 10^4 on the other side
        assert near(w[k].grad, p[k].grad) < limit, (k, near(w[k].grad, p[k].grad))


def calls(tk, g, dtype=BF):
    """Every operator's calls on inputs of their own: name -> function of the same tensors each time."""
    n, cols = 700, 96
    x, r, dy, gate = (randn(g, n, cols, dtype=dtype) for _ in range(4))
    w, b = 1 + 0.1 * randn(g, cols), randn(g, cols)
    table, ids = randn(g, 300, cols), torch.randint(0, 300, (n,), generator=g, device="cuda").int()
    cu, first = starts([0, 250, 251, 251, 700]), randn(g, 4, cols)
    kept = tk.recurrence(x, gate, cu=cu, initial=first, keep=True).kept
    q = tk.gated_silu(x, r)
    return {
        "layer": lambda: tk.layer_norm(x, w, b, residual=r), "layer gradient": lambda: tk.layer_norm_backward(dy, x, w, dtotal=r),
        "lookup": lambda: (tk.embedding(table, ids, 2.0, dtype),), "lookup gradient": lambda: (tk.embedding_backward(dy, ids, 300, 2.0),),
        "touched rows": lambda: [t[:int(300)] for t in tk.embedding_rows(dy, ids, 300, 2.0, out=(
            torch.full((300,), -1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"),
            torch.zeros(300, cols, device="cuda")))],
        "recurrence": lambda: tk.recurrence(x, gate, cu=cu, initial=first, keep=True),
        "recurrence gradient": lambda: tk.recurrence_backward(dy, x, gate, kept, cu=cu, initial=first, dfinal=first),
        "gate": lambda: [t.view(torch.uint8) if t.element_size() == 1 else t for t in tk.gated_silu(x, r)],
        "gate gradient": lambda: tk.gated_silu_backward(dy, q.u8, q.u_scale, q.v8, q.v_scale)}, (x, r, dy, gate, table, first)


def same(a, b):
    return all(torch.equal(s, t) for s, t in zip(a, b))


def test_captured_graphs_with_new_inputs_in_place(tk):
    """All operators in two graphs of one pool, whose workspaces lie in the same memory, replayed in turn with eager
    work between; every replay gives what the eager call gives."""
    g = gen(2)
    made, tensors = calls(tk, g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for f in made.values():
            f()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    pool = torch.cuda.graph_pool_handle()
    for names in (list(made)[:5], list(made)[5:]):
        graph, out = torch.cuda.CUDAGraph(), {}
        with torch.cuda.graph(graph, pool=pool):
            for k in names:
                out[k] = list(made[k]())
        graphs.append(graph)
        outs.append(out)
    for turn in range(4):
        for t in tensors:
            t.copy_(randn(g, *t.shape, dtype=t.dtype))
        for graph, out in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            copies = {k: [t.clone() for t in v if t is not None] for k, v in out.items()}
            for k, v in copies.items():
                eager = [t for t in made[k]() if t is not None]
                assert same(v, eager), (turn, k)


def test_streams_of_their_own(tk):
    """Two streams at once, each with its tensors; the results are those of one after the other."""
    pairs = [calls(tk, gen(s), dtype) for s, dtype in ((3, BF), (4, HF))]
    want = [{k: list(f()) for k, f in made.items()} for made, _ in pairs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    got = [{}, {}]
    for _ in range(3):
        for i, (made, _) in enumerate(pairs):
            with torch.cuda.stream(streams[i]):
                for k, f in made.items():
                    got[i][k] = list(f())
        torch.cuda.synchronize()
        for i in range(2):
            for k in want[i]:
                assert same([t for t in got[i][k] if t is not None], [t for t in want[i][k] if t is not None]), k


def test_touched_rows_are_what_the_sparse_optimizer_steps(tk, gs):
    """A table of 64 columns trained by gs_sparse_adam on the rows that embedding_rows gives."""
    g = gen(5)
    table = randn(g, 500, 64)
    ids = torch.randint(0, 500, (300,), generator=g, device="cuda").int()
    dout = randn(g, 300, 64)
    unique, count, grad = tk.embedding_rows(dout, ids, 500)
    m, v = torch.zeros(500, 64, device="cuda"), torch.zeros(500, 64, device="cuda")
    before = table.clone()
    gs.gs_sparse_adam(gs.make_adam_groups([(table, 0.1)]), 1, unique, count, unique.numel(), grad, 64, m, v, 64, 1, 0.9, 0.999,
                      1e-8)
    dense = tk.embedding_backward(dout, ids, 500)
    touched = torch.zeros(500, dtype=torch.bool, device="cuda")
    touched[ids.long()] = True
    assert int(count) == int(touched.sum()) and torch.equal(table[~touched], before[~touched])
    # the first step of Adam: lr * g / (|g| + eps), in fp32
    want = before.double() - 0.1 * dense.double() / (dense.double().abs() + 1e-8)
    within(table[touched], want[touched], 1e-5 * (1 + want[touched].abs()), "table")


def test_served_states_in_place(tk, gs):
    """The states' buffer is read and written by the same call, for steps, short runs and runs over many chunks."""
    g = gen(6)
    for lengths, cols in (([1] * 300, 130), ([1] * 90, 64), ([700, 0, 3, 500], 129), ([40, 0, 7], 66), ([300] * 9, 257)):
        n = sum(lengths)
        cu = starts([0] + torch.tensor(lengths).cumsum(0).tolist())
        state = randn(g, len(lengths), cols)
        for turn in range(3):
            x, gate = randn(g, n, cols, dtype=BF), randn(g, n, cols, dtype=BF)
            for reverse in (False, True):
                want = tk.recurrence(x, gate, cu=cu, initial=state, reverse=reverse)
                r = gs.make_recur(x, gate, cu, initial=state, reverse=reverse)
                y = torch.empty_like(x)
                ws = torch.empty(max(1, gs.gs_recurrence_ws_bytes(r)), dtype=torch.uint8, device="cuda")
                gs.gs_recurrence(r, y, final=state, ws=ws)
                assert torch.equal(y, want.y) and torch.equal(state, want.final), (lengths[:3], turn, reverse)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_recurrence_gives_the_same_bits(tk, dtype):
    """Whichever chunk's state is known first when another looks back: fp32 states and gradients, call after call, also
    beside work on another stream that delays some of the workgroups."""
    g = gen(16)
    n, cols = 40_000, 300
    x, gate, dy = (randn(g, n, cols, dtype=dtype) for _ in range(3))
    gate = (gate.float() + 3).to(dtype)                # states that reach over chunks
    first = randn(g, 2, cols)
    cu = starts([0, 7, n])
    want = tk.recurrence(x, gate, cu=cu, initial=first, keep=True)
    grads = tk.recurrence_backward(dy, x, gate, want.kept, cu=cu, initial=first, dfinal=first)
    other, big = torch.cuda.Stream(), randn(g, 4096, 4096)
    for turn in range(30):
        if turn % 3:
            with torch.cuda.stream(other):
                big.mul_(1.0)
        got = tk.recurrence(x, gate, cu=cu, initial=first, keep=True)
        assert same(got, want), turn
        assert same(tk.recurrence_backward(dy, x, gate, want.kept, cu=cu, initial=first, dfinal=first), grads), turn
    torch.cuda.synchronize()


def test_recurrence_past_two_to_the_31_elements(tk):
    """2,100,000 tokens of 1040 channels: the ends of the list are what they are alone."""
    n, cols, part = 2_100_000, 1040, 4096
    g = gen(7)
    x = torch.empty(n, cols, dtype=BF, device="cuda").normal_(generator=g)
    gate = torch.empty(n, cols, dtype=BF, device="cuda").normal_(generator=g)
    cu = starts([0, 1000, n - part, n])
    for reverse in (False, True):
        r = tk.recurrence(x, gate, cu=cu, reverse=reverse, keep=True)
        tail = tk.recurrence(x[n - part:], gate[n - part:], reverse=reverse)
        # the same tokens in chunks that start elsewhere: each within its bound of the exact state
        d = (r.y[n - part:].float() - tail.y.float()).abs()
        assert float((d - 2 * ref.UNIT[BF] * tail.y.float().abs()).max()) <= 1e-4
        assert float((r.final[2] - tail.final[0]).abs().max()) <= 1e-4
        dx, dg, _ = tk.recurrence_backward(x, x, gate, r.kept, cu=cu, reverse=reverse)
        t = tk.recurrence(x[n - part:], gate[n - part:], reverse=reverse, keep=True)
        a, b, _ = tk.recurrence_backward(x[n - part:], x[n - part:], gate[n - part:], t.kept, reverse=reverse)
        for got, want in ((dx[n - part:], a), (dg[n - part:], b)):
            d = (got.float() - want.float()).abs()
            assert float((d - 2 * ref.UNIT[BF] * want.float().abs()).max()) <= 1e-3
        del dx, dg, r


def test_lookup_and_gate_past_two_to_the_31_elements(tk):
    g = gen(8)
    rows, dim = 5_000_000, 1024                        # a table of 2^32 and more elements
    table = torch.empty(rows, dim, dtype=BF, device="cuda").normal_(generator=g)
    ids = torch.randint(rows - 1000, rows, (500,), generator=g, device="cuda").int()
    assert torch.equal(tk.embedding(table, ids), table[ids.long()])
    del table
    u, cols = 2_200_000, 1000
    x = torch.empty(u, cols, dtype=BF, device="cuda").normal_(generator=g)
    r = tk.gated_silu(x)
    few = tk.gated_silu(x[-300:].contiguous())
    assert torch.equal(r.h[-300:], few.h) and torch.equal(r.u8[-300:].view(torch.uint8), few.u8.view(torch.uint8))
    assert torch.equal(r.u_scale[-300:], few.u_scale)
    y = tk.layer_norm(x, torch.ones(cols, device="cuda"), None).y
    assert torch.equal(y[-300:], tk.layer_norm(x[-300:].contiguous(), torch.ones(cols, device="cuda"), None).y)
    grad = tk.embedding_backward(x, torch.full((u,), 3, dtype=torch.int32, device="cuda"), 5)
    want = x.double().sum(0) if u * cols < 1 << 33 else None
    # a sum of 2,200,000 numbers, the most of one chunk or group one after the other
    assert float((grad[3].double() - want).abs().max()) <= 3000 * ref.F * float(x.float().abs().sum(0).max())
    assert bool((grad[[0, 1, 2, 4]] == 0).all())


def test_layer_norm_gradient_past_two_to_the_31_elements(tk):
    g = gen(10)
    rows, cols = 2_200_000, 1000
    x = torch.empty(rows, cols, dtype=BF, device="cuda").normal_(generator=g)
    dy = torch.empty(rows, cols, dtype=BF, device="cuda").normal_(generator=g)
    w = randn(g, cols)
    dx, dw, db = tk.layer_norm_backward(dy, x, w, dtotal=x)
    assert torch.equal(dx[-300:], tk.layer_norm_backward(dy[-300:], x[-300:], w, dtotal=x[-300:])[0])
    want, size, wb, sb = (torch.zeros(cols, dtype=torch.float64, device="cuda") for _ in range(4))
    for a, b in zip(x.split(100_000), dy.split(100_000)):
        s, d = a.double(), b.double()
        n = (s - s.mean(1, keepdim=True)) / torch.sqrt(s.var(1, unbiased=False, keepdim=True) + 1e-5)
        want, size, wb, sb = want + (d * n).sum(0), size + (d * n).abs().sum(0), wb + d.sum(0), sb + d.abs().sum(0)
    # a workgroup's rows one after the other, then the partial rows; n's own roundings
    walk = (rows / 512 + 200) * ref.F
    assert bool(((dw.double() - want).abs() <= walk * size).all()) and bool(((db.double() - wb).abs() <= walk * sb).all())


def test_a_wait_that_nobody_ends_is_not_reached(tk):
    """Lists whose chunks outnumber what the card holds at once: every chunk finds its state."""
    g = gen(9)
    n, cols = 60_000, 8                                # hundreds of chunks of one block of channels
    x, gate = randn(g, n, cols), randn(g, n, cols) + 4
    r = tk.recurrence(x, gate)
    a = torch.sigmoid(gate.double())
    # a plain scan by doubling
    A, B, d = a.clone(), (1 - a) * x.double(), 1
    while d < n:
        B = torch.cat((B[:d], B[d:] + A[d:] * B[:-d]))
        A = torch.cat((A[:d], A[d:] * A[:-d]))
        d *= 2
    assert float((r.y.double() - B).abs().max()) <= 1e-4 and bool(torch.isfinite(r.y).all())
