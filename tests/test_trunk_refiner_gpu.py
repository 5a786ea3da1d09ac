"""The region refiner's recurrence trunk: the lookups, layer norms, recurrences and kept activations together with a
training view."""
import numpy as np
import pytest
import torch

import token_refs
import trunk_refs as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def made():
    from paper_2607_19893_amd import scenes
    from paper_2607_19893_amd.pipeline import ViewTrainer
    from paper_2607_19893_amd.refiner import RegionRefiner
    w = scenes.spatially_ordered(scenes.tiny(n=3000))
    cam = w.cameras[0]
    tr = ViewTrainer(w.scene, capacity=1 << 17, max_width=cam.width, max_height=cam.height)
    tr.ensure_capacity([cam], margin=4.0)
    tr.set_target(w.target(0))
    return tr, cam, RegionRefiner(tr, region=1100, seed=3, trunk="recurrence", cells=6)


class KeptProduct(torch.autograd.Function):
    """silu(u) * v @ down in double, with the gradients at u and v as 8 bits hold them."""

    @staticmethod
    def forward(ctx, u, v, down):
        (a, b), (c, d) = ref.eight(u), ref.eight(v)
        ctx.save_for_backward(ref.wide(a, b), ref.wide(c, d), down)
        return (torch.nn.functional.silu(u) * v) @ down

    @staticmethod
    def backward(ctx, dout):
        u, v, down = ctx.saved_tensors
        (du, dv, h), _ = ref.silu_bwd(dout @ down.T, u, v)
        return du, dv, h.T @ dout


def scan(x, gate, starts, reverse):
    """The recurrence in double under torch's autograd, token by token."""
    out = []
    a = torch.sigmoid(gate)
    order = list(range(x.shape[0]))
    heads = {s for s, e in zip(starts, starts[1:]) if e > s} if not reverse else {e - 1 for s, e in zip(starts, starts[1:]) if e > s}
    h = None
    for t in reversed(order) if reverse else order:
        h = (1 - a[t]) * x[t] if t in heads else a[t] * h + (1 - a[t]) * x[t]
        out.append(h)
    return torch.stack(out[::-1] if reverse else out)


def plain(net, ids):
    """The network in double, with plain operators and torch's own autograd."""
    ref.UNIT[torch.float64] = ref.TINY[torch.float64] = 0.0
    w = {k: v.detach().double().cpu().requires_grad_() for k, v in net.w.items()}
    table = net.table.detach().double().cpu().requires_grad_()
    rows = net.base[ids].double().cpu()
    norm = lambda x, g, b: torch.nn.functional.layer_norm(x, x.shape[1:], g, b, net.eps)
    x = (rows - net.shift.cpu()) / net.spread.cpu() @ w["inp"] + table[net.cell_ids(net.base[ids]).long().cpu()]
    mix = (norm(x, w["norm1"], w["bias1"]) @ w["mix"]).view(-1, 4, net.width)
    starts = torch.searchsorted(ids, net.starts).tolist()
    along = scan(mix[:, 0], mix[:, 1] + net.hold, starts, False)
    against = scan(mix[:, 2], mix[:, 3] + net.hold, starts, True)
    x = x + torch.cat((along, against), 1) @ w["out"]
    both = norm(x, w["norm2"], w["bias2"]) @ w["up"]
    hidden = both.shape[1] // 2
    x = x + KeptProduct.apply(both[:, :hidden], both[:, hidden:], w["down"])
    y = x * w["norm3"] / torch.sqrt(x.pow(2).mean(1, keepdim=True) + net.eps)
    return (y @ w["head"]) * (net.gain * net.spread.cpu()), w, table


def test_network_and_its_gradient(made):
    tr, cam, net = made
    ids = net.visible_ids(cam)
    assert 0 < ids.numel() <= tr.n
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    d = torch.randn(ids.numel(), tr.row_len, generator=g, device="cuda") / net.spread
    got = net.corrections(ids)
    want, w, table = plain(net, ids)
    want.backward(d.double().cpu())
    got.backward(d)
    # some twenty roundings to bfloat16 on the way, each of 2^-8 at most, none of them amplified much
    room = 20 * token_refs.UNIT[torch.bfloat16]
    assert float((got.detach().double().cpu() - want.detach()).norm() / want.detach().norm()) < room
    # a value near the border of two 8-bit numbers may be kept as the other one: a step of 2^-3 for one in 2^-8 / 2^-3
    # of them, 2^-3 2^-2.5 of a gradient's norm at most
    flips = 2.0 ** -5.5
    for k, v in net.w.items():
        assert float((v.grad.double().cpu() - w[k].grad).norm() / w[k].grad.norm()) < room + flips, k
        v.grad = None
    assert float((net.table.grad.double().cpu() - table.grad).norm() / table.grad.norm()) < room + flips
    unused = torch.ones(net.table.shape[0], dtype=torch.bool, device="cuda")
    unused[net.cell_ids(net.base[ids]).long()] = False
    assert bool((net.table.grad[unused] == 0).all())
    net.table.grad = None


def test_a_step_trains_every_weight_and_leaves_the_pool(made):
    tr, cam, net = made
    before = [p.clone() for p in tr.params]
    weights = {k: v.detach().clone() for k, v in net.w.items()}
    table = net.table.detach().clone()
    losses = [float(net.step(cam)) for _ in range(3)]
    assert all(np.isfinite(losses))
    assert all(torch.equal(a, b) for a, b in zip(before, tr.params))
    assert tr.host_status()[0] == 0
    for k, v in net.w.items():
        assert bool(torch.isfinite(v).all()) and not torch.equal(v.detach(), weights[k]), k
    assert not torch.equal(net.table.detach(), table)


def test_published_tokens(made):
    tr, cam, net = made
    net.step(cam)
    status = torch.zeros(4, dtype=torch.int32, device=tr.dev)
    versions = torch.zeros(tr.n, dtype=torch.int32, device=tr.dev)
    table, replica, msg = net.replica_table(), net.replica_table(), net.message()
    r = net.publish(7, table, msg, status)
    net.commit(msg, replica, versions, status)
    torch.cuda.synchronize()
    ids, _ = net.last
    assert int(status[0]) == 0 and bool((versions[ids] == 7).all()) and int((versions == 7).sum()) == ids.numel()
    assert torch.equal(net.read_tokens(replica, ids), r.q.float() * r.scale.repeat_interleave(128, 1)[:, :net.width])


def test_the_trunks_are_told_apart(made):
    from paper_2607_19893_amd.refiner import RegionRefiner
    with pytest.raises(ValueError, match="trunk"):
        RegionRefiner(made[0], trunk="convolution")
