"""The region refiner: the token operators together with a training view."""
import numpy as np
import pytest
import torch

import token_refs as ref

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
    return tr, cam, RegionRefiner(tr, region=257, seed=3)


def plain(net, ids):
    """The network in double, with plain operators and torch's own autograd."""
    w = {k: v.detach().double().requires_grad_() for k, v in net.w.items()}
    rows = net.base[ids].double()
    norm = lambda x, g: x * g / torch.sqrt(x.pow(2).mean(1, keepdim=True) + net.eps)
    H, G, D = net.heads, net.kv_heads, net.dim
    x = (rows - net.shift) / net.spread @ w["inp"]
    qkv = (norm(x, w["norm1"]) @ w["qkv"]).view(-1, H + 2 * G, D)
    pairs = sum(net.axis_pairs)
    axis = torch.arange(3, device=ids.device).repeat_interleave(net.axis_pairs[0])
    t = (rows[:, :3] * net.place)[:, axis] * net.freq.double()
    c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
    turn = lambda z: torch.cat((z[..., :pairs] * c - z[..., pairs:2 * pairs] * s,
                                z[..., :pairs] * s + z[..., pairs:2 * pairs] * c, z[..., 2 * pairs:]), -1)
    q, k, v = turn(qkv[:, :H]), turn(qkv[:, H:H + G]), qkv[:, H + G:]
    same = (ids // net.region)[:, None] == (ids // net.region)[None]
    o = []
    for h in range(H):
        z = q[:, h] @ k[:, h // (H // G)].T * D ** -0.5
        o.append(torch.softmax(z.masked_fill(~same, -torch.inf), 1) @ v[:, h // (H // G)])
    x = x + torch.stack(o, 1).reshape(-1, net.width) @ w["out"]
    x = x + torch.nn.functional.silu(norm(x, w["norm2"]) @ w["up"]) @ w["down"]
    return (norm(x, w["norm3"]) @ w["head"]) * (net.gain * net.spread), w


def test_network_and_its_gradient(made):
    tr, cam, net = made
    ids = net.visible_ids(cam)
    assert 0 < ids.numel() <= tr.n
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    d = torch.randn(ids.numel(), tr.row_len, generator=g, device="cuda") / net.spread
    got = net.corrections(ids)
    want, w = plain(net, ids)
    want.backward(d.double())
    got.backward(d)
    # some twenty roundings to bfloat16 on the way, each of 2^-8 at most, none of them amplified much
    room = 20 * ref.UNIT[torch.bfloat16]
    assert float((got.detach().double() - want.detach()).norm() / want.detach().norm()) < room
    for k, v in net.w.items():
        assert float((v.grad.double() - w[k].grad).norm() / w[k].grad.norm()) < room, k
        v.grad = None


def test_training_lowers_the_loss_and_leaves_the_pool(made):
    tr, cam, net = made
    before = [p.clone() for p in tr.params]
    losses = [float(net.step(cam)) for _ in range(25)]
    assert losses[-1] < 0.9 * losses[0], losses
    assert all(torch.equal(a, b) for a, b in zip(before, tr.params))
    assert tr.host_status()[0] == 0


def test_published_tokens(made):
    tr, cam, net = made
    net.step(cam)
    dev = tr.dev
    status = torch.zeros(4, dtype=torch.int32, device=dev)
    versions = torch.zeros(tr.n, dtype=torch.int32, device=dev)
    table, replica, msg = net.replica_table(), net.replica_table(), net.message()
    r = net.publish(7, table, msg, status)
    net.commit(msg, replica, versions, status)
    torch.cuda.synchronize()
    ids, total = net.last
    assert int(status[0]) == 0
    want = np.zeros(tr.n, np.int32)
    want[ids.cpu().numpy()] = 7
    assert np.array_equal(versions.cpu().numpy(), want)
    got = net.read_tokens(replica, ids)
    assert torch.equal(got, r.q.float() * r.scale.repeat_interleave(128, 1)[:, :net.width])
    y, _ = ref.norm(total, net.w["norm3"].detach(), net.eps)
    # three bits behind the leading one: a 16th of an element, and steps of 2^-9 of the scale near zero
    assert bool(((got.double() - y).abs() <= y.abs() / 15 + r.scale.double() * 2.0 ** -9).all())
    others = torch.ones(tr.n, dtype=torch.bool, device=dev)
    others[ids] = False
    assert bool((replica[others] == 0).all())
