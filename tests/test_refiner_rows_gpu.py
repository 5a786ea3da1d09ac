"""The region refiner and a pool that others write: rows as they are now, rows put back, tokens of one state."""
import pytest
import torch

import token_refs as ref

pytestmark = pytest.mark.gpu


@pytest.fixture
def made():
    from paper_2607_19893_amd import scenes
    from paper_2607_19893_amd.pipeline import ViewTrainer
    from paper_2607_19893_amd.refiner import RegionRefiner
    w = scenes.spatially_ordered(scenes.tiny(n=3000))
    cam = w.cameras[0]
    tr = ViewTrainer(w.scene, capacity=1 << 17, max_width=cam.width, max_height=cam.height)
    tr.ensure_capacity([cam], margin=4.0)
    tr.set_target(w.target(0))
    return tr, cam, RegionRefiner(tr, region=257, seed=3, lr=0.05)


def pool(tr):
    return [p.clone() for p in tr.params]


def test_a_step_keeps_what_others_wrote(made):
    tr, cam, net = made
    net.step(cam)
    for p in tr.params:
        p.mul_(1.001)
    now = pool(tr)
    net.step(cam)
    assert all(torch.equal(a, b) for a, b in zip(now, tr.params))


def test_corrections_follow_the_pool(made):
    tr, cam, net = made
    ids = net.visible_ids(cam)
    with torch.no_grad():
        first = net.corrections(ids)
        saved = pool(tr)
        for p in tr.params:
            p.mul_(1.1)
        assert not torch.equal(net.corrections(ids), first)
        for p, q in zip(tr.params, saved):
            p.copy_(q)
        assert torch.equal(net.corrections(ids), first)


@pytest.mark.parametrize("phase", ["bin_sort", "raster_bwd_pixels"])
def test_rows_are_put_back_when_a_phase_fails(made, phase, monkeypatch):
    tr, cam, net = made
    before = pool(tr)

    def fail(*a, **k):
        raise RuntimeError("no " + phase)

    monkeypatch.setattr(tr, phase, fail)
    with pytest.raises(RuntimeError, match="no " + phase):
        net.step(cam)
    assert all(torch.equal(a, b) for a, b in zip(before, tr.params))


def test_published_tokens_are_of_the_forward(made):
    tr, cam, net = made
    for _ in range(4):
        weight = net.w["norm3"].detach().clone()
        net.step(cam)
    assert float((net.w["norm3"].detach() - weight).abs().max()) > 0.01     # the step moved it
    status = torch.zeros(4, dtype=torch.int32, device=tr.dev)
    r = net.publish(1, net.replica_table(), net.message(), status)
    torch.cuda.synchronize()
    ids, total = net.last
    y, _ = ref.norm(total, weight, net.eps)
    got = r.q.double() * r.scale.double().repeat_interleave(128, 1)[:, :net.width]
    # e4m3: half a step of 2^-3 of an element, and half of 2^-9 of the scale near zero
    assert bool(((got - y).abs() <= y.abs() * (2.0 ** -4 + 1e-3) + r.scale.double() * 2.0 ** -10).all())
