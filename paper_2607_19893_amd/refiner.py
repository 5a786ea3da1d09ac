"""A network that refines the rows a view sees, trained through the view.

One token per visible primitive.  The pool's ids are cut into regions of
`region` consecutive primitives (a spatially ordered pool makes them compact);
a token attends to the tokens of its own region, turned by its primitive's
place in space.  With trunk="recurrence" the cost is linear in the tokens, and
regions may be as long as the pool: a token adds the vector of its cell in
space, two gated recurrences run along its region and against it, and the
activations are kept in 8 bits for the gradient.
The network writes a correction of every visible row; the view
is rendered with the corrected rows, and the gradient rows of its backward go
back through the network.  The tokens' last norm in 8 bits can be published to
a replica as any other rows are.

The lookups, norms, rotations, attention, recurrences and gates are the package's
token operators; the plain matrix products and the weights' Adam are torch's.

    python -m paper_2607_19893_amd.refiner [attention | recurrence]
"""
from __future__ import annotations

import sys

import torch

from . import gsmi, tokens
from .pipeline import ViewTrainer, to_u32

AXES = 3


class RegionRefiner:
    """Corrections for the rows of `trainer`'s pool, which itself stays as it is between steps."""

    def __init__(self, trainer: ViewTrainer, region=1024, width=128, heads=4, kv_heads=2, gain=1.0, lr=1e-3, seed=0,
                 trunk="attention", cells=16):
        if trunk not in ("attention", "recurrence"):
            raise ValueError("trunk is attention or recurrence, not %r" % (trunk,))
        if width % heads or width % 4 or heads % kv_heads or (width // heads) % 8:
            raise ValueError("width %d does not fit %d heads over %d" % (width, heads, kv_heads))
        self.tr, self.region, self.width, self.heads, self.kv_heads = trainer, int(region), width, heads, kv_heads
        self.dim = width // heads
        self.gain, self.eps, self.trunk, self.cells = gain, 1e-6, trunk, int(cells)
        dev = trainer.dev
        n = trainer.n
        base = self.base
        self.shift = base.mean(0)
        self.spread = base.std(0).clamp_min(1e-3)
        self.starts = torch.arange(0, n + self.region, self.region, device=dev).clamp_max(n)
        # a third of the pairs per axis, over distances from the pool's extent down to a thousandth of it
        per = self.dim // 2 // AXES
        freq, _ = gsmi.gs_rotary_freqs(per, base=1000.0)
        self.freq = torch.from_numpy(freq).to(dev).repeat(AXES)
        self.axis_pairs = (per,) * AXES
        extent = float((base[:, :3].amax(0) - base[:, :3].amin(0)).amax())
        self.place = 100.0 / max(extent, 1e-6)
        self.corner, self.cell = base[:, :3].amin(0), max(extent, 1e-6) / self.cells
        g = torch.Generator(device=dev)
        g.manual_seed(seed)

        def matrix(rows, cols, scale=1.0):
            return (torch.randn(rows, cols, generator=g, device=dev) * (scale * rows ** -0.5)).requires_grad_()

        row = trainer.row_len
        if trunk == "attention":
            self.w = dict(inp=matrix(row, width), qkv=matrix(width, (heads + 2 * kv_heads) * self.dim),
                          out=matrix(width, width), up=matrix(width, 4 * width), down=matrix(4 * width, width),
                          head=matrix(width, row, 0.1))
        else:
            # mix: a gate and a token for each of the two directions; up: the two sides of the gated activation
            self.w = dict(inp=matrix(row, width), mix=matrix(width, 4 * width), out=matrix(2 * width, width),
                          up=matrix(width, 8 * width), down=matrix(4 * width, width), head=matrix(width, row, 0.1))
            for k in ("bias1", "bias2"):
                self.w[k] = torch.zeros(width, device=dev, requires_grad=True)
            # `table` is looked up by row, no matrix product's operand
            self.table = (0.1 * torch.randn(self.cells ** 3, width, generator=g, device=dev)).requires_grad_()
            # gates that hold a state for some tokens at the start
            self.hold = 1.5
        for k in ("norm1", "norm2", "norm3"):
            self.w[k] = torch.ones(width, device=dev, requires_grad=True)
        self.opt = torch.optim.Adam(list(self.w.values()) + ([self.table] if trunk == "recurrence" else []), lr=lr)
        self.last = self.last_norm = None     # (ids, total) of the last forward and its last norm's weight, for publish()

    def rows(self, ids):
        """[len(ids), row_len] rows of the pool, as they are now."""
        return torch.cat([p[ids].reshape(-1, c) for p, c in zip(self.tr.params, self.tr.cols)], 1)

    @property
    def base(self):
        """All rows of the pool."""
        return self.rows(slice(None))

    def visible_ids(self, cam):
        """Ids the camera sees, ascending (synchronizes for their number)."""
        self.tr.project(cam)
        self.tr.visible()
        count = int(to_u32(self.tr.counts[0:1])[0])
        return self.tr.vis_idx[:count].long()

    def corrections(self, ids, rows=None):
        """[V, row_len] corrections of the rows `ids` (ascending), under autograd.  rows: those rows, if at hand."""
        bf = torch.bfloat16
        w = {k: v.to(bf) if v.dim() == 2 else v for k, v in self.w.items()}
        rows = self.rows(ids) if rows is None else rows
        cu = torch.searchsorted(ids, self.starts).int()
        pos = (rows[:, :AXES] * self.place).contiguous()
        x = ((rows - self.shift) / self.spread).to(bf) @ w["inp"]
        if self.trunk == "recurrence":
            h, total = self._recurrence(x, rows, w, cu)
            return self._head(h, total, ids, w)
        y, total = tokens.RmsNorm.apply(x, None, w["norm1"], self.eps)
        qkv = (y @ w["qkv"]).view(-1, self.heads + 2 * self.kv_heads, self.dim)
        q, k = tokens.Rotary.apply(qkv[:, :self.heads], qkv[:, self.heads:self.heads + self.kv_heads], pos, self.freq,
                                   self.axis_pairs, False, 1.0)
        o, _ = tokens.Attention.apply(q, k, qkv[:, self.heads + self.kv_heads:], dict(cu_q=cu, cu_k=cu))
        y, total = tokens.RmsNorm.apply(o.reshape(-1, self.width) @ w["out"], total, w["norm2"], self.eps)
        h = torch.nn.functional.silu(y @ w["up"]) @ w["down"]
        return self._head(h, total, ids, w)

    def _head(self, h, total, ids, w):
        y, last = tokens.RmsNorm.apply(h, total, w["norm3"], self.eps)
        self.last, self.last_norm = (ids, last.detach()), w["norm3"].detach().clone()
        return (y @ w["head"]).float() * (self.gain * self.spread)

    def cell_ids(self, rows):
        """The rows' cells in space, int32."""
        at = ((rows[:, :AXES] - self.corner) / self.cell).long().clamp(0, self.cells - 1)
        return ((at[:, 0] * self.cells + at[:, 1]) * self.cells + at[:, 2]).int()

    def _recurrence(self, x, rows, w, cu):
        """(the last block's output, the sum in front of it)."""
        where = tokens.Embedding.apply(self.table, self.cell_ids(rows), 1.0, x.dtype)
        y, total = tokens.LayerNorm.apply(x, where, w["norm1"], w["bias1"], self.eps)
        mix = (y @ w["mix"]).view(-1, 4, self.width)
        along, _ = tokens.Recurrence.apply(mix[:, 0], mix[:, 1] + self.hold, None, dict(cu=cu))
        against, _ = tokens.Recurrence.apply(mix[:, 2], mix[:, 3] + self.hold, None, dict(cu=cu, reverse=True))
        y, total = tokens.LayerNorm.apply(torch.cat((along, against), 1) @ w["out"], total, w["norm2"], w["bias2"], self.eps)
        return tokens.GatedProjection.apply(y @ w["up"], w["down"]), total

    def write_rows(self, ids, rows):
        """Rows of the pool's groups."""
        for p, part in zip(self.tr.params, rows.split(self.tr.cols, 1)):
            p[ids] = part.reshape(-1, *p.shape[1:])

    def step(self, cam, target=None):
        """One view: correct, render, back-propagate, update the weights.  Returns the view's loss (a device
        tensor).  target: 3*H*W floats on the device, or None for the trainer's target buffer."""
        tr = self.tr
        ids = self.visible_ids(cam)
        rows = self.rows(ids)
        delta = self.corrections(ids, rows)
        try:
            self.write_rows(ids, rows + delta.detach())
            seen = self.visible_ids(cam)                   # of the corrected rows: some of `ids`
            tr.bin_sort()
            tr.raster_fwd_l1(target)
            tr.raster_bwd_pixels()
            tr.raster_bwd_project()
        finally:
            self.write_rows(ids, rows)
        grad = torch.zeros_like(delta)
        grad[torch.searchsorted(ids, seen)] = tr.grad_rows[:seen.numel(), :tr.row_len]
        self.opt.zero_grad(set_to_none=True)
        delta.backward(grad)
        self.opt.step()
        return tr.loss.clone()

    # -- publication ------------------------------------------------------------

    def token_words(self):
        """fp32 words of a published token: its bytes, then its scales."""
        return self.width // 4, -(-self.width // gsmi.GS_NORM_BLOCK)

    def replica_table(self):
        return torch.zeros(self.tr.n, sum(self.token_words()), device=self.tr.dev)

    def _groups(self, table):
        a, b = self.token_words()
        return gsmi.make_groups([table[:, :a], table[:, a:a + b]])

    def publish(self, version, table, msg, status):
        """Stages the last step's tokens (their last norm with the weight of that forward, 8 bits) as a message:
        `table` [n, words] takes the rows by id, the message those of the ids."""
        ids, total = self.last
        r = tokens.rms_norm(total, self.last_norm, self.eps, eight_bit=True)
        table[ids] = torch.cat((r.q.view(torch.float32), r.scale), 1)
        count = torch.tensor([ids.numel()], dtype=torch.int32, device=table.device)
        gsmi.gs_delta_pack(ids.int(), count, self.tr.n, self._groups(table), 2, version, msg, status)
        return r

    def commit(self, msg, replica, versions, status):
        """Writes a message's tokens into a replica's table."""
        gsmi.gs_delta_apply(msg, self._groups(replica), 2, self.tr.n, self.tr.n, gsmi.GS_APPLY_OVERWRITE, versions,
                            status)

    def message(self):
        words = gsmi.gs_delta_msg_bytes(self.tr.n, sum(self.token_words()), 2)
        return torch.zeros((words + 15) // 16 * 4, dtype=torch.int32, device=self.tr.dev)

    def read_tokens(self, table, ids):
        """[V, width] fp32 tokens of a table's rows."""
        a, b = self.token_words()
        rows = table[ids]
        q = rows[:, :a].contiguous().view(torch.float8_e4m3fn).float()
        return q * rows[:, a:a + b].repeat_interleave(gsmi.GS_NORM_BLOCK, 1)[:, :self.width]


def main(steps=60, n=10_000, seed=0, trunk="attention"):
    from . import scenes

    w = scenes.spatially_ordered(scenes.tiny(seed=seed, n=n))
    cam = w.cameras[0]
    tr = ViewTrainer(w.scene, capacity=1 << 18, max_width=cam.width, max_height=cam.height)
    tr.ensure_capacity([cam], margin=4.0)
    tr.set_target(w.target(0))
    net = RegionRefiner(tr, seed=seed, trunk=trunk, region=1024 if trunk == "attention" else n)
    losses = [net.step(cam) for _ in range(steps)]
    status, versions = torch.zeros(4, dtype=torch.int32, device=tr.dev), torch.zeros(n, dtype=torch.int32, device=tr.dev)
    table, replica, msg = net.replica_table(), net.replica_table(), net.message()
    net.publish(1, table, msg, status)
    net.commit(msg, replica, versions, status)
    torch.cuda.synchronize()
    print("loss %.5f -> %.5f over %d steps; %d tokens published, status %d"
          % (float(losses[0]), float(losses[-1]), steps, int((versions == 1).sum()), int(status[0])))
    return [float(x) for x in losses]


if __name__ == "__main__":
    main(trunk=(sys.argv[1:] or ["attention"])[0])
