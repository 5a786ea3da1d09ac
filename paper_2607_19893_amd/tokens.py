"""Token operators for a network that writes rows of the pool: lookups of a
table's rows, the norms with the residual's addition, the rotation by position,
attention and the gated recurrence over ragged segments, and the gated SiLU whose
inputs are kept in 8 bits, each with its gradient.

The functions allocate their outputs and workspaces with torch on the current
stream of their tensors' GPU and call the gs_* entry points there; every step
runs in libgsmi's kernels.  `RmsNorm`, `LayerNorm`, `Embedding`, `Rotary`, `Attention`, `Recurrence`, `GatedSilu` and
`GatedProjection` put them under torch's autograd; their gradients have none of their own, a second derivative raises.
"""
from __future__ import annotations

import contextlib
from typing import NamedTuple, Optional

import torch
from torch.autograd.function import once_differentiable

from . import gsmi


_DENSE = torch.contiguous_format


class Normed(NamedTuple):
    """What rms_norm returns: y (None in 8 bits), the sum (x itself without a
    residual), and with eight_bit the rows as float8_e4m3fn and their scales
    [rows, ceil(cols / 128)]: y ~ q * scale."""
    y: Optional[torch.Tensor]
    total: torch.Tensor
    q: Optional[torch.Tensor] = None
    scale: Optional[torch.Tensor] = None


_HERE = contextlib.nullcontext()


def _device_of(*tensors):
    """Makes the tensors' device the current one, whose stream the call then takes."""
    d = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != d:
            raise ValueError("tensors on %s and %s" % (tensors[0].device, t.device))
    if d < 0:
        raise ValueError("tokens live on the GPU, not on %s" % tensors[0].device)
    return _HERE if d == torch.cuda.current_device() else torch.cuda.device(d)


def _fp32(t, n, what):
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError("%s is %d contiguous float32 values" % (what, n))


def _workspace(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def rms_norm(x, weight, eps=1e-6, residual=None, eight_bit=False) -> Normed:
    """s = x + residual; y = s * weight / sqrt(mean(s^2) + eps), for x [rows, cols]."""
    with _device_of(x, weight, residual):
        rows, cols = x.shape
        _fp32(weight, cols, "weight")
        total = torch.empty_like(x, memory_format=_DENSE) if residual is not None else None
        y = q = scale = None
        if eight_bit:
            q = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=x.device)
            scale = torch.empty(rows, -(-cols // gsmi.GS_NORM_BLOCK), dtype=torch.float32, device=x.device)
        else:
            y = torch.empty_like(x, memory_format=_DENSE)
        gsmi.gs_rms_norm(x, weight, eps, y=y, residual=residual, total=total, q=q, q_scale=scale)
        return Normed(y, x if total is None else total, q, scale)


def rms_norm_backward(dy, total, weight, eps=1e-6, dtotal=None):
    """(dx, dweight) of rms_norm; dx is the gradient of x and of residual."""
    with _device_of(dy, total, weight, dtotal):
        rows, cols = total.shape
        _fp32(weight, cols, "weight")
        dx = torch.empty_like(total, memory_format=_DENSE)
        dweight = torch.empty_like(weight)
        ws = _workspace(gsmi.gs_rms_norm_bwd_ws_bytes(rows, cols), total.device)
        gsmi.gs_rms_norm_bwd(dy, total, weight, eps, dx, dweight, ws, dtotal=dtotal)
        return dx, dweight


def rotary(tensors, pos, freq, axis_pairs, interleaved=False, inverse=False, amplitude=1.0, inplace=False):
    """Turns one or two [tokens, heads, dim] tensors by pos [tokens, axes]; returns them as a tuple.

    inplace: the tensors themselves are turned; autograd sees that they changed (as for the other functions here, not
    how: `Rotary` is the form with a gradient)."""
    tensors = (tensors,) if isinstance(tensors, torch.Tensor) else tuple(tensors)
    with _device_of(*tensors, pos, freq):
        if pos.dtype != torch.float32 or pos.dim() != 2 or pos.shape != (tensors[0].shape[0], len(axis_pairs)):
            raise ValueError("pos is float32 [tokens, %d]" % len(axis_pairs))
        _fp32(freq, sum(axis_pairs), "freq")
        out = tensors if inplace else tuple(torch.empty_like(t, memory_format=_DENSE) for t in tensors)
        gsmi.gs_rotary(tensors, out, pos, freq, axis_pairs, interleaved, inverse, amplitude)
        if inplace:
            torch.autograd.graph.increment_version(tensors)    # what autograd has saved of them is no longer there
        return out


def attention(q, k, v, cu_q=None, cu_k=None, n_seg=1, key_on=None, scale=None, left=-1, right=-1):
    """(out, lse): q [n_q, heads, dim] over k, v [n_k, kv_heads, dim], segment by segment.

    Rows outside every segment (behind the last start of a buffer at capacity) have out 0 and lse -inf."""
    with _device_of(q, k, v, cu_q, cu_k, key_on):
        a = gsmi.make_attn(q, k, v, q.shape[2] ** -0.5 if scale is None else scale, n_seg, cu_q, cu_k, key_on, left, right,
                           fill=True)
        out = torch.empty_like(q, memory_format=_DENSE)
        lse = torch.empty(q.shape[0], q.shape[1], dtype=torch.float32, device=q.device)
        gsmi.gs_attention(a, out, lse, _workspace(gsmi.gs_attention_ws_bytes(a), q.device))
        return out, lse


def attention_backward(dout, q, k, v, out, lse, cu_q=None, cu_k=None, n_seg=1, key_on=None, scale=None, left=-1,
                       right=-1):
    """(dq, dk, dv) of attention, from its result and log sums; 0 for rows and keys outside every segment."""
    with _device_of(q, k, v, dout, out, lse, cu_q, cu_k, key_on):
        for t, what in ((dout, "dout"), (out, "out")):
            if t.shape != q.shape or t.dtype != q.dtype:
                raise ValueError("%s has q's shape and type" % what)
        _fp32(lse, q.shape[0] * q.shape[1], "lse")
        a = gsmi.make_attn(q, k, v, q.shape[2] ** -0.5 if scale is None else scale, n_seg, cu_q, cu_k, key_on, left, right,
                           fill=True)
        dq, dk, dv = (torch.empty_like(t, memory_format=_DENSE) for t in (q, k, v))
        gsmi.gs_attention_bwd(a, out, lse, dout, dq, dk, dv, _workspace(gsmi.gs_attention_ws_bytes(a, True), q.device))
        return dq, dk, dv


class LayerNormed(NamedTuple):
    """What layer_norm returns: y and the sum (x itself without a residual)."""
    y: torch.Tensor
    total: torch.Tensor


def layer_norm(x, weight, bias=None, eps=1e-5, residual=None) -> LayerNormed:
    """s = x + residual; y = (s - mean(s)) * weight / sqrt(var(s) + eps) + bias, for x [rows, cols]."""
    with _device_of(x, weight, bias, residual):
        cols = x.shape[1]
        _fp32(weight, cols, "weight")
        if bias is not None:
            _fp32(bias, cols, "bias")
        total = torch.empty_like(x, memory_format=_DENSE) if residual is not None else None
        y = torch.empty_like(x, memory_format=_DENSE)
        gsmi.gs_layer_norm(x, weight, bias, eps, y=y, residual=residual, total=total)
        return LayerNormed(y, x if total is None else total)


def layer_norm_backward(dy, total, weight, eps=1e-5, dtotal=None):
    """(dx, dweight, dbias) of layer_norm; dx is the gradient of x and of residual."""
    with _device_of(dy, total, weight, dtotal):
        rows, cols = total.shape
        _fp32(weight, cols, "weight")
        dx = torch.empty_like(total, memory_format=_DENSE)
        dweight, dbias = torch.empty_like(weight), torch.empty_like(weight)
        ws = _workspace(gsmi.gs_layer_norm_bwd_ws_bytes(rows, cols), total.device)
        gsmi.gs_layer_norm_bwd(dy, total, weight, eps, dx, dweight, dbias, ws, dtotal=dtotal)
        return dx, dweight, dbias


def embedding(table, ids, scale=1.0, dtype=None):
    """scale * table[ids] as [tokens, dim] of `dtype` (None: the table's); zeros for ids outside the table (-1: none).

    table [rows, dim] is float32 or of that type, ids [tokens] int32."""
    with _device_of(table, ids):
        out = torch.empty(ids.numel(), table.shape[1], dtype=dtype or table.dtype, device=table.device)
        gsmi.gs_embedding(table, ids, scale, out)
        return out


def embedding_backward(dout, ids, rows, scale=1.0):
    """The gradient of a table of `rows` rows, [rows, dim] fp32, from dout [tokens, dim]."""
    with _device_of(dout, ids):
        grad = torch.empty(rows, dout.shape[1], dtype=torch.float32, device=dout.device)
        ws = _workspace(gsmi.gs_embedding_bwd_ws_bytes(dout.shape[0], rows, dout.shape[1]), dout.device)
        gsmi.gs_embedding_bwd(dout, ids, rows, scale, grad, ws)
        return grad


def embedding_rows(dout, ids, rows, scale=1.0, out=None):
    """(unique, count, grad): the ids that have a token, ascending, how many, and their rows of the table's gradient;
    what gs_sparse_adam takes.  Their room is min(tokens, rows); behind the count they are left as they were.
    out: the three tensors, for a program that keeps them."""
    with _device_of(dout, ids, *(out or ())):
        tokens, dim = dout.shape
        most = min(tokens, rows)
        if out is None:
            out = (torch.empty(most, dtype=torch.int32, device=dout.device),
                   torch.empty(1, dtype=torch.int32, device=dout.device),
                   torch.empty(most, dim, dtype=torch.float32, device=dout.device))
        unique, count, grad = out
        ws = _workspace(gsmi.gs_embedding_bwd_ws_bytes(tokens, rows, dim, True), dout.device)
        gsmi.gs_embedding_bwd(dout, ids, rows, scale, grad, ws, unique=unique, count=count)
        return unique, count, grad


class Scanned(NamedTuple):
    """What recurrence returns: y [n, cols], the segments' last states [n_seg, cols] fp32, and with keep the states
    that the gradient reads."""
    y: torch.Tensor
    final: torch.Tensor
    kept: Optional[torch.Tensor] = None


def recurrence(x, gate, cu=None, n_seg=1, initial=None, reverse=False, keep=False) -> Scanned:
    """h_t = a_t h_(t-1) + (1 - a_t) x_t with a = sigmoid(gate), channel by channel along each segment of x [n, cols].

    initial [n_seg, cols] fp32: the states in front of the segments' first tokens (reverse: behind their last ones).
    Rows outside every segment (behind the last start of a buffer at capacity) have y 0."""
    with _device_of(x, gate, cu, initial):
        a = gsmi.make_recur(x, gate, cu, n_seg, initial, reverse, fill=True)
        y = torch.empty_like(x, memory_format=_DENSE)
        final = torch.empty(a.n_seg, x.shape[1], dtype=torch.float32, device=x.device)
        kept = None
        if keep:
            kept = torch.empty(-(-x.shape[0] // gsmi.GS_RECUR_KEEP), x.shape[1], dtype=torch.float32, device=x.device)
        gsmi.gs_recurrence(a, y, final, kept, _workspace(gsmi.gs_recurrence_ws_bytes(a), x.device))
        return Scanned(y, final, kept)


def recurrence_backward(dy, x, gate, kept, cu=None, n_seg=1, initial=None, dfinal=None, reverse=False):
    """(dx, dgate, dinitial) of recurrence, from the states that it kept; 0 for rows outside every segment.
    dinitial is None without `initial`."""
    with _device_of(x, gate, dy, kept, cu, initial, dfinal):
        a = gsmi.make_recur(x, gate, cu, n_seg, initial, reverse, fill=True)
        dx, dgate = (torch.empty_like(x, memory_format=_DENSE) for _ in range(2))
        dinitial = torch.empty_like(initial) if initial is not None else None
        gsmi.gs_recurrence_bwd(a, dy, kept, dx, dgate, dfinal, dinitial,
                               _workspace(gsmi.gs_recurrence_ws_bytes(a), x.device))
        return dx, dgate, dinitial


class Gated(NamedTuple):
    """What gated_silu returns: h, and with keep the inputs as float8_e4m3fn with a scale byte for every 32 columns:
    u ~ 2^(u_scale - 127) * u8.

    A kept value is off by at most a 16th of itself or 2^-10 of its block's power of two, whichever is more.  The power
    follows the block's largest value (it is a 224th of that at most): beside it, what is less than a 14,336th of it
    keeps fewer bits, and what is less than a 229,376th can be kept as 0."""
    h: torch.Tensor
    u8: Optional[torch.Tensor] = None
    u_scale: Optional[torch.Tensor] = None
    v8: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None


def gated_silu(u, v=None, keep=True) -> Gated:
    """h = silu(u) * v (v None: silu(u)) for u, v [rows, cols], which may be columns of one matrix."""
    with _device_of(u, v):
        rows, cols = u.shape

        def room(t):
            if not keep or t is None:
                return None, None
            return (torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=u.device),
                    torch.empty(rows, -(-cols // gsmi.GS_KEEP_BLOCK), dtype=torch.uint8, device=u.device))

        h = torch.empty(rows, cols, dtype=u.dtype, device=u.device)
        (u8, u_scale), (v8, v_scale) = room(u), room(v)
        gsmi.gs_gated_silu(u, v, h, u8, u_scale, v8, v_scale)
        return Gated(h, u8, u_scale, v8, v_scale)


def gated_silu_backward(dh, u8, u_scale, v8=None, v_scale=None, again=True):
    """(du, dv, h) at the inputs that gated_silu kept; dv is None without v8, h without `again`."""
    with _device_of(dh, u8, u_scale, v8, v_scale):
        du, dv, h = (torch.empty(dh.shape, dtype=dh.dtype, device=dh.device) if wanted else None
                     for wanted in (True, v8 is not None, again))
        gsmi.gs_gated_silu_bwd(dh, u8, u_scale, du, v8, v_scale, dv, h)
        return du, dv, h


class RmsNorm(torch.autograd.Function):
    """RmsNorm.apply(x, residual or None, weight, eps) -> (y, total).

    The gradient reads `total` as it was rounded to the tokens' type."""

    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        r = rms_norm(x, weight, eps, residual=residual)
        total = r.total if residual is not None else x.view_as(x)
        ctx.save_for_backward(total, weight)
        ctx.eps, ctx.has_residual = eps, residual is not None
        ctx.set_materialize_grads(False)
        return r.y, total

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dtotal):
        total, weight = ctx.saved_tensors
        if dy is None:
            return dtotal, (dtotal if ctx.has_residual else None), None, None
        dx, dw = rms_norm_backward(dy.contiguous(), total, weight, ctx.eps,
                                   dtotal=None if dtotal is None else dtotal.contiguous())
        return dx, (dx if ctx.has_residual else None), dw, None


class Rotary(torch.autograd.Function):
    """Rotary.apply(q, k, pos, freq, axis_pairs, interleaved, amplitude) -> (q, k).

    q and k have gradients; pos, freq and amplitude have none (a position that is trained gets nothing from here)."""

    @staticmethod
    def forward(ctx, q, k, pos, freq, axis_pairs, interleaved, amplitude):
        ctx.save_for_backward(pos, freq)
        ctx.how = (axis_pairs, interleaved, amplitude)
        return rotary((q, k), pos, freq, axis_pairs, interleaved=interleaved, amplitude=amplitude)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        pos, freq = ctx.saved_tensors
        axis_pairs, interleaved, amplitude = ctx.how
        dq, dk = rotary((dq.contiguous(), dk.contiguous()), pos, freq, axis_pairs, interleaved=interleaved,
                        inverse=True, amplitude=amplitude)
        return dq, dk, None, None, None, None, None


class Attention(torch.autograd.Function):
    """Attention.apply(q, k, v, how) -> (out, lse); `how` holds attention()'s keyword arguments.

    q, k and v have gradients through out; lse is marked as not differentiable."""

    @staticmethod
    def forward(ctx, q, k, v, how):
        out, lse = attention(q, k, v, **how)
        tensors = {n: t for n, t in how.items() if isinstance(t, torch.Tensor)}
        ctx.save_for_backward(q, k, v, out, lse, *tensors.values())
        ctx.names, ctx.how = tuple(tensors), {n: t for n, t in how.items() if n not in tensors}
        ctx.mark_non_differentiable(lse)
        return out, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, _):
        q, k, v, out, lse, *tensors = ctx.saved_tensors
        how = dict(ctx.how, **dict(zip(ctx.names, tensors)))
        return (*attention_backward(dout.contiguous(), q, k, v, out, lse, **how), None)


class LayerNorm(torch.autograd.Function):
    """LayerNorm.apply(x, residual or None, weight, bias or None, eps) -> (y, total).

    The gradient reads `total` as it was rounded to the tokens' type."""

    @staticmethod
    def forward(ctx, x, residual, weight, bias, eps):
        r = layer_norm(x, weight, bias, eps, residual=residual)
        total = r.total if residual is not None else x.view_as(x)
        ctx.save_for_backward(total, weight)
        ctx.eps, ctx.has_residual, ctx.has_bias = eps, residual is not None, bias is not None
        ctx.set_materialize_grads(False)
        return r.y, total

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dtotal):
        total, weight = ctx.saved_tensors
        if dy is None:
            return dtotal, (dtotal if ctx.has_residual else None), None, None, None
        dx, dw, db = layer_norm_backward(dy.contiguous(), total, weight, ctx.eps,
                                         dtotal=None if dtotal is None else dtotal.contiguous())
        return dx, (dx if ctx.has_residual else None), dw, (db if ctx.has_bias else None), None


class Embedding(torch.autograd.Function):
    """Embedding.apply(table, ids, scale, dtype or None) -> [tokens, dim]; table has a dense gradient, in fp32 until it
    is rounded to the table's type."""

    @staticmethod
    def forward(ctx, table, ids, scale, dtype):
        ctx.save_for_backward(ids)
        ctx.how = (table.shape[0], scale, table.dtype)
        return embedding(table, ids, scale, dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        (ids,) = ctx.saved_tensors
        rows, scale, dtype = ctx.how
        return embedding_backward(dout.contiguous(), ids, rows, scale).to(dtype), None, None, None


class Recurrence(torch.autograd.Function):
    """Recurrence.apply(x, gate, initial or None, how) -> (y, final); `how` holds cu or n_seg, and reverse.

    x, gate and initial have gradients, through y and final alike."""

    @staticmethod
    def forward(ctx, x, gate, initial, how):
        r = recurrence(x, gate, initial=initial, keep=True, **how)
        ctx.save_for_backward(x, gate, initial, r.kept, how.get("cu"))
        ctx.how = {k: v for k, v in how.items() if k != "cu"}
        ctx.set_materialize_grads(False)
        return r.y, r.final

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dfinal):
        x, gate, initial, kept, cu = ctx.saved_tensors
        if dy is None and dfinal is None:
            return None, None, None, None
        dy = torch.zeros_like(x) if dy is None else dy.contiguous()
        dfinal = None if dfinal is None else dfinal.contiguous()
        return (*recurrence_backward(dy, x, gate, kept, cu=cu, initial=initial, dfinal=dfinal, **ctx.how), None)


class GatedSilu(torch.autograd.Function):
    """GatedSilu.apply(u, v or None) -> h.  Saved for the gradient are u and v in 8 bits, not themselves; the gradient
    is that at those values.  `Gated` says how far off they are: a 16th at most, but for values far below the largest of
    their 32 columns."""

    @staticmethod
    def forward(ctx, u, v):
        r = gated_silu(u, v)
        ctx.save_for_backward(r.u8, r.u_scale, r.v8, r.v_scale)
        return r.h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        du, dv, _ = gated_silu_backward(dh.contiguous(), *ctx.saved_tensors, again=False)
        return du, dv


class GatedProjection(torch.autograd.Function):
    """GatedProjection.apply(both, down) -> silu(u) * v @ down, for both [rows, 2 * hidden] = (u, v) as one projection
    gives them and down [hidden, cols].

    Saved for the gradient are u and v in 8 bits and `down`; the product's operand is formed again from them, so that
    none of the three [rows, hidden] matrices is held in the tokens' type.  The gradients are those at the kept values
    (`Gated` says how far off those are)."""

    @staticmethod
    def forward(ctx, both, down):
        hidden = both.shape[1] // 2
        if both.shape[1] != 2 * hidden or down.shape[0] != hidden:
            raise ValueError("both %s is not twice as wide as down %s is high" % (tuple(both.shape), tuple(down.shape)))
        r = gated_silu(both[:, :hidden], both[:, hidden:])
        ctx.save_for_backward(r.u8, r.u_scale, r.v8, r.v_scale, down)
        return r.h @ down

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        u8, u_scale, v8, v_scale, down = ctx.saved_tensors
        rows, hidden = u8.shape
        dh = dout @ down.T
        with _device_of(dh, u8):
            dboth = torch.empty(rows, 2 * hidden, dtype=dh.dtype, device=dh.device)
            h = torch.empty_like(dh, memory_format=_DENSE)
            gsmi.gs_gated_silu_bwd(dh, u8, u_scale, dboth[:, :hidden], v8, v_scale, dboth[:, hidden:], h)
        return dboth, h.T @ dout
