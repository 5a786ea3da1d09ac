"""Token operators for a network that writes rows of the pool: the norm with
the residual's addition, the rotation by position and attention over ragged
segments, each with its gradient.

The functions allocate their outputs and workspaces with torch on the current
stream of their tensors' GPU and call the gs_* entry points there; every step
runs in libgsmi's kernels.  `RmsNorm`, `Rotary` and `Attention` put them under torch's autograd;
their gradients have none of their own, a second derivative raises.
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
