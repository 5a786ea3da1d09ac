"""The token operators' entry points reject bad arguments before any GPU call,
and the frequency table follows its formula (host calls, no GPU needed)."""
import ctypes
import math

import numpy as np
import pytest


@pytest.fixture(scope="module")
def gs():
    from paper_2607_19893_amd import gsmi
    return gsmi


def refused(gs, status, word, code=None):
    assert status == (gs.GS_ERR_INVALID_ARG if code is None else code), gs.gs_last_error()
    assert word in gs.gs_last_error(), gs.gs_last_error()


def norm_args(gs, **kw):
    a = gs.gs_norm_args(4, 64, gs.GS_BF16, 1e-6, 256, None, 256, None, 512, None, None, 64, 64, 64, 64, 64, 1)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("word,kw", [
    ("dtype", dict(dtype=3)), ("rows", dict(rows=-1)), ("cols", dict(cols=0)), ("eps", dict(eps=-1.0)),
    ("eps", dict(eps=math.nan)), ("weight", dict(weight=None)), ("weight", dict(weight=258)), ("null x", dict(x=None)),
    ("aligned", dict(x=257)), ("below", dict(ld_x=63)), ("residual", dict(residual=256, ld_residual=1)),
    ("total", dict(total=256, ld_total=2)), ("no output", dict(y=None)), ("q_scale", dict(q=1)),
    ("q_scale", dict(q=1, q_scale=4, ld_scale=0))])
def test_norm_arguments(gs, word, kw):
    refused(gs, gs.raw().gs_rms_norm(ctypes.byref(norm_args(gs, **kw)), None), word)


def test_norm_sizes(gs):
    L = gs.raw()
    refused(gs, L.gs_rms_norm(None, None), "null args")
    a = norm_args(gs, cols=16385, ld_x=16385, ld_y=16385)
    refused(gs, L.gs_rms_norm(ctypes.byref(a), None), "16384", gs.GS_ERR_UNSUPPORTED)
    assert L.gs_rms_norm(ctypes.byref(norm_args(gs, rows=0, x=None, y=None)), None) == gs.GS_OK
    b = gs.gs_norm_bwd_args(4, 64, gs.GS_F32, 1e-6, 256, 256, None, 256, 256, 256, 64, 64, 64, 64)
    refused(gs, L.gs_rms_norm_bwd(ctypes.byref(b), None, 1 << 20, None), "workspace")
    refused(gs, L.gs_rms_norm_bwd(ctypes.byref(b), 8, 1 << 20, None), "workspace")
    refused(gs, L.gs_rms_norm_bwd(ctypes.byref(b), 256, 0, None), "too small", gs.GS_ERR_WORKSPACE)
    for field in ("dy", "total", "dx", "dweight", "weight"):
        c = gs.gs_norm_bwd_args.from_buffer_copy(b)
        setattr(c, field, None)
        refused(gs, L.gs_rms_norm_bwd(ctypes.byref(c), 256, 1 << 20, None), field)
    assert gs.gs_rms_norm_bwd_ws_bytes(-1, 5) == 0 and gs.gs_rms_norm_bwd_ws_bytes(100000, 768) >= 512 * 768 * 4


def rotary_args(gs, **kw):
    a = gs.gs_rotary_args()
    a.dtype, a.tokens, a.dim, a.pairs, a.n_axes = gs.GS_BF16, 8, 64, 32, 1
    a.axis_pairs[0] = 32
    a.amplitude, a.pos, a.ld_pos, a.freq, a.n_tensors = 1.0, 256, 1, 256, 1
    a.heads[0] = 2
    a.inp[0] = a.out[0] = gs.gs_rows(256, 128, 64)
    for k, v in kw.items():
        if k == "axis_pairs":
            for i, n in enumerate(v):
                a.axis_pairs[i] = n
        elif k in ("inp", "out", "heads"):
            getattr(a, k)[0] = v
        else:
            setattr(a, k, v)
    return a


def test_rotary_arguments(gs):
    L = gs.raw()
    refused(gs, L.gs_rotary(None, None), "null args")
    for word, kw in (("dtype", dict(dtype=9)), ("size", dict(tokens=-1)), ("size", dict(dim=0)), ("pairs", dict(pairs=33)),
                     ("axes", dict(n_axes=4)), ("axes", dict(n_axes=0)), ("sum", dict(axis_pairs=[31])),
                     ("negative", dict(axis_pairs=[-1])), ("amplitude", dict(amplitude=math.inf)),
                     ("tensors", dict(n_tensors=3)), ("freq", dict(freq=None)), ("pos", dict(pos=None)),
                     ("ld_pos", dict(ld_pos=0)), ("heads", dict(heads=-1)), ("misaligned", dict(inp=gs.gs_rows(257, 128, 64))),
                     ("null", dict(out=gs.gs_rows(None, 128, 64))), ("head stride", dict(inp=gs.gs_rows(256, 128, 63))),
                     ("row stride", dict(out=gs.gs_rows(512, 8, 64))), ("in place", dict(out=gs.gs_rows(256, 256, 64)))):
        refused(gs, L.gs_rotary(ctypes.byref(rotary_args(gs, **kw)), None), word)
    refused(gs, L.gs_rotary(ctypes.byref(rotary_args(gs, dim=1024)), None), "512", gs.GS_ERR_UNSUPPORTED)
    assert L.gs_rotary(ctypes.byref(rotary_args(gs, tokens=0)), None) == gs.GS_OK


def attn(gs, **kw):
    r = gs.gs_rows(256, 128, 64)
    a = gs.gs_attn(gs.GS_BF16, 8, 8, 1, 2, 2, 64, -1, -1, 0.125, None, None, None, r, r, r)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_attention_arguments(gs):
    L = gs.raw()
    out = gs.gs_rows(256, 128, 64)
    call = lambda a, o=out, lse=256: L.gs_attention(ctypes.byref(a), ctypes.byref(o), lse, 256, 1 << 30, None)
    refused(gs, L.gs_attention(None, None, None, None, 0, None), "null args")
    for word, kw in (("dtype", dict(dtype=gs.GS_F32)), ("count", dict(n_q=-1)), ("count", dict(n_seg=0)),
                     ("divide", dict(heads=3)), ("divide", dict(kv_heads=0)), ("dim", dict(dim=20)), ("dim", dict(dim=0)),
                     ("scale", dict(scale=0.0)), ("scale", dict(scale=math.nan)), ("scale", dict(scale=math.inf)),
                     ("together", dict(cu_q=256)), ("misaligned", dict(cu_q=258, cu_k=256)),
                     ("equal length", dict(n_seg=3)), ("null q", dict(q=gs.gs_rows(None, 128, 64))),
                     ("16-byte", dict(k=gs.gs_rows(264, 128, 64))), ("multiples", dict(v=gs.gs_rows(256, 132, 64))),
                     ("row stride", dict(k=gs.gs_rows(256, 0, 64))), ("row stride", dict(k=gs.gs_rows(256, 1 << 24, 64))),
                     ("row stride", dict(k=gs.gs_rows(256, -128, 64)))):
        refused(gs, call(attn(gs, **kw)), word)
    refused(gs, call(attn(gs, dim=136)), "128", gs.GS_ERR_UNSUPPORTED)
    refused(gs, call(attn(gs, n_q=1 << 30, heads=4, kv_heads=2)), "2^31", gs.GS_ERR_UNSUPPORTED)
    refused(gs, call(attn(gs), gs.gs_rows(None, 128, 64)), "null out")
    refused(gs, call(attn(gs), lse=None), "lse")
    few = attn(gs, n_q=1, n_k=8192)
    assert gs.gs_attention_ws_bytes(few) > 0
    refused(gs, L.gs_attention(ctypes.byref(few), ctypes.byref(out), 256, 256, 16, None), "too small",
            gs.GS_ERR_WORKSPACE)
    refused(gs, L.gs_attention(ctypes.byref(few), ctypes.byref(out), 256, None, 1 << 30, None), "workspace")
    assert call(attn(gs, n_q=0)) == gs.GS_OK
    g = gs.gs_attn_grads(out, out, out, out, out, 256)
    need = gs.gs_attention_ws_bytes(attn(gs), True)
    assert need >= 8 * 2 * 8
    refused(gs, L.gs_attention_bwd(ctypes.byref(attn(gs)), None, 256, 1 << 20, None), "null gradients")
    refused(gs, L.gs_attention_bwd(ctypes.byref(attn(gs)), ctypes.byref(g), 256, need - 1, None), "too small",
            gs.GS_ERR_WORKSPACE)
    refused(gs, L.gs_attention_bwd(ctypes.byref(attn(gs)), ctypes.byref(g), 8, need, None), "workspace")
    for field in ("out", "dout", "dq", "dk", "dv"):
        b = gs.gs_attn_grads.from_buffer_copy(g)
        setattr(b, field, gs.gs_rows(None, 128, 64))
        refused(gs, L.gs_attention_bwd(ctypes.byref(attn(gs)), ctypes.byref(b), 256, need, None), "null " + field)
    assert gs.gs_attention_ws_bytes(attn(gs, kv_heads=0)) == 0


def test_attention_sizes_that_no_launch_holds(gs):
    """Places near 2^31, and more tiles than a launch has workgroups (128 key heads of 2^25 segments wrap a 32-bit grid)."""
    L = gs.raw()
    out, g = gs.gs_rows(256, 128, 64), gs.gs_attn_grads(*[gs.gs_rows(256, 128, 64)] * 5, 256)
    for word, kw in (("2^30", dict(n_k=(1 << 30) + 1, heads=1, kv_heads=1)), ("2^30", dict(n_k=0x7FFFFFFF, heads=1, kv_heads=1)),
                     ("2^30", dict(n_q=(1 << 29) + 1)), ("tiles", dict(n_seg=1 << 25, cu_q=256, cu_k=256)),
                     ("tiles", dict(n_seg=1 << 18, heads=128, kv_heads=128, cu_q=256, cu_k=256)),
                     ("tiles", dict(n_seg=0x7FFFFFFF, heads=256, kv_heads=256, cu_q=256, cu_k=256))):
        a = attn(gs, **kw)
        refused(gs, L.gs_attention(ctypes.byref(a), ctypes.byref(out), 256, 256, 1 << 62, None), word, gs.GS_ERR_UNSUPPORTED)
        refused(gs, L.gs_attention_bwd(ctypes.byref(a), ctypes.byref(g), 256, 1 << 62, None), word, gs.GS_ERR_UNSUPPORTED)
    a = rotary_args(gs, heads=1 << 25)
    refused(gs, L.gs_rotary(ctypes.byref(a), None), "2^30", gs.GS_ERR_UNSUPPORTED)


def test_frequencies(gs):
    for pairs, base in ((1, 10000.0), (32, 10000.0), (64, 500000.0)):
        plain = base ** -(np.arange(pairs) / pairs)
        f, amp = gs.gs_rotary_freqs(pairs, base)
        assert amp == 1.0 and np.allclose(f, plain, rtol=1e-7, atol=0)
        f, _ = gs.gs_rotary_freqs(pairs, base, gs.GS_ROPE_LINEAR, 4.0)
        assert np.allclose(f, plain / 4, rtol=1e-7, atol=0)
        if pairs > 1:
            f, _ = gs.gs_rotary_freqs(pairs, base, gs.GS_ROPE_BASE, 4.0)
            assert f[0] == 1.0 and np.isclose(f[-1], plain[-1] / 4, rtol=1e-6)
            f, amp = gs.gs_rotary_freqs(pairs, base, gs.GS_ROPE_PARTS, 8.0, 4096.0, 1.0, 32.0)
            turns = 4096 * plain / (2 * math.pi)
            t = np.clip((turns - 1) / 31, 0, 1)
            assert np.allclose(f, t * plain + (1 - t) * plain / 8, rtol=1e-6, atol=0)
            assert np.isclose(amp, 1 + 0.1 * math.log(8.0))
    for bad in (dict(pairs=0), dict(base=1.0), dict(scaling=4), dict(scaling=1, factor=0.5), dict(pairs=1, scaling=2, factor=2.0),
                dict(scaling=3, factor=2.0), dict(scaling=3, factor=2.0, trained=100.0, slow=5.0, fast=5.0)):
        with pytest.raises(gs.GsmiError):
            gs.gs_rotary_freqs(**dict(dict(pairs=8), **bad))
