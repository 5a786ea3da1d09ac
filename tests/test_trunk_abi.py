"""The entry points of the layer norm, embedding, recurrence and gated SiLU reject bad arguments before any GPU call
(host calls, no GPU needed)."""
import ctypes
import math
import os
import re

import pytest

from test_tokens_abi import gs, refused  # noqa: F401 (gs: a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def changed(a, kw):
    b = type(a).from_buffer_copy(a)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def test_constants_match_header(gs):
    d = dict(re.findall(r"#define (GS_\w+) (\d+)", open(os.path.join(ROOT, "include", "gsmi.h")).read()))
    for k in ("GS_EMBED_MAX_DIM", "GS_EMBED_MAX_TOKENS", "GS_RECUR_KEEP", "GS_KEEP_BLOCK", "GS_SILU_MAX_COLS"):
        assert int(d[k]) == getattr(gs, k), k


def layer(gs):
    return gs.gs_layer_args(4, 64, gs.GS_BF16, 1e-5, 256, None, 256, 256, None, 512, 64, 64, 64, 64)


@pytest.mark.parametrize("word,kw", [
    ("dtype", dict(dtype=3)), ("rows", dict(rows=-1)), ("cols", dict(cols=0)), ("eps", dict(eps=-1.0)),
    ("eps", dict(eps=math.inf)), ("weight", dict(weight=None)), ("weight", dict(weight=258)), ("bias", dict(bias=258)),
    ("null x", dict(x=None)), ("aligned", dict(x=257)), ("below", dict(ld_x=63)), ("residual", dict(residual=256, ld_residual=1)),
    ("total", dict(total=256, ld_total=2)), ("y", dict(ld_y=63)), ("no output", dict(y=None))])
def test_layer_norm_arguments(gs, word, kw):
    refused(gs, gs.raw().gs_layer_norm(ctypes.byref(changed(layer(gs), kw)), None), word)


def test_layer_norm_sizes(gs):
    L = gs.raw()
    refused(gs, L.gs_layer_norm(None, None), "null args")
    refused(gs, L.gs_layer_norm(ctypes.byref(changed(layer(gs), dict(cols=16385, ld_x=16385, ld_y=16385))), None), "16384",
            gs.GS_ERR_UNSUPPORTED)
    assert L.gs_layer_norm(ctypes.byref(changed(layer(gs), dict(rows=0, x=None, y=None))), None) == gs.GS_OK
    b = gs.gs_layer_bwd_args(4, 64, gs.GS_F32, 1e-5, 256, 256, None, 256, 256, 256, 256, 64, 64, 64, 64)
    refused(gs, L.gs_layer_norm_bwd(None, 256, 1 << 20, None), "null args")
    refused(gs, L.gs_layer_norm_bwd(ctypes.byref(b), None, 1 << 20, None), "workspace")
    refused(gs, L.gs_layer_norm_bwd(ctypes.byref(b), 8, 1 << 20, None), "workspace")
    refused(gs, L.gs_layer_norm_bwd(ctypes.byref(b), 256, 0, None), "too small", gs.GS_ERR_WORKSPACE)
    for field in ("dy", "total", "dx", "dweight", "weight"):
        refused(gs, L.gs_layer_norm_bwd(ctypes.byref(changed(b, {field: None})), 256, 1 << 20, None), field)
    for word, kw in (("dbias", dict(dbias=257)), ("dtotal", dict(dtotal=256, ld_dtotal=3)), ("dtype", dict(dtype=7))):
        refused(gs, L.gs_layer_norm_bwd(ctypes.byref(changed(b, kw)), 256, 1 << 20, None), word)
    assert gs.gs_layer_norm_bwd_ws_bytes(-1, 5) == 0
    assert gs.gs_layer_norm_bwd_ws_bytes(100000, 768) >= 512 * 2 * 768 * 4


def embed(gs):
    return gs.gs_embed_args(gs.GS_BF16, gs.GS_F32, 8, 10, 64, 1.0, 256, 256, 512, 64, 64)


@pytest.mark.parametrize("word,kw", [
    ("dtype", dict(dtype=3)), ("table_dtype", dict(table_dtype=2)), ("tokens", dict(tokens=-1)),
    ("rows", dict(rows=-1)), ("dim", dict(dim=0)), ("scale", dict(scale=math.nan)), ("scale", dict(scale=math.inf)),
    ("ids", dict(ids=None)), ("ids", dict(ids=258)), ("null table", dict(table=None)), ("table", dict(table=258)),
    ("below", dict(ld_table=63)), ("null out", dict(out=None)), ("out", dict(out=257)), ("below", dict(ld_out=1))])
def test_embedding_arguments(gs, word, kw):
    refused(gs, gs.raw().gs_embedding(ctypes.byref(changed(embed(gs), kw)), None), word)


def test_embedding_sizes(gs):
    L = gs.raw()
    refused(gs, L.gs_embedding(None, None), "null args")
    big = dict(dim=16385, ld_table=16385, ld_out=16385)
    refused(gs, L.gs_embedding(ctypes.byref(changed(embed(gs), big)), None), "16384", gs.GS_ERR_UNSUPPORTED)
    assert L.gs_embedding(ctypes.byref(changed(embed(gs), dict(tokens=0, ids=None, out=None))), None) == gs.GS_OK
    b = gs.gs_embed_bwd_args(gs.GS_BF16, 8, 10, 64, 1.0, 256, 256, 256, None, None, 64, 64)
    need = gs.gs_embedding_bwd_ws_bytes(8, 10, 64)
    call = lambda a, ws=256, n=1 << 30: L.gs_embedding_bwd(ctypes.byref(a), ws, n, None)
    refused(gs, L.gs_embedding_bwd(None, 256, 1 << 30, None), "null args")
    refused(gs, call(b, ws=None), "workspace")
    refused(gs, call(b, ws=8), "workspace")
    refused(gs, call(b, n=need - 1), "too small", gs.GS_ERR_WORKSPACE)
    for word, kw in (("dtype", dict(dtype=3)), ("ids", dict(ids=None)), ("null dout", dict(dout=None)), ("below", dict(ld_dout=63)),
                     ("null grad", dict(grad=None)), ("grad", dict(grad=258)), ("below", dict(ld_grad=63)),
                     ("together", dict(unique=256)), ("together", dict(count=256)), ("misaligned", dict(unique=257, count=256)),
                     ("misaligned", dict(unique=256, count=258))):
        refused(gs, call(changed(b, kw)), word)
    refused(gs, call(changed(b, dict(tokens=(1 << 28) + 1))), "tokens", gs.GS_ERR_UNSUPPORTED)
    assert call(changed(b, dict(rows=0, grad=None))) == gs.GS_OK
    for bad in ((-1, 10, 64), (8, -1, 64), (8, 10, 0), (8, 10, 16385), ((1 << 28) + 1, 10, 64)):
        assert gs.gs_embedding_bwd_ws_bytes(*bad) == 0
    # the workspace holds the sorted tokens twice, never the table; its marks only where the whole gradient is wanted
    assert gs.gs_embedding_bwd_ws_bytes(1000, 1 << 30, 64, True) < 1 << 21
    assert (1 << 30) < gs.gs_embedding_bwd_ws_bytes(1000, 1 << 30, 64, False) < (1 << 30) + (1 << 21)


def recur(gs, **kw):
    return changed(gs.gs_recur(gs.GS_BF16, 8, 64, 2, 0, 0, None, 256, 256, None, 64, 64), kw)


@pytest.mark.parametrize("word,kw", [
    ("dtype", dict(dtype=3)), ("n < 0", dict(n=-1)), ("cols", dict(cols=0)), ("n_seg", dict(n_seg=0)),
    ("equal length", dict(n_seg=3)), ("cu", dict(cu=258)), ("initial", dict(initial=258)), ("null x", dict(x=None)),
    ("null gate", dict(gate=None)), ("aligned", dict(x=257)), ("below", dict(ld_x=63)), ("below", dict(ld_gate=1))])
def test_recurrence_arguments(gs, word, kw):
    L = gs.raw()
    a = recur(gs, **kw)
    refused(gs, L.gs_recurrence(ctypes.byref(a), 256, 64, None, None, 256, 1 << 30, None), word)
    g = gs.gs_recur_grads(256, None, 256, 256, 256, None, 64, 64, 64)
    refused(gs, L.gs_recurrence_bwd(ctypes.byref(a), ctypes.byref(g), 256, 1 << 30, None), word)


def test_recurrence_sizes(gs):
    L = gs.raw()
    fwd = lambda a, y=256, ld=64, final=None, kept=None, ws=256, n=1 << 40: L.gs_recurrence(
        ctypes.byref(a), y, ld, final, kept, ws, n, None)
    refused(gs, L.gs_recurrence(None, 256, 64, None, None, 256, 0, None), "null args")
    refused(gs, fwd(recur(gs), y=None), "null y")
    refused(gs, fwd(recur(gs), ld=63), "below")
    refused(gs, fwd(recur(gs), final=258), "final")
    refused(gs, fwd(recur(gs), kept=258), "kept")
    long = recur(gs, n=4000)
    need = gs.gs_recurrence_ws_bytes(long)
    assert need > 0
    refused(gs, fwd(long, ws=None), "workspace")
    refused(gs, fwd(long, ws=8), "workspace")
    refused(gs, fwd(long, n=need - 1), "too small", gs.GS_ERR_WORKSPACE)
    for word, kw in (("2^30", dict(n=(1 << 30) + 2)), ("2^28", dict(n_seg=(1 << 28) + 1, cu=256)),
                     ("2^22", dict(n=1 << 28, cols=1024, ld_x=1024, ld_gate=1024)), ("2^22", dict(cols=0x7FFFFFF0))):
        refused(gs, fwd(recur(gs, **kw)), word, gs.GS_ERR_UNSUPPORTED)
    g = gs.gs_recur_grads(256, None, 256, 256, 256, None, 64, 64, 64)
    bwd = lambda a, b=g, ws=256, n=1 << 40: L.gs_recurrence_bwd(ctypes.byref(a), ctypes.byref(b), ws, n, None)
    refused(gs, L.gs_recurrence_bwd(ctypes.byref(recur(gs)), None, 256, 1 << 30, None), "null gradients")
    for word, kw in (("null dy", dict(dy=None)), ("kept", dict(kept=None)), ("null dx", dict(dx=None)), ("null dgate", dict(dgate=None)),
                     ("below", dict(ld_dx=63)), ("dfinal", dict(dfinal=257)), ("dinitial", dict(dinitial=258))):
        refused(gs, bwd(recur(gs), changed(g, kw)), word)
    refused(gs, bwd(long, n=need - 1), "too small", gs.GS_ERR_WORKSPACE)
    assert gs.gs_recurrence_ws_bytes(recur(gs, n=-1)) == 0


def silu(gs):
    return gs.gs_silu_args(4, 64, gs.GS_BF16, 256, 256, 256, 1, 1, 1, 1, 64, 64, 64, 64, 2, 64, 2)


@pytest.mark.parametrize("word,kw", [
    ("dtype", dict(dtype=3)), ("rows", dict(rows=-1)), ("cols", dict(cols=0)), ("null u", dict(u=None)), ("aligned", dict(u=257)),
    ("below", dict(ld_u=63)), ("below", dict(ld_v=63)), ("below", dict(ld_h=63)), ("together", dict(v8=None)),
    ("together", dict(u8=None)), ("together", dict(v=None)), ("u_scale", dict(u_scale=None)), ("v_scale", dict(v_scale=None)),
    ("below", dict(ld_u8=63)), ("below", dict(ld_u_scale=1)), ("below", dict(ld_v_scale=1)),
    ("no output", dict(h=None, u8=None, v8=None))])
def test_gated_silu_arguments(gs, word, kw):
    refused(gs, gs.raw().gs_gated_silu(ctypes.byref(changed(silu(gs), kw)), None), word)


def test_gated_silu_sizes(gs):
    L = gs.raw()
    refused(gs, L.gs_gated_silu(None, None), "null args")
    refused(gs, L.gs_gated_silu(ctypes.byref(changed(silu(gs), dict(cols=(1 << 22) + 1))), None), "4194304",
            gs.GS_ERR_UNSUPPORTED)
    assert L.gs_gated_silu(ctypes.byref(changed(silu(gs), dict(rows=0))), None) == gs.GS_OK
    b = gs.gs_silu_bwd_args(4, 64, gs.GS_F32, 256, 1, 1, 1, 1, 256, 256, 256, 64, 64, 2, 64, 2, 64, 64, 64)
    refused(gs, L.gs_gated_silu_bwd(None, None), "null args")
    for word, kw in (("dtype", dict(dtype=3)), ("null dh", dict(dh=None)), ("null u8", dict(u8=None)), ("u_scale", dict(u_scale=None)),
                     ("null du", dict(du=None)), ("together", dict(dv=None)), ("together", dict(v8=None)), ("v_scale", dict(v_scale=None)),
                     ("below", dict(ld_dv=63)), ("below", dict(ld_h=1)), ("aligned", dict(h=258))):
        refused(gs, L.gs_gated_silu_bwd(ctypes.byref(changed(b, kw)), None), word)
