"""Edges of the trunk's entry points that need no GPU: workspaces, sizes, types, what the documentation says."""
import pytest
import torch

from test_tokens_abi import gs, refused  # noqa: F401 (gs: a fixture)
from test_trunk_abi import recur


@pytest.mark.parametrize("n,cols", [(257, 1), (4000, 64), (4000, 129), (400_000, 2048)])
def test_recurrence_workspace_holds_lines_of_its_own(gs, n, cols):
    """Any 16-byte aligned workspace is taken, and the chunks' maps and the groups' states in it start at a line: there is
    room to move up to one."""
    up = lambda b: -(-b // 256) * 256
    chunks, width = -(-n // 128), 126 if cols % 128 == 1 and cols > 1 else 128
    groups, blocks = -(-chunks // 16), -(-cols // width)
    regions = up(chunks * blocks * 64 * 16) + up(groups * blocks * 64 * 16) + up(groups * blocks * 64 * 8) \
        + up((chunks + groups + 32) * blocks * 4)
    assert gs.gs_recurrence_ws_bytes(recur(gs, n=n, cols=cols, ld_x=cols, ld_gate=cols, n_seg=1)) >= regions + 240


def test_recurrence_of_one_chunk_needs_no_workspace(gs):
    assert gs.gs_recurrence_ws_bytes(recur(gs, n=256, n_seg=1)) == 0


@pytest.mark.parametrize("n,cols", [(1, 2 ** 29 - 129), (127, (2 ** 22 * 126 - 25_000) // 128 * 128 + 1)])
def test_recurrence_of_more_threads_than_a_launch_holds(gs, n, cols):
    """The only chunk's workgroups have 1024 threads, blocks of channels can be narrower than 128, and workgroups that see to
    empty segments come on top."""
    import ctypes

    L = gs.raw()
    a = recur(gs, n=n, cols=cols, ld_x=cols, ld_gate=cols, n_seg=1, cu=256)
    blocks = -(-cols // (126 if cols % 128 == 1 else 128))
    assert (n // 128 + 1) * (cols // 128 + 1) < 1 << 22 and (blocks + 256) * 1024 >= 1 << 32
    refused(gs, L.gs_recurrence(ctypes.byref(a), 256, cols, 256, 256, None, 0, None), "2^22", gs.GS_ERR_UNSUPPORTED)
    g = gs.gs_recur_grads(256, 256, 256, 256, 256, 256, cols, cols, cols)
    refused(gs, L.gs_recurrence_bwd(ctypes.byref(a), ctypes.byref(g), None, 0, None), "2^22", gs.GS_ERR_UNSUPPORTED)


@pytest.mark.parametrize("q,scale", [("float8_e5m2", "uint8"), ("float8_e4m3fnuz", "uint8"), ("float8_e4m3fn", "float8_e4m3fn"),
                                     ("float16", "uint8"), ("float8_e4m3fn", None)])
def test_other_numbers_of_eight_bits_are_refused(q, scale):
    """By the binding, before the library reads them as e4m3 and powers of two."""
    from paper_2607_19893_amd import gsmi

    made = lambda name, *shape: None if name is None else torch.zeros(*shape).to(getattr(torch, name))
    x, q, s = torch.zeros(5, 64), made(q, 5, 64), made(scale, 5, 2)
    with pytest.raises(ValueError, match="e4m3"):
        gsmi.gs_gated_silu(x, None, x, q, s)
    with pytest.raises(ValueError, match="e4m3"):
        gsmi.gs_gated_silu_bwd(x, q, s, x)


def test_bytes_and_their_types_are_taken(monkeypatch):
    from paper_2607_19893_amd import gsmi

    seen = []
    monkeypatch.setattr(gsmi, "current_stream", lambda: None)
    monkeypatch.setattr(gsmi._lib, "gs_gated_silu_bwd", lambda a, s: seen.append(1) or 0, raising=False)
    x = torch.zeros(5, 64)
    for q in (torch.uint8, torch.int8, torch.float8_e4m3fn):
        for s in (torch.uint8, torch.float8_e8m0fnu):
            gsmi.gs_gated_silu_bwd(x, torch.zeros(5, 64, dtype=torch.uint8).view(q), torch.zeros(5, 2, dtype=torch.uint8).view(s), x)
    assert len(seen) == 6


PAST = 2 ** 32 + 5                                     # 5 in its low 32 bits


@pytest.mark.parametrize("what", ["rms norm", "rotary", "layer", "layer gradient", "lookup", "lookup's table", "touched rows",
                                  "table's gradient", "recurrence", "segments", "silu", "silu gradient"])
def test_sizes_past_32_bits_are_refused(what):
    """By the binding: the library would see their low bits and leave the other rows as they were."""
    from paper_2607_19893_amd import gsmi

    far = torch.empty(PAST, 1, device="meta", dtype=torch.bfloat16)
    one, x, w = torch.zeros(1, 1, dtype=torch.bfloat16), torch.zeros(5, 1, dtype=torch.bfloat16), torch.zeros(1)
    ids, q, s = torch.zeros(5, dtype=torch.int32), far.to(torch.uint8), far.to(torch.uint8)
    calls = {
        "rms norm": lambda: gsmi.gs_rms_norm(far, w, 1e-5, y=far),
        "rotary": lambda: gsmi.make_rows(far.unsqueeze(1)),
        "layer": lambda: gsmi.gs_layer_norm(far, w, None, 1e-5, y=far),
        "layer gradient": lambda: gsmi.gs_layer_norm_bwd(far, far, w, 1e-5, far, w, w, None),
        "lookup": lambda: gsmi.gs_embedding(one, torch.empty(PAST, dtype=torch.int32, device="meta"), 1.0, far),
        "lookup's table": lambda: gsmi.gs_embedding(far, ids, 1.0, x),
        "touched rows": lambda: gsmi.gs_embedding_bwd(x, ids, PAST, 1.0, x.float(), None, ids, ids[:1]),
        "table's gradient": lambda: gsmi.gs_embedding_bwd(x, ids, PAST, 1.0, far.float(), None),
        "recurrence": lambda: gsmi.make_recur(far, far),
        "segments": lambda: gsmi.make_recur(x, x, n_seg=PAST),
        "silu": lambda: gsmi.gs_gated_silu(far, None, far),
        "silu gradient": lambda: gsmi.gs_gated_silu_bwd(far, q, s, far),
    }
    with pytest.raises(ValueError, match="2.31 - 1"):
        calls[what]()
