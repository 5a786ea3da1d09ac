"""The token operators' entry points at the ends of what they accept (host calls, no GPU needed)."""
import ctypes

from test_tokens_abi import attn, gs, refused  # noqa: F401 (gs: a fixture)


def test_fill_flag(gs):
    """GS_ATTN_FILL goes with either 16-bit type and with no other number."""
    L, out = gs.raw(), gs.gs_rows(256, 128, 64)
    call = lambda dtype: L.gs_attention(ctypes.byref(attn(gs, dtype=dtype, n_q=0)), ctypes.byref(out), 256, 256, 1 << 30, None)
    assert call(gs.GS_BF16 | gs.GS_ATTN_FILL) == gs.GS_OK and call(gs.GS_F16 | gs.GS_ATTN_FILL) == gs.GS_OK
    for bad in (gs.GS_F32 | gs.GS_ATTN_FILL, gs.GS_ATTN_FILL | 3, gs.GS_BF16 | 512, gs.GS_BF16 | 2 * gs.GS_ATTN_FILL):
        refused(gs, call(bad), "dtype")


def test_gradient_of_narrow_windows_takes_no_parts(gs):
    """One row a segment that admits one of its 64 keys: most key tiles have nothing to do, and cutting them into parts
    would take 2 * 4 bytes an element of k for every part (275 GB for 2^20 segments whose keys are 8.6 GB)."""
    for segments in (1 << 10, 1 << 20):
        a = attn(gs, n_seg=segments, n_q=segments, n_k=64 * segments, heads=64, kv_heads=1, left=0, right=0)
        assert gs.gs_attention_ws_bytes(a, True) == segments * 64 * 8          # the rows' bases and deltas
