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
