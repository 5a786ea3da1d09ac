"""Thin ctypes binding of libgsmi (include/gsmi.h): same names, argument
marshalling only.  Tensors are torch tensors on the GPU; their data pointers
and the current HIP stream are handed to the C ABI unchanged.

Importing this module loads the in-tree libgsmi.so and fails loudly if it is
missing; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgsmi.so")

if not os.path.exists(LIB_PATH):
    raise ImportError("libgsmi.so is not built (run __graft_entry__.build() or "
                      "python -m paper_2607_19893_amd.build); there is no fallback path")

_lib = ctypes.CDLL(LIB_PATH)

P = ctypes.c_void_p
i32, u32, i64, f32, sz = ctypes.c_int32, ctypes.c_uint32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t

GS_OK, GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED, GS_ERR_WORKSPACE, GS_ERR_HIP = range(5)
GS_WS_VISIBLE_SET, GS_WS_BIN_SORT, GS_WS_RASTER_BWD, GS_WS_LOSS, GS_WS_SCOPE, GS_WS_RASTER_FWD_L1 = 1, 2, 3, 4, 5, 6
GS_PRED_U32_NONZERO, GS_PRED_U8_NONZERO, GS_PRED_BITMAP, GS_PRED_U8_NONZERO_CLEAR = 0, 1, 2, 3
(GS_GATE_NO_DELAY, GS_GATE_ADMIT, GS_GATE_WAIT_RHO, GS_GATE_WAIT_NO_ACTIVE, GS_GATE_WAIT_MISSING, GS_GATE_WAIT_SECOND,
 GS_GATE_WAIT_GRADIENT) = range(7)
GS_APPLY_ADD, GS_APPLY_OVERWRITE = 0, 1
GS_DEV_PAIR_OVERFLOW, GS_DEV_MSG_OVERFLOW, GS_DEV_MSG_MISMATCH, GS_DEV_MSG_ORDER = 1, 2, 4, 8
GS_MSG_MAGIC = 0x47534D31
GS_F32, GS_BF16, GS_F16 = 0, 1, 2
GS_ROPE_PLAIN, GS_ROPE_LINEAR, GS_ROPE_BASE, GS_ROPE_PARTS = 0, 1, 2, 3
GS_ATTN_FILL = 256
GS_NORM_BLOCK, GS_NORM_MAX_COLS, GS_ROTARY_MAX_DIM, GS_ATTN_MAX_DIM = 128, 16384, 512, 128
GS_EMBED_MAX_DIM, GS_EMBED_MAX_TOKENS, GS_RECUR_KEEP = 16384, 1 << 28, 64
GS_KEEP_BLOCK, GS_SILU_MAX_COLS = 32, 1 << 22
GS_MAX_GROUPS = 8


class gs_scene(ctypes.Structure):
    _fields_ = [("n", i32), ("sh_degree", i32), ("mean", P), ("log_scale", P), ("quat", P), ("opacity", P),
                ("sh", P), ("ld_mean", i32), ("ld_log_scale", i32), ("ld_quat", i32), ("ld_opacity", i32),
                ("ld_sh", i32)]


class gs_camera(ctypes.Structure):
    _fields_ = [("width", i32), ("height", i32), ("fx", f32), ("fy", f32), ("cx", f32), ("cy", f32),
                ("tan_fovx", f32), ("tan_fovy", f32), ("near_z", f32), ("R", f32 * 9), ("t", f32 * 3),
                ("campos", f32 * 3)]


class gs_proj(ctypes.Structure):
    _fields_ = [("radius", P), ("tiles", P), ("rect", P), ("depth", P), ("mean2d", P), ("conic_opacity", P),
                ("rgb", P), ("clamp", P)]


class gs_adam_group(ctypes.Structure):
    _fields_ = [("p", P), ("cols", i32), ("lr", f32), ("ld", i32)]


class gs_group(ctypes.Structure):
    _fields_ = [("ptr", P), ("cols", i32), ("ld", i32)]


class gs_ring(ctypes.Structure):
    _fields_ = [("slot", P * 2), ("slot_bytes", sz), ("state", P), ("background", i32)]


class gs_gate_args(ctypes.Structure):
    _fields_ = [("active", P), ("evidence", P), ("g", P), ("skip", P), ("producer_version", u32),
                ("tau", ctypes.c_double)]


class gs_gate_result(ctypes.Structure):
    """Mirror of the device-side result record (64 bytes)."""
    _fields_ = [("admit", u32), ("reason", u32), ("n_read", u32), ("n_delayed", u32), ("n_active", u32),
                ("n_missing", u32), ("n_second", u32), ("reserved", u32), ("rho", ctypes.c_double),
                ("mean_g", ctypes.c_double), ("max_g", ctypes.c_double), ("threshold", ctypes.c_double)]


class gs_rows(ctypes.Structure):
    _fields_ = [("ptr", P), ("ld_row", i64), ("ld_head", i64)]


class gs_norm_args(ctypes.Structure):
    _fields_ = [("rows", i32), ("cols", i32), ("dtype", i32), ("eps", f32), ("x", P), ("residual", P), ("weight", P),
                ("total", P), ("y", P), ("q", P), ("q_scale", P), ("ld_x", i64), ("ld_residual", i64),
                ("ld_total", i64), ("ld_y", i64), ("ld_q", i64), ("ld_scale", i64)]


class gs_norm_bwd_args(ctypes.Structure):
    _fields_ = [("rows", i32), ("cols", i32), ("dtype", i32), ("eps", f32), ("dy", P), ("total", P), ("dtotal", P),
                ("weight", P), ("dx", P), ("dweight", P), ("ld_dy", i64), ("ld_total", i64), ("ld_dtotal", i64),
                ("ld_dx", i64)]


class gs_rotary_args(ctypes.Structure):
    _fields_ = [("dtype", i32), ("tokens", i32), ("dim", i32), ("pairs", i32), ("n_axes", i32), ("axis_pairs", i32 * 3),
                ("interleaved", i32), ("inverse", i32), ("amplitude", f32), ("pos", P), ("ld_pos", i64), ("freq", P),
                ("n_tensors", i32), ("heads", i32 * 2), ("inp", gs_rows * 2), ("out", gs_rows * 2)]


class gs_attn(ctypes.Structure):
    _fields_ = [("dtype", i32), ("n_q", i32), ("n_k", i32), ("n_seg", i32), ("heads", i32), ("kv_heads", i32),
                ("dim", i32), ("left", i32), ("right", i32), ("scale", f32), ("cu_q", P), ("cu_k", P), ("key_on", P),
                ("q", gs_rows), ("k", gs_rows), ("v", gs_rows)]


class gs_attn_grads(ctypes.Structure):
    _fields_ = [("out", gs_rows), ("dout", gs_rows), ("dq", gs_rows), ("dk", gs_rows), ("dv", gs_rows), ("lse", P)]


class gs_layer_args(ctypes.Structure):
    _fields_ = [("rows", i32), ("cols", i32), ("dtype", i32), ("eps", f32), ("x", P), ("residual", P), ("weight", P),
                ("bias", P), ("total", P), ("y", P), ("ld_x", i64), ("ld_residual", i64), ("ld_total", i64),
                ("ld_y", i64)]


class gs_layer_bwd_args(ctypes.Structure):
    _fields_ = [("rows", i32), ("cols", i32), ("dtype", i32), ("eps", f32), ("dy", P), ("total", P), ("dtotal", P),
                ("weight", P), ("dx", P), ("dweight", P), ("dbias", P), ("ld_dy", i64), ("ld_total", i64),
                ("ld_dtotal", i64), ("ld_dx", i64)]


class gs_embed_args(ctypes.Structure):
    _fields_ = [("dtype", i32), ("table_dtype", i32), ("tokens", i32), ("rows", i32), ("dim", i32), ("scale", f32),
                ("ids", P), ("table", P), ("out", P), ("ld_table", i64), ("ld_out", i64)]


class gs_embed_bwd_args(ctypes.Structure):
    _fields_ = [("dtype", i32), ("tokens", i32), ("rows", i32), ("dim", i32), ("scale", f32), ("ids", P), ("dout", P),
                ("grad", P), ("unique", P), ("count", P), ("ld_dout", i64), ("ld_grad", i64)]


class gs_recur(ctypes.Structure):
    _fields_ = [("dtype", i32), ("n", i32), ("cols", i32), ("n_seg", i32), ("reverse", i32), ("fill", i32), ("cu", P),
                ("x", P), ("gate", P), ("initial", P), ("ld_x", i64), ("ld_gate", i64)]


class gs_recur_grads(ctypes.Structure):
    _fields_ = [("dy", P), ("dfinal", P), ("kept", P), ("dx", P), ("dgate", P), ("dinitial", P), ("ld_dy", i64),
                ("ld_dx", i64), ("ld_dgate", i64)]


class gs_silu_args(ctypes.Structure):
    _fields_ = [("rows", i32), ("cols", i32), ("dtype", i32), ("u", P), ("v", P), ("h", P), ("u8", P), ("u_scale", P),
                ("v8", P), ("v_scale", P), ("ld_u", i64), ("ld_v", i64), ("ld_h", i64), ("ld_u8", i64),
                ("ld_u_scale", i64), ("ld_v8", i64), ("ld_v_scale", i64)]


class gs_silu_bwd_args(ctypes.Structure):
    _fields_ = [("rows", i32), ("cols", i32), ("dtype", i32), ("dh", P), ("u8", P), ("u_scale", P), ("v8", P),
                ("v_scale", P), ("du", P), ("dv", P), ("h", P), ("ld_dh", i64), ("ld_u8", i64), ("ld_u_scale", i64),
                ("ld_v8", i64), ("ld_v_scale", i64), ("ld_du", i64), ("ld_dv", i64), ("ld_h", i64)]


def scope_words(n) -> int:
    return (int(n) + 31) // 32


_lib.gs_abi_version.restype = i32
# the structs above mirror this version of the header; a library built from
# another one would read them with a different layout
ABI_VERSION = 4
if _lib.gs_abi_version() != ABI_VERSION:
    raise ImportError("libgsmi ABI version %d, binding expects %d: rebuild the library"
                      % (_lib.gs_abi_version(), ABI_VERSION))
_lib.gs_status_string.restype = ctypes.c_char_p
_lib.gs_status_string.argtypes = [i32]
_lib.gs_last_error.restype = ctypes.c_char_p
_lib.gs_workspace_bytes.restype = sz
_lib.gs_workspace_bytes.argtypes = [i32, i32, u32, i32, i32]
_lib.gs_delta_msg_bytes.restype = sz
_lib.gs_delta_msg_bytes.argtypes = [u32, i32, i32]
_lib.gs_project.argtypes = [ctypes.POINTER(gs_scene), ctypes.POINTER(gs_camera), ctypes.POINTER(gs_proj), P]
_lib.gs_visible_set.argtypes = [i32, P, i32, P, P, P, sz, P]
_lib.gs_visible_set_noalloc.argtypes = [i32, P, i32, P, P, P]
_lib.gs_bin_sort.argtypes = [ctypes.POINTER(gs_proj), i32, P, P, i32, i32, u32, P, P, P, P, P, P, P, P, P, sz, P]
_lib.gs_raster_fwd.argtypes = [ctypes.POINTER(gs_proj), i32, P, P, P, i32, i32, P, P, P, P, P, P, P]
_lib.gs_loss_l1.argtypes = [P, P, i32, i32, P, P, P, sz, P]
_lib.gs_raster_fwd_l1.argtypes = [ctypes.POINTER(gs_proj), i32, P, P, P, i32, i32, P, P, P, P, P, P, P, P, P, sz, P]
_lib.gs_raster_bwd.argtypes = [ctypes.POINTER(gs_scene), ctypes.POINTER(gs_camera), ctypes.POINTER(gs_proj), P, P, P,
                               P, P, P, P, u32, P, P, P, P, P, i32, P, P, P, sz, P]
_lib.gs_raster_bwd_pixels.argtypes = [ctypes.POINTER(gs_proj), ctypes.POINTER(gs_camera), P, P, P, P, u32, P, P, P,
                                      P, P, sz, P]
_lib.gs_raster_bwd_project.argtypes = [ctypes.POINTER(gs_scene), ctypes.POINTER(gs_camera), ctypes.POINTER(gs_proj),
                                       P, P, P, u32, P, i32, P, P, P, sz, P]
_lib.gs_raster_bwd_project_accum.argtypes = [ctypes.POINTER(gs_scene), ctypes.POINTER(gs_camera),
                                             ctypes.POINTER(gs_proj), P, P, P, u32, P, P, i32, P, i32, P, P, sz, P]
_lib.gs_sparse_adam.argtypes = [ctypes.POINTER(gs_adam_group), i32, P, P, i32, P, i32, P, P, i32, i32,
                                ctypes.c_double, ctypes.c_double, ctypes.c_double, P, i32, P]
_lib.gs_sparse_adam_publish.argtypes = [ctypes.POINTER(gs_adam_group), i32, P, P, i32, P, i32, P, P, i32, i32,
                                        ctypes.c_double, ctypes.c_double, ctypes.c_double, u32, P, sz, P, P]
_lib.gs_delta_pack.argtypes = [P, P, i32, ctypes.POINTER(gs_group), i32, u32, P, sz, P, P]
_lib.gs_delta_apply.argtypes = [P, sz, ctypes.POINTER(gs_group), i32, i32, i32, i32, P, P, P]
_lib.gs_publish_commit.argtypes = [ctypes.POINTER(gs_ring), u32, ctypes.POINTER(gs_group), i32, i32, i32, i32, P, P,
                                   P, P]
_lib.gs_scope_from_ids.argtypes = [P, P, i32, i32, i32, P, P]
_lib.gs_scope_from_pred.argtypes = [i32, P, i32, i32, P, P]
_lib.gs_scope_conflicts.argtypes = [P, P, P, P, i32, P, P, P, P, P, P, P, P, sz, P]
_lib.gs_admission_gate.argtypes = [P, P, ctypes.POINTER(gs_gate_args), i32, P, P, sz, P]
_lib.gs_rms_norm.argtypes = [ctypes.POINTER(gs_norm_args), P]
_lib.gs_rms_norm_bwd_ws_bytes.restype = sz
_lib.gs_rms_norm_bwd_ws_bytes.argtypes = [i32, i32]
_lib.gs_rms_norm_bwd.argtypes = [ctypes.POINTER(gs_norm_bwd_args), P, sz, P]
_lib.gs_rotary.argtypes = [ctypes.POINTER(gs_rotary_args), P]
_lib.gs_rotary_freqs.argtypes = [i32, ctypes.c_double, i32, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                 ctypes.c_double, P, P]
_lib.gs_attention_ws_bytes.restype = sz
_lib.gs_attention_ws_bytes.argtypes = [ctypes.POINTER(gs_attn), i32]
_lib.gs_attention.argtypes = [ctypes.POINTER(gs_attn), ctypes.POINTER(gs_rows), P, P, sz, P]
_lib.gs_attention_bwd.argtypes = [ctypes.POINTER(gs_attn), ctypes.POINTER(gs_attn_grads), P, sz, P]
_lib.gs_layer_norm.argtypes = [ctypes.POINTER(gs_layer_args), P]
_lib.gs_layer_norm_bwd_ws_bytes.restype = sz
_lib.gs_layer_norm_bwd_ws_bytes.argtypes = [i32, i32]
_lib.gs_layer_norm_bwd.argtypes = [ctypes.POINTER(gs_layer_bwd_args), P, sz, P]
_lib.gs_embedding.argtypes = [ctypes.POINTER(gs_embed_args), P]
_lib.gs_embedding_bwd_ws_bytes.restype = sz
_lib.gs_embedding_bwd_ws_bytes.argtypes = [i32, i32, i32, i32]
_lib.gs_embedding_bwd.argtypes = [ctypes.POINTER(gs_embed_bwd_args), P, sz, P]
_lib.gs_recurrence_ws_bytes.restype = sz
_lib.gs_recurrence_ws_bytes.argtypes = [ctypes.POINTER(gs_recur)]
_lib.gs_recurrence.argtypes = [ctypes.POINTER(gs_recur), P, i64, P, P, P, sz, P]
_lib.gs_recurrence_bwd.argtypes = [ctypes.POINTER(gs_recur), ctypes.POINTER(gs_recur_grads), P, sz, P]
_lib.gs_gated_silu.argtypes = [ctypes.POINTER(gs_silu_args), P]
_lib.gs_gated_silu_bwd.argtypes = [ctypes.POINTER(gs_silu_bwd_args), P]
_lib.gs_rlg_build.argtypes = [i32, i32, P, P, i32, i32, P, P, P, ctypes.c_int64, P]
_lib.gs_lp_partition.argtypes = [i32, P, P, P, P, i32, i32, P, P, P]
_lib.gs_sds_order.argtypes = [i32, P, i32, P, P, P, P, i32, P, P, P, P, P, P]
for _name in ("gs_project", "gs_visible_set", "gs_visible_set_noalloc", "gs_bin_sort", "gs_raster_fwd", "gs_loss_l1", "gs_raster_bwd",
              "gs_raster_bwd_pixels", "gs_raster_bwd_project", "gs_sparse_adam", "gs_sparse_adam_publish",
              "gs_delta_pack", "gs_delta_apply", "gs_scope_from_ids", "gs_scope_from_pred", "gs_scope_conflicts",
              "gs_admission_gate", "gs_publish_commit", "gs_raster_bwd_project_accum", "gs_raster_fwd_l1",
              "gs_rlg_build", "gs_lp_partition", "gs_sds_order", "gs_rms_norm", "gs_rms_norm_bwd", "gs_rotary",
              "gs_rotary_freqs", "gs_attention", "gs_attention_bwd", "gs_layer_norm", "gs_layer_norm_bwd",
              "gs_embedding", "gs_embedding_bwd", "gs_recurrence", "gs_recurrence_bwd", "gs_gated_silu",
              "gs_gated_silu_bwd"):
    getattr(_lib, _name).restype = i32

EXPORTS = ["gs_abi_version", "gs_status_string", "gs_last_error", "gs_workspace_bytes", "gs_delta_msg_bytes",
           "gs_project", "gs_visible_set", "gs_visible_set_noalloc", "gs_bin_sort", "gs_raster_fwd", "gs_loss_l1",
           "gs_raster_bwd", "gs_raster_bwd_pixels", "gs_raster_bwd_project", "gs_sparse_adam", "gs_sparse_adam_publish",
           "gs_delta_pack", "gs_delta_apply", "gs_scope_from_ids", "gs_scope_from_pred", "gs_scope_conflicts",
           "gs_admission_gate", "gs_publish_commit", "gs_raster_bwd_project_accum", "gs_raster_fwd_l1",
           "gs_rlg_build", "gs_lp_partition", "gs_sds_order", "gs_rms_norm", "gs_rms_norm_bwd_ws_bytes",
           "gs_rms_norm_bwd", "gs_rotary", "gs_rotary_freqs", "gs_attention_ws_bytes", "gs_attention",
           "gs_attention_bwd", "gs_layer_norm", "gs_layer_norm_bwd_ws_bytes", "gs_layer_norm_bwd", "gs_embedding",
           "gs_embedding_bwd_ws_bytes", "gs_embedding_bwd", "gs_recurrence_ws_bytes", "gs_recurrence",
           "gs_recurrence_bwd", "gs_gated_silu", "gs_gated_silu_bwd"]


class GsmiError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        msg = _lib.gs_last_error().decode()
        super().__init__("%s -> %s: %s" % (fn, _lib.gs_status_string(status).decode(), msg))


def _check(fn, st):
    if st != GS_OK:
        raise GsmiError(fn, st)
    return st


def ptr(t):
    """Device pointer of a tensor (or None)."""
    if t is None:
        return None
    return ctypes.c_void_p(t.data_ptr())


_raw_stream = None


def current_stream():
    """The current HIP stream of torch's current device, as an address."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()                # torch sets the GPU up
        # torch's own short way to the address (an object per call costs 3 us)
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and device is not None:
            _raw_stream = lambda: raw(device())
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream
    return ctypes.c_void_p(_raw_stream())


def make_camera(cam) -> gs_camera:
    c = gs_camera()
    c.width, c.height = int(cam.width), int(cam.height)
    for k in ("fx", "fy", "cx", "cy", "tan_fovx", "tan_fovy", "near_z"):
        setattr(c, k, float(getattr(cam, k)))
    R = [float(x) for x in cam.R.reshape(9)]
    for i in range(9):
        c.R[i] = R[i]
    for i in range(3):
        c.t[i] = float(cam.t[i])
        c.campos[i] = float(cam.campos[i])
    return c


def row_stride(t) -> int:
    """Floats between consecutive rows of a parameter group: the first-dim
    stride of a tensor whose rows are contiguous (a dense tensor or a column
    range of a wider table)."""
    if t is None or t.numel() == 0:
        return 0
    per_row = t[0].numel() if t.dim() > 1 else 1
    if t.dim() > 1 and not t[0].is_contiguous():
        raise ValueError("rows of a parameter group must be contiguous")
    return int(t.stride(0)) if t.shape[0] > 1 else per_row


def make_scene(n, sh_degree, mean, log_scale, quat, opacity, sh) -> gs_scene:
    return gs_scene(int(n), int(sh_degree), ptr(mean), ptr(log_scale), ptr(quat), ptr(opacity), ptr(sh),
                    row_stride(mean), row_stride(log_scale), row_stride(quat), row_stride(opacity), row_stride(sh))


def make_proj(radius, tiles, rect, depth, mean2d, conic_opacity, rgb, clamp) -> gs_proj:
    return gs_proj(ptr(radius), ptr(tiles), ptr(rect), ptr(depth), ptr(mean2d), ptr(conic_opacity), ptr(rgb),
                   ptr(clamp))


# ---- the entry points -------------------------------------------------------

def gs_abi_version() -> int:
    return int(_lib.gs_abi_version())


def gs_status_string(s: int) -> str:
    return _lib.gs_status_string(int(s)).decode()


def gs_last_error() -> str:
    return _lib.gs_last_error().decode()


def gs_workspace_bytes(which, n, capacity=0, width=0, height=0) -> int:
    return int(_lib.gs_workspace_bytes(int(which), int(n), int(capacity), int(width), int(height)))


def gs_delta_msg_bytes(count, row_len, n_groups) -> int:
    return int(_lib.gs_delta_msg_bytes(int(count), int(row_len), int(n_groups)))


def gs_project(scene: gs_scene, cam: gs_camera, proj: gs_proj, stream=None):
    return _check("gs_project", _lib.gs_project(ctypes.byref(scene), ctypes.byref(cam), ctypes.byref(proj),
                                                stream if stream is not None else current_stream()))


def gs_visible_set(kind, src, n, out_idx, out_count, ws, stream=None):
    return _check("gs_visible_set", _lib.gs_visible_set(int(kind), ptr(src), int(n), ptr(out_idx), ptr(out_count),
                                                        ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0,
                                                        stream if stream is not None else current_stream()))


def gs_visible_set_noalloc(kind, src, n, out_idx, out_count, stream=None):
    return _check("gs_visible_set_noalloc",
                  _lib.gs_visible_set_noalloc(int(kind), ptr(src), int(n), ptr(out_idx), ptr(out_count),
                                              stream if stream is not None else current_stream()))


GS_NOALLOC_SCRATCH_BYTES = 262144
GS_NOALLOC_MAX_N = 134215680


def gs_bin_sort(proj: gs_proj, n, vis_idx, vis_count, width, height, capacity, vals, ranges, pair_offset,
                pair_emit, keys, num_pairs, status, ws, stream=None, tile_order=None):
    return _check("gs_bin_sort", _lib.gs_bin_sort(ctypes.byref(proj), int(n), ptr(vis_idx), ptr(vis_count),
                                                  int(width), int(height), int(capacity), ptr(vals), ptr(ranges),
                                                  ptr(tile_order), ptr(pair_offset), ptr(pair_emit), ptr(keys),
                                                  ptr(num_pairs), ptr(status), ptr(ws),
                                                  ws.numel() * ws.element_size(),
                                                  stream if stream is not None else current_stream()))


def _bg(bg):
    arr = (ctypes.c_float * 3)(*[float(x) for x in bg])
    return arr


def gs_raster_fwd(proj: gs_proj, n, vals, ranges, width, height, bg, img, final_T, n_contrib, active=None,
                  pair_stats=None, stream=None, tile_order=None):
    b = _bg(bg)
    return _check("gs_raster_fwd", _lib.gs_raster_fwd(ctypes.byref(proj), int(n), ptr(vals), ptr(ranges),
                                                      ptr(tile_order), int(width), int(height), ctypes.cast(b, P),
                                                      ptr(img), ptr(final_T), ptr(n_contrib), ptr(active),
                                                      ptr(pair_stats),
                                                      stream if stream is not None else current_stream()))


def gs_raster_fwd_l1(proj: gs_proj, n, vals, ranges, width, height, bg, target, img, final_T, n_contrib, active, loss,
                     dL_dimg, ws, stream=None, tile_order=None):
    b = _bg(bg)
    return _check("gs_raster_fwd_l1", _lib.gs_raster_fwd_l1(
        ctypes.byref(proj), int(n), ptr(vals), ptr(ranges), ptr(tile_order), int(width), int(height),
        ctypes.cast(b, P), ptr(target), ptr(img), ptr(final_T), ptr(n_contrib), ptr(active), ptr(loss),
        ptr(dL_dimg), ptr(ws),
        ws.numel() * ws.element_size(), stream if stream is not None else current_stream()))


def gs_loss_l1(img, target, width, height, loss, dL_dimg, ws, stream=None):
    return _check("gs_loss_l1", _lib.gs_loss_l1(ptr(img), ptr(target), int(width), int(height), ptr(loss),
                                                ptr(dL_dimg), ptr(ws), ws.numel() * ws.element_size(),
                                                stream if stream is not None else current_stream()))


def gs_raster_bwd(scene: gs_scene, cam: gs_camera, proj: gs_proj, vals, ranges, pair_offset, pair_emit, vis_idx,
                  vis_count, capacity, final_T, n_contrib, dL_dimg, bg, grad_rows, grad_ld, grad2d, grad_norm, ws,
                  stream=None, tile_order=None):
    b = _bg(bg)
    return _check("gs_raster_bwd", _lib.gs_raster_bwd(ctypes.byref(scene), ctypes.byref(cam), ctypes.byref(proj),
                                                      ptr(vals), ptr(ranges), ptr(tile_order), ptr(pair_offset),
                                                      ptr(pair_emit), ptr(vis_idx), ptr(vis_count), int(capacity),
                                                      ptr(final_T),
                                                      ptr(n_contrib), ptr(dL_dimg), ctypes.cast(b, P),
                                                      ptr(grad_rows), int(grad_ld), ptr(grad2d), ptr(grad_norm),
                                                      ptr(ws), ws.numel() * ws.element_size(),
                                                      stream if stream is not None else current_stream()))


def gs_raster_bwd_pixels(proj: gs_proj, cam: gs_camera, vals, ranges, pair_emit, capacity, final_T, n_contrib, dL_dimg,
                         bg, ws, stream=None, tile_order=None):
    b = _bg(bg)
    return _check("gs_raster_bwd_pixels", _lib.gs_raster_bwd_pixels(
        ctypes.byref(proj), ctypes.byref(cam), ptr(vals), ptr(ranges), ptr(tile_order), ptr(pair_emit), int(capacity),
        ptr(final_T), ptr(n_contrib), ptr(dL_dimg), ctypes.cast(b, P), ptr(ws), ws.numel() * ws.element_size(),
        stream if stream is not None else current_stream()))


def gs_raster_bwd_project(scene: gs_scene, cam: gs_camera, proj: gs_proj, pair_offset, vis_idx, vis_count,
                          capacity, grad_rows, grad_ld, grad2d, grad_norm, ws, stream=None):
    return _check("gs_raster_bwd_project", _lib.gs_raster_bwd_project(
        ctypes.byref(scene), ctypes.byref(cam), ctypes.byref(proj), ptr(pair_offset), ptr(vis_idx),
        ptr(vis_count), int(capacity), ptr(grad_rows), int(grad_ld), ptr(grad2d), ptr(grad_norm), ptr(ws),
        ws.numel() * ws.element_size(), stream if stream is not None else current_stream()))


def gs_raster_bwd_project_accum(scene: gs_scene, cam: gs_camera, proj: gs_proj, pair_offset, vis_idx, vis_count,
                                capacity, union_idx, union_count, first, grad_rows, grad_ld, grad_norm, ws, stream=None):
    return _check("gs_raster_bwd_project_accum", _lib.gs_raster_bwd_project_accum(
        ctypes.byref(scene), ctypes.byref(cam), ctypes.byref(proj), ptr(pair_offset), ptr(vis_idx), ptr(vis_count),
        int(capacity), ptr(union_idx), ptr(union_count), int(first), ptr(grad_rows), int(grad_ld), ptr(grad_norm),
        ptr(ws), ws.numel() * ws.element_size(), stream if stream is not None else current_stream()))


def make_adam_groups(groups):
    """groups: list of (p [n, cols] tensor, lr)."""
    arr = (gs_adam_group * len(groups))()
    for i, (p, lr) in enumerate(groups):
        arr[i] = gs_adam_group(ptr(p), int(p.shape[1]), float(lr), row_stride(p))
    return arr


def gs_sparse_adam(groups_arr, n_groups, idx, count, max_rows, grad_rows, grad_ld, m, v, state_ld, step, beta1,
                   beta2, eps, delta_rows=None, delta_ld=0, stream=None):
    return _check("gs_sparse_adam", _lib.gs_sparse_adam(
        groups_arr, int(n_groups), ptr(idx), ptr(count), int(max_rows), ptr(grad_rows), int(grad_ld), ptr(m), ptr(v),
        int(state_ld), int(step), float(beta1), float(beta2), float(eps), ptr(delta_rows), int(delta_ld),
        stream if stream is not None else current_stream()))


def gs_sparse_adam_publish(groups_arr, n_groups, idx, count, max_rows, grad_rows, grad_ld, m, v, state_ld, step,
                           beta1, beta2, eps, version, msg, status, stream=None):
    return _check("gs_sparse_adam_publish", _lib.gs_sparse_adam_publish(
        groups_arr, int(n_groups), ptr(idx), ptr(count), int(max_rows), ptr(grad_rows), int(grad_ld), ptr(m), ptr(v),
        int(state_ld), int(step), float(beta1), float(beta2), float(eps), int(version), ptr(msg),
        msg.numel() * msg.element_size(), ptr(status), stream if stream is not None else current_stream()))


def make_groups(tensors):
    arr = (gs_group * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = gs_group(ptr(t), int(t.shape[1]), row_stride(t))
    return arr


def gs_delta_pack(idx, count, max_rows, groups_arr, n_groups, version, msg, status, stream=None):
    return _check("gs_delta_pack", _lib.gs_delta_pack(ptr(idx), ptr(count), int(max_rows), groups_arr, int(n_groups),
                                                      int(version), ptr(msg), msg.numel() * msg.element_size(),
                                                      ptr(status), stream if stream is not None else current_stream()))


def gs_delta_apply(msg, groups_arr, n_groups, n_rows, max_rows, mode, prim_version, status, stream=None):
    return _check("gs_delta_apply", _lib.gs_delta_apply(ptr(msg), msg.numel() * msg.element_size(), groups_arr,
                                                        int(n_groups), int(n_rows),
                                                        int(max_rows), int(mode), ptr(prim_version), ptr(status),
                                                        stream if stream is not None else current_stream()))


def make_ring(slots, state, background=False) -> gs_ring:
    """slots: two device tensors of equal byte size (slot v & 1 holds version v); state: >= 8 uint32 words;
    background: the commit runs beside compute on another stream (one workgroup per compute unit)."""
    nb = min(t.numel() * t.element_size() for t in slots)
    r = gs_ring()
    r.slot[0], r.slot[1] = slots[0].data_ptr(), slots[1].data_ptr()
    r.slot_bytes = nb
    r.state = state.data_ptr()
    r.background = 1 if background else 0
    return r


def gs_publish_commit(ring: gs_ring, version, groups_arr, n_groups, n_rows, max_rows, mode, prim_version, skip, status,
                      stream=None):
    return _check("gs_publish_commit", _lib.gs_publish_commit(
        ctypes.byref(ring), int(version), groups_arr, int(n_groups), int(n_rows), int(max_rows), int(mode),
        ptr(prim_version), ptr(skip), ptr(status), stream if stream is not None else current_stream()))


def gs_scope_from_ids(idx, count, max_rows, n, accumulate, scope, stream=None):
    return _check("gs_scope_from_ids", _lib.gs_scope_from_ids(ptr(idx), ptr(count), int(max_rows), int(n),
                                                              int(accumulate), ptr(scope),
                                                              stream if stream is not None else current_stream()))


def gs_scope_from_pred(kind, src, n, accumulate, scope, stream=None):
    return _check("gs_scope_from_pred", _lib.gs_scope_from_pred(int(kind), ptr(src), int(n), int(accumulate),
                                                                ptr(scope),
                                                                stream if stream is not None else current_stream()))


def gs_scope_conflicts(RA, WA, RB, WB, n, waw, raw_, war, waw_idx, raw_idx, war_idx, counts, ws, stream=None):
    return _check("gs_scope_conflicts", _lib.gs_scope_conflicts(
        ptr(RA), ptr(WA), ptr(RB), ptr(WB), int(n), ptr(waw), ptr(raw_), ptr(war), ptr(waw_idx), ptr(raw_idx),
        ptr(war_idx), ptr(counts), ptr(ws), ws.numel() * ws.element_size() if ws is not None else 0,
        stream if stream is not None else current_stream()))


def make_gate_args(active, g, tau, evidence=None, skip=None, producer_version=0) -> gs_gate_args:
    return gs_gate_args(ptr(active), ptr(evidence), ptr(g), ptr(skip), int(producer_version), float(tau))


def gs_admission_gate(RB, D, args: gs_gate_args, n, result, ws, stream=None):
    """result: a device tensor of >= 64 bytes (see gate_result_from)."""
    return _check("gs_admission_gate", _lib.gs_admission_gate(
        ptr(RB), ptr(D), ctypes.byref(args), int(n), ptr(result), ptr(ws),
        ws.numel() * ws.element_size() if ws is not None else 0,
        stream if stream is not None else current_stream()))


def gate_result_from(buf) -> gs_gate_result:
    """Decode a result record copied to the host (bytes-like or a tensor)."""
    if hasattr(buf, "cpu"):
        buf = buf.detach().cpu().numpy().tobytes()
    return gs_gate_result.from_buffer_copy(bytes(buf)[:ctypes.sizeof(gs_gate_result)])


# ---- token operators ----------------------------------------------------------

def _ws(ws):
    return (ws.data_ptr(), ws.numel() * ws.element_size()) if ws is not None else (None, 0)


_TOKEN_TYPES = {}


def token_dtype(t) -> int:
    if not _TOKEN_TYPES:
        import torch
        _TOKEN_TYPES.update({torch.float32: GS_F32, torch.bfloat16: GS_BF16, torch.float16: GS_F16})
    d = _TOKEN_TYPES.get(t.dtype)
    if d is None:
        raise ValueError("tokens are float32, bfloat16 or float16, not %s" % t.dtype)
    return d


def _at(t):
    return None if t is None else t.data_ptr()


def _count(n, what):
    """A size that the library takes in 32 bits (ctypes would cut a larger one down to its low bits)."""
    if not 0 <= n <= 0x7FFFFFFF:
        raise ValueError("%s: %d is not between 0 and 2^31 - 1" % (what, n))
    return n


def make_rows(t) -> gs_rows:
    """A [rows, heads, dim] tensor whose heads' elements are contiguous."""
    st = t.stride()
    _count(t.shape[0], "rows")
    if len(st) != 3 or (st[2] != 1 and t.shape[2] > 1):
        raise ValueError("a token matrix is [rows, heads, dim] with contiguous elements, not %s with strides %s"
                         % (tuple(t.shape), st))
    return gs_rows(t.data_ptr(), st[0], st[1])


def _ld(t, shape, what, dtype=None):
    """Row stride of a tensor of that shape with contiguous rows (0 for None)."""
    if t is None:
        return 0
    st = t.stride()
    if t.shape != shape or (st[1] != 1 and shape[1] > 1):
        raise ValueError("%s is %s with contiguous rows, not %s with strides %s" % (what, list(shape), list(t.shape), st))
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s is %s, not %s" % (what, dtype, t.dtype))
    if (shape[0] | shape[1]) >> 31:
        raise ValueError("%s: %s is past 2^31 - 1" % (what, list(shape)))
    return st[0] if shape[0] > 1 else max(shape[1], st[0])


def gs_rms_norm(x, weight, eps, y=None, residual=None, total=None, q=None, q_scale=None, stream=None):
    shape, dt = x.shape, x.dtype
    rows, cols = shape
    a = gs_norm_args(rows, cols, token_dtype(x), eps, x.data_ptr(), _at(residual), _at(weight), _at(total),
                     _at(y), _at(q), _at(q_scale), _ld(x, shape, "x"), _ld(residual, shape, "residual", dt),
                     _ld(total, shape, "total", dt), _ld(y, shape, "y", dt), _ld(q, shape, "q"),
                     _ld(q_scale, (rows, -(-cols // GS_NORM_BLOCK)), "q_scale"))
    return _check("gs_rms_norm", _lib.gs_rms_norm(ctypes.byref(a), stream if stream is not None else current_stream()))


def gs_rms_norm_bwd_ws_bytes(rows, cols) -> int:
    return int(_lib.gs_rms_norm_bwd_ws_bytes(int(rows), int(cols)))


def gs_rms_norm_bwd(dy, total, weight, eps, dx, dweight, ws, dtotal=None, stream=None):
    shape, dt = total.shape, total.dtype
    a = gs_norm_bwd_args(shape[0], shape[1], token_dtype(total), eps, dy.data_ptr(), total.data_ptr(), _at(dtotal),
                         _at(weight), dx.data_ptr(), _at(dweight), _ld(dy, shape, "dy", dt),
                         _ld(total, shape, "total"), _ld(dtotal, shape, "dtotal", dt), _ld(dx, shape, "dx", dt))
    p, n = _ws(ws)
    return _check("gs_rms_norm_bwd", _lib.gs_rms_norm_bwd(ctypes.byref(a), p, n,
                                                          stream if stream is not None else current_stream()))


_Axes, _Pair, _RowsPair = i32 * 3, i32 * 2, gs_rows * 2


def gs_rotary(inputs, outputs, pos, freq, axis_pairs, interleaved=False, inverse=False, amplitude=1.0, stream=None):
    """inputs, outputs: one or two [tokens, heads, dim] tensors each; pos [tokens, axes] fp32."""
    n = len(inputs)
    if not 1 <= n <= 2 or len(outputs) != n:
        raise ValueError("one or two tensors, with an output each")
    x = inputs[0]
    shape, dt = x.shape, x.dtype
    ps, axes = pos.stride(), len(axis_pairs)
    if pos.dim() != 2 or (axes > 1 and ps[1] != 1):
        raise ValueError("pos is [tokens, axes] with contiguous rows, not strides %s" % (ps,))
    for t, o in zip(inputs, outputs):
        ts = t.shape
        if ts != o.shape or t.dtype != dt or o.dtype != dt or ts[0] != shape[0] or ts[2] != shape[2]:
            raise ValueError("tensors and outputs share tokens, dim and type; got %s -> %s" % (ts, o.shape))
    a = gs_rotary_args(token_dtype(x), shape[0], shape[2], sum(axis_pairs), axes, _Axes(*axis_pairs[:3]),
                       interleaved, inverse, amplitude, pos.data_ptr(), ps[0] if shape[0] > 1 else max(axes, ps[0]),
                       freq.data_ptr(), n,
                       _Pair(*[t.shape[1] for t in inputs]), _RowsPair(*[make_rows(t) for t in inputs]),
                       _RowsPair(*[make_rows(o) for o in outputs]))
    return _check("gs_rotary", _lib.gs_rotary(ctypes.byref(a), stream if stream is not None else current_stream()))


def gs_rotary_freqs(pairs, base=10000.0, scaling=GS_ROPE_PLAIN, factor=1.0, trained=0.0, slow=1.0, fast=32.0):
    """Returns (freq [pairs] numpy float32, amplitude)."""
    import numpy as np
    freq = np.zeros(max(int(pairs), 1), np.float32)
    amp = ctypes.c_float(1.0)
    _check("gs_rotary_freqs", _lib.gs_rotary_freqs(int(pairs), float(base), int(scaling), float(factor), float(trained),
                                                   float(slow), float(fast), ctypes.c_void_p(freq.ctypes.data),
                                                   ctypes.byref(amp)))
    return freq[:int(pairs)], float(amp.value)


def make_attn(q, k, v, scale, n_seg=1, cu_q=None, cu_k=None, key_on=None, left=-1, right=-1,
              fill=False) -> gs_attn:
    """fill: rows outside every segment are written (zeros, log sums of -inf)."""
    qs, ks = q.shape, k.shape
    if ks != v.shape or ks[2] != qs[2] or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k, v do not fit: %s, %s, %s" % (qs, ks, v.shape))
    if cu_q is not None:
        n_seg = cu_q.numel() - 1
        if cu_k is None or cu_k.numel() != n_seg + 1 or cu_q.element_size() != 4 or cu_q.is_floating_point() \
                or cu_k.dtype != cu_q.dtype or not cu_q.is_contiguous() or not cu_k.is_contiguous():
            raise ValueError("cu_q and cu_k are contiguous int32 of the same length")
    _count(n_seg, "n_seg")
    if key_on is not None and (key_on.numel() != ks[0] or key_on.element_size() != 1 or not key_on.is_contiguous()):
        raise ValueError("key_on is one contiguous byte per key")
    return gs_attn(token_dtype(q) | (GS_ATTN_FILL if fill else 0), qs[0], ks[0], n_seg, qs[1], ks[1], qs[2], left, right, scale, _at(cu_q), _at(cu_k),
                   _at(key_on), make_rows(q), make_rows(k), make_rows(v))


def gs_attention_ws_bytes(attn: gs_attn, backward=False) -> int:
    return int(_lib.gs_attention_ws_bytes(ctypes.byref(attn), int(backward)))


def gs_attention(attn: gs_attn, out, lse, ws=None, stream=None):
    p, n = _ws(ws)
    return _check("gs_attention", _lib.gs_attention(ctypes.byref(attn), ctypes.byref(make_rows(out)), ptr(lse), p, n,
                                                    stream if stream is not None else current_stream()))


def gs_attention_bwd(attn: gs_attn, out, lse, dout, dq, dk, dv, ws, stream=None):
    g = gs_attn_grads(make_rows(out), make_rows(dout), make_rows(dq), make_rows(dk), make_rows(dv), lse.data_ptr())
    p, n = _ws(ws)
    return _check("gs_attention_bwd", _lib.gs_attention_bwd(ctypes.byref(attn), ctypes.byref(g), p, n,
                                                            stream if stream is not None else current_stream()))


def gs_layer_norm(x, weight, bias, eps, y=None, residual=None, total=None, stream=None):
    shape, dt = x.shape, x.dtype
    a = gs_layer_args(shape[0], shape[1], token_dtype(x), eps, x.data_ptr(), _at(residual), _at(weight), _at(bias),
                      _at(total), _at(y), _ld(x, shape, "x"), _ld(residual, shape, "residual", dt),
                      _ld(total, shape, "total", dt), _ld(y, shape, "y", dt))
    return _check("gs_layer_norm", _lib.gs_layer_norm(ctypes.byref(a), stream if stream is not None else current_stream()))


def gs_layer_norm_bwd_ws_bytes(rows, cols) -> int:
    return int(_lib.gs_layer_norm_bwd_ws_bytes(int(rows), int(cols)))


def gs_layer_norm_bwd(dy, total, weight, eps, dx, dweight, dbias, ws, dtotal=None, stream=None):
    shape, dt = total.shape, total.dtype
    a = gs_layer_bwd_args(shape[0], shape[1], token_dtype(total), eps, dy.data_ptr(), total.data_ptr(), _at(dtotal),
                          _at(weight), dx.data_ptr(), _at(dweight), _at(dbias), _ld(dy, shape, "dy", dt),
                          _ld(total, shape, "total"), _ld(dtotal, shape, "dtotal", dt), _ld(dx, shape, "dx", dt))
    p, n = _ws(ws)
    return _check("gs_layer_norm_bwd", _lib.gs_layer_norm_bwd(ctypes.byref(a), p, n,
                                                              stream if stream is not None else current_stream()))


def _int32(t, n, what):
    if t.numel() != n or t.element_size() != 4 or t.is_floating_point() or not t.is_contiguous():
        raise ValueError("%s is %d contiguous int32 values" % (what, n))


def gs_embedding(table, ids, scale, out, stream=None):
    """table [rows, dim], ids [tokens] int32, out [tokens, dim]."""
    _int32(ids, out.shape[0], "ids")
    a = gs_embed_args(token_dtype(out), token_dtype(table), out.shape[0], table.shape[0], out.shape[1], scale, _at(ids),
                      table.data_ptr(), out.data_ptr(), _ld(table, (table.shape[0], out.shape[1]), "table"),
                      _ld(out, out.shape, "out"))
    return _check("gs_embedding", _lib.gs_embedding(ctypes.byref(a), stream if stream is not None else current_stream()))


def gs_embedding_bwd_ws_bytes(tokens, rows, dim, touched=False) -> int:
    return int(_lib.gs_embedding_bwd_ws_bytes(int(tokens), int(rows), int(dim), int(touched)))


def gs_embedding_bwd(dout, ids, rows, scale, grad, ws, unique=None, count=None, stream=None):
    """grad [rows, dim] fp32, or with unique and count the touched rows [min(tokens, rows), dim]."""
    import torch
    tokens, dim = dout.shape
    _int32(ids, tokens, "ids")
    most = _count(rows, "rows")
    if unique is not None:
        most = min(tokens, rows)
        _int32(unique, most, "unique")
        _int32(count, 1, "count")
    a = gs_embed_bwd_args(token_dtype(dout), tokens, rows, dim, scale, _at(ids), dout.data_ptr(), grad.data_ptr(),
                          _at(unique), _at(count), _ld(dout, dout.shape, "dout"),
                          _ld(grad, (most, dim), "grad", torch.float32))
    p, n = _ws(ws)
    if unique is not None and most == 0:          # tensors without elements have no address
        a.unique = a.count
    return _check("gs_embedding_bwd", _lib.gs_embedding_bwd(ctypes.byref(a), p, n,
                                                            stream if stream is not None else current_stream()))


def _states(t, shape, what):
    import torch
    if t is not None and (t.shape != shape or t.dtype != torch.float32 or not t.is_contiguous()):
        raise ValueError("%s is contiguous float32 %s" % (what, list(shape)))


def make_recur(x, gate, cu=None, n_seg=1, initial=None, reverse=False, fill=False) -> gs_recur:
    """x, gate [n, cols]; cu [n_seg + 1] int32; initial [n_seg, cols] fp32.  fill: tokens outside every segment are
    written (zeros)."""
    shape = x.shape
    if cu is not None:
        n_seg = cu.numel() - 1
        _int32(cu, n_seg + 1, "cu")
    _count(n_seg, "n_seg")
    _states(initial, (n_seg, shape[1]), "initial")
    return gs_recur(token_dtype(x), shape[0], shape[1], n_seg, reverse, fill, _at(cu), x.data_ptr(), gate.data_ptr(),
                    _at(initial), _ld(x, shape, "x"), _ld(gate, shape, "gate", x.dtype))


def gs_recurrence_ws_bytes(recur: gs_recur) -> int:
    return int(_lib.gs_recurrence_ws_bytes(ctypes.byref(recur)))


def gs_recurrence(recur: gs_recur, y, final=None, kept=None, ws=None, stream=None):
    n, cols = y.shape
    if token_dtype(y) != recur.dtype:
        raise ValueError("y has x's type")
    _states(final, (recur.n_seg, cols), "final")
    _states(kept, (-(-n // GS_RECUR_KEEP), cols), "kept")
    p, nb = _ws(ws)
    return _check("gs_recurrence", _lib.gs_recurrence(ctypes.byref(recur), y.data_ptr(), _ld(y, (recur.n, recur.cols), "y"),
                                                      _at(final), _at(kept), p, nb,
                                                      stream if stream is not None else current_stream()))


def gs_recurrence_bwd(recur: gs_recur, dy, kept, dx, dgate, dfinal=None, dinitial=None, ws=None, stream=None):
    shape = (recur.n, recur.cols)
    states = (recur.n_seg, recur.cols)
    _states(kept, (-(-recur.n // GS_RECUR_KEEP), recur.cols), "kept")
    _states(dfinal, states, "dfinal")
    _states(dinitial, states, "dinitial")
    dt = dy.dtype
    if token_dtype(dy) != recur.dtype:
        raise ValueError("dy has x's type")
    g = gs_recur_grads(dy.data_ptr(), _at(dfinal), _at(kept), dx.data_ptr(), dgate.data_ptr(), _at(dinitial),
                       _ld(dy, shape, "dy"), _ld(dx, shape, "dx", dt), _ld(dgate, shape, "dgate", dt))
    p, n = _ws(ws)
    return _check("gs_recurrence_bwd", _lib.gs_recurrence_bwd(ctypes.byref(recur), ctypes.byref(g), p, n,
                                                              stream if stream is not None else current_stream()))


def _eight(t, kind):
    """Bytes, or torch's type of what they stand for: another type of 8 bits would be read as other numbers."""
    import torch
    return t.element_size() == 1 and (not t.is_floating_point() or t.dtype == getattr(torch, kind, None))


def _kept8(q, scale, shape, name):
    """(addresses and strides) of rows in 8 bits and their scale bytes."""
    if q is None:
        return None, None, 0, 0
    blocks = (shape[0], -(-shape[1] // GS_KEEP_BLOCK))
    if scale is None or not (_eight(q, "float8_e4m3fn") and _eight(scale, "float8_e8m0fnu")):
        raise ValueError("%s is float8_e4m3fn or its bytes, its scales are bytes" % name)
    return q.data_ptr(), scale.data_ptr(), _ld(q, shape, name), _ld(scale, blocks, name + "'s scale")


def gs_gated_silu(u, v=None, h=None, u8=None, u_scale=None, v8=None, v_scale=None, stream=None):
    shape, dt = u.shape, u.dtype
    up, us, ldu, ldus = _kept8(u8, u_scale, shape, "u8")
    vp, vs, ldv, ldvs = _kept8(v8, v_scale, shape, "v8")
    a = gs_silu_args(shape[0], shape[1], token_dtype(u), u.data_ptr(), _at(v), _at(h), up, us, vp, vs, _ld(u, shape, "u"),
                     _ld(v, shape, "v", dt), _ld(h, shape, "h", dt), ldu, ldus, ldv, ldvs)
    return _check("gs_gated_silu", _lib.gs_gated_silu(ctypes.byref(a), stream if stream is not None else current_stream()))


def gs_gated_silu_bwd(dh, u8, u_scale, du, v8=None, v_scale=None, dv=None, h=None, stream=None):
    shape, dt = dh.shape, dh.dtype
    up, us, ldu, ldus = _kept8(u8, u_scale, shape, "u8")
    vp, vs, ldv, ldvs = _kept8(v8, v_scale, shape, "v8")
    a = gs_silu_bwd_args(shape[0], shape[1], token_dtype(dh), dh.data_ptr(), up, us, vp, vs, du.data_ptr(), _at(dv),
                         _at(h), _ld(dh, shape, "dh"), ldu, ldus, ldv, ldvs, _ld(du, shape, "du", dt),
                         _ld(dv, shape, "dv", dt), _ld(h, shape, "h", dt))
    return _check("gs_gated_silu_bwd", _lib.gs_gated_silu_bwd(ctypes.byref(a),
                                                              stream if stream is not None else current_stream()))


def raw():
    """The loaded ctypes library (for tests of argument validation)."""
    return _lib


# ---- the ahead-of-time planner (host arrays) --------------------------------

def _np(a, dtype):
    """A C-contiguous numpy array of dtype and its pointer (kept alive by the caller)."""
    import numpy as np
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, ctypes.c_void_p(a.ctypes.data)


class PlanGraph:
    """The retained relative locality graph in CSR form (numpy arrays)."""

    def __init__(self, edge_ptr, edge_dst, edge_w):
        self.edge_ptr, self.edge_dst, self.edge_w = edge_ptr, edge_dst, edge_w

    def ptrs(self):
        return (ctypes.c_void_p(self.edge_ptr.ctypes.data), ctypes.c_void_p(self.edge_dst.ctypes.data),
                ctypes.c_void_p(self.edge_w.ctypes.data))


def gs_rlg_build(item_ptr, item_tracks, n_tracks, track_cap, top_k) -> PlanGraph:
    import numpy as np
    ip, ip_p = _np(item_ptr, np.int64)
    it, it_p = _np(item_tracks if len(item_tracks) else np.zeros(1, np.int32), np.int32)
    n = ip.size - 1
    cap = 2 * n * int(top_k) if top_k > 0 else 0
    for _ in range(2):
        eptr = np.zeros(n + 1, np.int64)
        edst = np.zeros(max(cap, 1), np.int32)
        ew = np.zeros(max(cap, 1), np.float64)
        ne = ctypes.c_int64(0)
        st = _lib.gs_rlg_build(int(n), int(n_tracks), ip_p, it_p, int(track_cap), int(top_k),
                               ctypes.c_void_p(eptr.ctypes.data), ctypes.c_void_p(edst.ctypes.data),
                               ctypes.c_void_p(ew.ctypes.data), int(cap), ctypes.byref(ne))
        if st == GS_ERR_WORKSPACE and cap < ne.value:
            cap = int(ne.value)
            continue
        _check("gs_rlg_build", st)
        return PlanGraph(eptr, edst[:ne.value].copy(), ew[:ne.value].copy())
    raise GsmiError("gs_rlg_build", GS_ERR_WORKSPACE)


def gs_lp_partition(position, graph: PlanGraph, K, max_iters):
    """Returns (group [n] int32, coupling [K, K] float64, rounds run)."""
    import numpy as np
    pos, pos_p = _np(np.asarray(position, np.float64).reshape(-1, 3), np.float64)
    n = pos.shape[0]
    group = np.zeros(max(n, 1), np.int32)
    coupling = np.zeros((K, K), np.float64)
    it = ctypes.c_int32(0)
    ep, ed, ew = graph.ptrs()
    _check("gs_lp_partition", _lib.gs_lp_partition(int(n), pos_p, ep, ed, ew, int(K), int(max_iters),
                                                   ctypes.c_void_p(group.ctypes.data),
                                                   ctypes.c_void_p(coupling.ctypes.data), ctypes.byref(it)))
    return group[:n], coupling, int(it.value)


def gs_sds_order(group, coupling, graph: PlanGraph, unit_size):
    """Returns (cycle, order, unit_group, transition) as numpy arrays."""
    import numpy as np
    g, g_p = _np(group, np.int32)
    K = int(np.asarray(coupling).shape[0])
    C, C_p = _np(coupling, np.float64)
    n = g.size
    units = -(-n // int(unit_size)) if n else 0
    cycle = np.zeros(K, np.int32)
    order = np.zeros(max(n, 1), np.int32)
    ug = np.zeros(max(units, 1), np.int32)
    tr = np.zeros(max(units, 1), np.float64)
    nc, nu = ctypes.c_int32(0), ctypes.c_int32(0)
    ep, ed, ew = graph.ptrs()
    _check("gs_sds_order", _lib.gs_sds_order(int(n), g_p, K, C_p, ep, ed, ew, int(unit_size),
                                             ctypes.c_void_p(cycle.ctypes.data), ctypes.byref(nc),
                                             ctypes.c_void_p(order.ctypes.data), ctypes.c_void_p(ug.ctypes.data),
                                             ctypes.c_void_p(tr.ctypes.data), ctypes.byref(nu)))
    assert nu.value == units
    return cycle[:nc.value], order[:n], ug[:units], tr[:units]
