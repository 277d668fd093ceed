"""Python binding of libtg.so (include/tg.h): argument marshalling only.

Every step of the path runs in the native library: packing in its host C++ code,
stitch and unstitch in its HIP kernels. PyTorch supplies device memory and the
stream. There is no fallback: if libtg.so is missing this module raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import numpy as np

# TG_LIBTG names another build of the same library (the host-sanitizer build, say).
LIB_PATH = os.environ.get("TG_LIBTG") or os.path.join(os.path.dirname(os.path.abspath(__file__)),
                                                      "libtg.so")

SHELF_FFDH, SHELF_ARRIVAL, GUILLOTINE_BSSF = 0, 1, 2
OK = 0
E_INVAL, E_ROI_TOO_LARGE, E_ROI_OOB, E_RANGE, E_WORKSPACE, E_HIP, E_INTERNAL = range(-1, -8, -1)

ROI_DTYPE = np.dtype([("frame", "<i4"), ("x", "<i4"), ("y", "<i4"), ("w", "<i4"), ("h", "<i4")])
DET_DTYPE = np.dtype([("box", "<i4"), ("roi", "<i4"), ("frame", "<i4"),
                      ("x1", "<f4"), ("y1", "<f4"), ("x2", "<f4"), ("y2", "<f4")])
DET_WORDS = 7  # int32 words per tg_det
SLO_PATCH_DTYPE = np.dtype([("w", "<i4"), ("h", "<i4"), ("t_arrive", "<f8"), ("t_ddl", "<f8")])
INVOCATION_DTYPE = np.dtype([("t_fire", "<f8"), ("t_ddl", "<f8"), ("t_slack", "<f8"),
                             ("first", "<i4"), ("count", "<i4"), ("n_canvases", "<i4"),
                             ("reason", "<i4")])
FIRE_DEADLINE, FIRE_SLO, FIRE_MEMORY = 0, 1, 2

_i32, _i64, _f32, _u8, _vp = (ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_uint8,
                              ctypes.c_void_p)


class PackParams(ctypes.Structure):
    _fields_ = [("canvas_w", _i32), ("canvas_h", _i32), ("frame_w", _i32), ("frame_h", _i32),
                ("n_frames", _i32), ("policy", _i32)]


class StitchArgs(ctypes.Structure):
    _fields_ = [("frames", _vp), ("frame_stride", _i64), ("n_frames", _i32), ("frame_w", _i32),
                ("frame_h", _i32), ("row_pitch", _i32), ("rois", _vp), ("place", _vp),
                ("order", _vp), ("canvas_begin", _vp), ("n_rois", _i32), ("n_canvases", _i32),
                ("canvas_first", _i32), ("canvas_count", _i32), ("canvas_w", _i32),
                ("canvas_h", _i32), ("mean", _f32 * 3), ("std", _f32 * 3), ("pad", _u8 * 3),
                ("out", _vp), ("unit_order", _vp)]


class UnstitchArgs(ctypes.Structure):
    _fields_ = [("boxes", _vp), ("box_canvas", _vp), ("n_boxes", _i32), ("rois", _vp),
                ("place", _vp), ("order", _vp), ("canvas_begin", _vp), ("n_rois", _i32),
                ("n_canvases", _i32), ("clip", _i32), ("roi_of_box", _vp), ("dets", _vp),
                ("n_out", _vp), ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t),
                ("rule", _i32)]


class PartitionArgs(ctypes.Structure):
    _fields_ = [("boxes", _vp), ("frame_begin", _vp), ("n_boxes", _i32), ("n_frames", _i32),
                ("frame_w", _i32), ("frame_h", _i32), ("zones_x", _i32), ("zones_y", _i32),
                ("patches", _vp), ("zone_of_box", _vp), ("n_patches", _vp), ("workspace", _vp),
                ("workspace_bytes", ctypes.c_size_t)]


class MergeArgs(ctypes.Structure):
    _fields_ = [("dets", _vp), ("n_dets", _vp), ("n_max", _i32), ("scores", _vp),
                ("n_scores", _i32), ("n_frames", _i32), ("iou_threshold", _f32),
                ("cross_only", _i32), ("keep", _vp), ("out", _vp), ("n_kept", _vp),
                ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t)]


class SloParams(ctypes.Structure):
    _fields_ = [("canvas_w", _i32), ("canvas_h", _i32), ("policy", _i32), ("max_canvases", _i32),
                ("n_lat", _i32), ("lat_mean", _vp), ("lat_std", _vp)]


class GmmParams(ctypes.Structure):
    _fields_ = [("n_mix", _i32), ("alpha", _f32), ("var_threshold", _f32),
                ("var_threshold_gen", _f32), ("var_init", _f32), ("var_min", _f32),
                ("var_max", _f32), ("background_ratio", _f32), ("complexity_reduction", _f32)]


class GmmArgs(ctypes.Structure):
    _fields_ = [("frames", _vp), ("n_frames", _i32), ("width", _i32), ("height", _i32),
                ("state", _vp), ("modes", _vp), ("mask", _vp), ("params", GmmParams)]


class MaskRoisArgs(ctypes.Structure):
    _fields_ = [("mask", _vp), ("n_frames", _i32), ("width", _i32), ("height", _i32),
                ("min_area", _i32), ("rois", _vp), ("areas", _vp), ("max_rois", _i32),
                ("frame_begin", _vp), ("n_rois", _vp), ("n_components", _vp),
                ("max_components", _i32), ("workspace", _vp),
                ("workspace_bytes", ctypes.c_size_t)]


class ProjectArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("x_stride", _i64), ("w", _vp), ("w_stride", _i64), ("adapter", _vp),
                ("a", _vp), ("b", _vp), ("scale", _vp), ("y", _vp), ("y_stride", _i64),
                ("n_tokens", _i32), ("k", _i32), ("n", _i32), ("n_adapters", _i32),
                ("rank", _i32), ("type", _i32), ("workspace", _vp),
                ("workspace_bytes", ctypes.c_size_t)]


class RotateArgs(ctypes.Structure):
    _fields_ = [("q", _vp), ("k", _vp), ("v", _vp), ("q_stride", _i64), ("q_head_stride", _i64),
                ("k_stride", _i64), ("k_head_stride", _i64), ("v_stride", _i64),
                ("v_head_stride", _i64), ("q_weight", _vp), ("k_weight", _vp), ("table", _vp),
                ("pos", _vp), ("q_out", _vp), ("k_out", _vp), ("v_out", _vp),
                ("q_out_stride", _i64), ("q_out_head_stride", _i64), ("k_out_stride", _i64),
                ("k_out_head_stride", _i64), ("v_out_stride", _i64), ("v_out_head_stride", _i64),
                ("slot", _vp), ("n_rows", _i64), ("eps", _f32), ("n_tokens", _i32),
                ("n_heads", _i32), ("n_kv_heads", _i32), ("d", _i32), ("rot", _i32),
                ("axes", _i32), ("interleaved", _i32), ("n_positions", _i32), ("type", _i32)]


class AttendArgs(ctypes.Structure):
    _fields_ = [("q", _vp), ("k", _vp), ("v", _vp), ("q_stride", _i64), ("q_head_stride", _i64),
                ("k_stride", _i64), ("k_head_stride", _i64), ("v_stride", _i64),
                ("v_head_stride", _i64), ("out", _vp), ("out_stride", _i64),
                ("out_head_stride", _i64), ("q_begin", _vp), ("kv_begin", _vp), ("kv_len", _vp),
                ("prefix", _vp), ("q_doc", _vp), ("k_doc", _vp), ("q_pos", _vp), ("k_pos", _vp),
                ("slope", _vp), ("scale", _f32), ("cap", _f32), ("causal", _i32),
                ("n_seqs", _i32), ("n_q_rows", _i32), ("n_k_rows", _i64), ("max_q_len", _i32),
                ("max_kv_len", _i32), ("n_heads", _i32), ("n_kv_heads", _i32), ("d", _i32),
                ("type", _i32), ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t)]


class PagesArgs(ctypes.Structure):
    _fields_ = [("q_begin", _vp), ("kv_len", _vp), ("kv_len_out", _vp), ("release", _vp),
                ("table", _vp), ("table_stride", _i64), ("free_pages", _vp), ("n_free", _vp),
                ("n_free_out", _vp), ("slot", _vp), ("pos", _vp), ("refused", _vp),
                ("n_seqs", _i32), ("n_tokens", _i32), ("n_pages", _i32), ("page_size", _i32),
                ("max_pages", _i32), ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t)]


class AttendPagesArgs(ctypes.Structure):
    _fields_ = [("q", _vp), ("k", _vp), ("v", _vp), ("q_stride", _i64), ("q_head_stride", _i64),
                ("k_stride", _i64), ("k_head_stride", _i64), ("v_stride", _i64),
                ("v_head_stride", _i64), ("out", _vp), ("out_stride", _i64),
                ("out_head_stride", _i64), ("table", _vp), ("table_stride", _i64),
                ("kv_len", _vp), ("q_begin", _vp), ("slope", _vp), ("scale", _f32),
                ("cap", _f32), ("window", _i32), ("n_seqs", _i32), ("n_pages", _i32),
                ("page_size", _i32), ("max_pages", _i32), ("n_q_rows", _i32),
                ("max_kv_len", _i32), ("n_heads", _i32), ("n_kv_heads", _i32), ("d", _i32),
                ("type", _i32), ("workspace", _vp), ("workspace_bytes", ctypes.c_size_t)]


class NormArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("x_stride", _i64), ("y", _vp), ("y_stride", _i64), ("y_norm", _i32),
                ("y_weight", _vp), ("y_bias", _vp), ("gate", _vp), ("gate_stride", _i64),
                ("gate_row", _vp), ("x_scale", _f32), ("y_scale", _f32), ("x_out", _vp),
                ("x_out_stride", _i64), ("h", _vp), ("h_stride", _i64), ("norm", _i32),
                ("weight", _vp), ("bias", _vp), ("eps", _f32), ("n_tokens", _i32), ("n", _i32),
                ("n_gates", _i32), ("type", _i32)]


class QuantizeArgs(ctypes.Structure):
    _fields_ = [("x", _vp), ("x_stride", _i64), ("q", _vp), ("q_stride", _i64), ("scale", _vp),
                ("n_rows", _i32), ("k", _i32), ("type", _i32)]


class ProjectI8Args(ctypes.Structure):
    _fields_ = [("x", _vp), ("x_stride", _i64), ("x_scale", _vp), ("w", _vp), ("w_stride", _i64),
                ("w_scale", _vp), ("y", _vp), ("y_stride", _i64), ("n_tokens", _i32), ("k", _i32),
                ("n", _i32), ("type", _i32)]


GMM_MAX_MIX = 5
F16, BF16 = 0, 1  # enum tg_type
PROJECT_MAX_RANK = 64
ATTEND_MAX_D = 128
PAGES_MAX_SEQS = 1 << 20
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2  # enum tg_norm_kind
NORM_MAX_N = 32768
PROJECT_I8_MAX_K = 131056

EXPORTS = ["tg_gmm_plane_stride", "tg_gmm_state_bytes", "tg_gmm_update",
           "tg_mask_rois_workspace_bytes", "tg_mask_rois", "tg_partition_workspace_bytes", "tg_partition", "tg_plan_pack", "tg_batch_count",
           "tg_batch_range", "tg_plan_upload", "tg_slo_replay", "tg_stitch",
           "tg_stitch_units", "tg_stitch_norm_uses_table",
           "tg_unstitch_workspace_bytes", "tg_unstitch", "tg_unstitch_noalloc",
           "tg_merge_workspace_bytes", "tg_merge",
           "tg_project_workspace_bytes", "tg_project", "tg_rotate",
           "tg_attend_workspace_bytes", "tg_attend",
           "tg_pages_workspace_bytes", "tg_pages",
           "tg_attend_pages_workspace_bytes", "tg_attend_pages",
           "tg_norm", "tg_quantize", "tg_project_i8",
           "tg_strerror", "tg_abi_version"]

_lib = None


class TgError(RuntimeError):
    def __init__(self, call, code, bad_index=-1):
        msg = f"{call}: {strerror(code)} ({code})"
        if bad_index >= 0:
            msg += f", first bad RoI {bad_index}"
        super().__init__(msg)
        self.code = code
        self.bad_index = bad_index


def _device_count(call: str, value) -> int:
    """A count a kernel wrote: negative values are status codes (TG_E_INTERNAL when a
    device pass could not complete), raised as TgError."""
    n = int(value)
    if n < 0:
        raise TgError(call, n)
    return n


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2404_09267_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        L.tg_plan_pack.argtypes = [_vp, _i32, ctypes.POINTER(PackParams), _vp, _vp, _vp, _vp, _vp]
        L.tg_plan_pack.restype = ctypes.c_int
        L.tg_batch_count.argtypes = [_i32, _i32]
        L.tg_batch_count.restype = _i32
        L.tg_batch_range.argtypes = [_i32, _i32, _i32, _vp, _vp]
        L.tg_batch_range.restype = ctypes.c_int
        L.tg_plan_upload.argtypes = [_vp, _vp, ctypes.c_size_t, _vp]
        L.tg_plan_upload.restype = ctypes.c_int
        L.tg_partition_workspace_bytes.argtypes = [_i32]
        L.tg_partition_workspace_bytes.restype = ctypes.c_size_t
        L.tg_partition.argtypes = [ctypes.POINTER(PartitionArgs), _vp]
        L.tg_partition.restype = ctypes.c_int
        L.tg_slo_replay.argtypes = [_vp, _i32, ctypes.POINTER(SloParams), _vp, _vp, _vp, _vp,
                                    _vp]
        L.tg_slo_replay.restype = ctypes.c_int
        L.tg_stitch.argtypes = [ctypes.POINTER(StitchArgs), _vp]
        L.tg_stitch.restype = ctypes.c_int
        L.tg_stitch_norm_uses_table.argtypes = [ctypes.POINTER(_f32), ctypes.POINTER(_f32)]
        L.tg_stitch_norm_uses_table.restype = _i32
        L.tg_stitch_units.argtypes = [_i32, _i32, _i32]
        L.tg_stitch_units.restype = _i32
        L.tg_unstitch_workspace_bytes.argtypes = [_i32, _i32]
        L.tg_unstitch_workspace_bytes.restype = ctypes.c_size_t
        L.tg_unstitch.argtypes = [ctypes.POINTER(UnstitchArgs), _vp]
        L.tg_unstitch.restype = ctypes.c_int
        L.tg_unstitch_noalloc.argtypes = [ctypes.POINTER(UnstitchArgs), _vp]
        L.tg_unstitch_noalloc.restype = ctypes.c_int
        L.tg_merge_workspace_bytes.argtypes = [_i32, _i32]
        L.tg_merge_workspace_bytes.restype = ctypes.c_size_t
        L.tg_merge.argtypes = [ctypes.POINTER(MergeArgs), _vp]
        L.tg_merge.restype = ctypes.c_int
        L.tg_gmm_plane_stride.argtypes = [ctypes.c_int64]
        L.tg_gmm_plane_stride.restype = ctypes.c_int64
        L.tg_gmm_state_bytes.argtypes = [ctypes.c_int64, _i32]
        L.tg_gmm_state_bytes.restype = ctypes.c_size_t
        L.tg_gmm_update.argtypes = [ctypes.POINTER(GmmArgs), _vp]
        L.tg_gmm_update.restype = ctypes.c_int
        L.tg_mask_rois_workspace_bytes.argtypes = [_i32, _i32, _i32, _i32]
        L.tg_mask_rois_workspace_bytes.restype = ctypes.c_size_t
        L.tg_mask_rois.argtypes = [ctypes.POINTER(MaskRoisArgs), _vp]
        L.tg_mask_rois.restype = ctypes.c_int
        L.tg_project_workspace_bytes.argtypes = [_i32] * 5
        L.tg_project_workspace_bytes.restype = ctypes.c_size_t
        L.tg_project.argtypes = [ctypes.POINTER(ProjectArgs), _vp]
        L.tg_project.restype = ctypes.c_int
        L.tg_rotate.argtypes = [ctypes.POINTER(RotateArgs), _vp]
        L.tg_rotate.restype = ctypes.c_int
        L.tg_attend_workspace_bytes.argtypes = [_i32] * 7
        L.tg_attend_workspace_bytes.restype = ctypes.c_size_t
        L.tg_attend.argtypes = [ctypes.POINTER(AttendArgs), _vp]
        L.tg_attend.restype = ctypes.c_int
        L.tg_pages_workspace_bytes.argtypes = [_i32] * 2
        L.tg_pages_workspace_bytes.restype = ctypes.c_size_t
        L.tg_pages.argtypes = [ctypes.POINTER(PagesArgs), _vp]
        L.tg_pages.restype = ctypes.c_int
        L.tg_attend_pages_workspace_bytes.argtypes = [_i32] * 5
        L.tg_attend_pages_workspace_bytes.restype = ctypes.c_size_t
        L.tg_attend_pages.argtypes = [ctypes.POINTER(AttendPagesArgs), _vp]
        L.tg_attend_pages.restype = ctypes.c_int
        L.tg_norm.argtypes = [ctypes.POINTER(NormArgs), _vp]
        L.tg_norm.restype = ctypes.c_int
        L.tg_quantize.argtypes = [ctypes.POINTER(QuantizeArgs), _vp]
        L.tg_quantize.restype = ctypes.c_int
        L.tg_project_i8.argtypes = [ctypes.POINTER(ProjectI8Args), _vp]
        L.tg_project_i8.restype = ctypes.c_int
        L.tg_strerror.argtypes = [ctypes.c_int]
        L.tg_strerror.restype = ctypes.c_char_p
        L.tg_abi_version.argtypes = []
        L.tg_abi_version.restype = _i32
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().tg_strerror(int(code)).decode()


def _np_ptr(a: np.ndarray):
    return a.ctypes.data_as(_vp)


# --------------------------------------------------------------------------- planning

@dataclass
class Plan:
    """Host outputs of tg_plan_pack."""
    place: np.ndarray         # int32 [n, 3] = {canvas, x, y}
    order: np.ndarray         # int32 [n]
    canvas_begin: np.ndarray  # int32 [J + 1]
    n_canvases: int


def plan_pack(rois: np.ndarray, canvas_w: int, canvas_h: int, frame_w: int, frame_h: int,
              n_frames: int, policy: int = SHELF_FFDH) -> Plan:
    r = np.ascontiguousarray(rois, dtype=np.int32).reshape(-1, 5)
    n = r.shape[0]
    place = np.empty((n, 3), dtype=np.int32)
    order = np.empty(n, dtype=np.int32)
    cbeg = np.empty(n + 1, dtype=np.int32)
    J = np.zeros(1, dtype=np.int32)
    bad = np.full(1, -1, dtype=np.int32)
    p = PackParams(canvas_w, canvas_h, frame_w, frame_h, n_frames, policy)
    rc = lib().tg_plan_pack(_np_ptr(r), n, ctypes.byref(p), _np_ptr(place), _np_ptr(order),
                            _np_ptr(cbeg), _np_ptr(J), _np_ptr(bad))
    if rc != OK:
        raise TgError("tg_plan_pack", rc, int(bad[0]))
    j = int(J[0])
    return Plan(place, order, cbeg[: j + 1].copy(), j)


def plan_pack_raw(rois: np.ndarray, params: PackParams, place, order, cbeg, J, bad) -> int:
    """Unchecked call on caller-provided numpy buffers (for tests of error codes)."""
    r = np.ascontiguousarray(rois, dtype=np.int32).reshape(-1, 5)
    return lib().tg_plan_pack(_np_ptr(r), r.shape[0], ctypes.byref(params), _np_ptr(place),
                              _np_ptr(order), _np_ptr(cbeg), _np_ptr(J), _np_ptr(bad))


def batch_count(n_canvases: int, batch_cap: int) -> int:
    return int(lib().tg_batch_count(n_canvases, batch_cap))


def batch_range(n_canvases: int, batch_cap: int, k: int):
    first = np.zeros(1, dtype=np.int32)
    count = np.zeros(1, dtype=np.int32)
    rc = lib().tg_batch_range(n_canvases, batch_cap, k, _np_ptr(first), _np_ptr(count))
    if rc != OK:
        raise TgError("tg_batch_range", rc)
    return int(first[0]), int(count[0])


def plan_upload(src, dst, stream=None) -> None:
    """Copies pinned host tensor `src` into device tensor `dst` (same byte size) with
    tg_plan_upload on `stream` (the current stream by default)."""
    import torch

    if not src.is_pinned():
        raise ValueError("plan_upload: the source must be pinned host memory")
    if not dst.is_cuda or not dst.is_contiguous() or not src.is_contiguous():
        raise ValueError("plan_upload: a contiguous pinned source and device destination")
    n = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != n:
        raise ValueError("plan_upload: source and destination sizes differ")
    s = stream or torch.cuda.current_stream()
    rc = lib().tg_plan_upload(_vp(src.data_ptr()), _vp(dst.data_ptr()), n, _vp(s.cuda_stream))
    if rc != OK:
        raise TgError("tg_plan_upload", rc)


@dataclass
class SloReplay:
    """Host outputs of tg_slo_replay."""
    order: np.ndarray        # int32 [n]: patch ids grouped by invocation
    place: np.ndarray        # int32 [n, 3]: {canvas inside its invocation, x, y} per patch
    invocations: np.ndarray  # INVOCATION_DTYPE [n_inv]


def slo_patches(w, h, t_arrive, t_ddl) -> np.ndarray:
    """Packs per-patch arrays into tg_slo_patch records."""
    out = np.zeros(len(w), dtype=SLO_PATCH_DTYPE)
    out["w"], out["h"], out["t_arrive"], out["t_ddl"] = w, h, t_arrive, t_ddl
    return out


def slo_replay(patches: np.ndarray, canvas_w: int, canvas_h: int, policy: int, max_canvases: int,
               lat_mean, lat_std) -> SloReplay:
    pt = np.ascontiguousarray(patches, dtype=SLO_PATCH_DTYPE)
    n = pt.shape[0]
    mean = np.ascontiguousarray(lat_mean, dtype=np.float64)
    sd = np.ascontiguousarray(lat_std, dtype=np.float64)
    if mean.shape != sd.shape:
        raise ValueError("latency mean and std tables differ in length")
    p = SloParams(canvas_w, canvas_h, policy, max_canvases, mean.shape[0], _np_ptr(mean),
                  _np_ptr(sd))
    order = np.empty(n, dtype=np.int32)
    place = np.empty((n, 3), dtype=np.int32)
    inv = np.empty(max(n, 1), dtype=INVOCATION_DTYPE)
    n_inv = np.zeros(1, dtype=np.int32)
    bad = np.full(1, -1, dtype=np.int32)
    rc = lib().tg_slo_replay(_np_ptr(pt), n, ctypes.byref(p), _np_ptr(order), _np_ptr(place),
                             _np_ptr(inv), _np_ptr(n_inv), _np_ptr(bad))
    if rc != OK:
        raise TgError("tg_slo_replay", rc, int(bad[0]))
    return SloReplay(order, place, inv[: int(n_inv[0])].copy())


# --------------------------------------------------------------------------- device side

_raw_stream = None  # torch's call for the current stream's handle, where it has one


def _stream_handle(stream):
    global _raw_stream
    if stream is not None:
        return _vp(stream.cuda_stream)
    if _raw_stream is None:
        import torch

        torch.cuda.current_stream()  # initialises the device once
        raw, device = (getattr(torch._C, n, None) for n in
                       ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        if raw is not None and device is not None:
            _raw_stream = lambda: raw(device())  # without a Stream object: a call takes 5 us instead of 8
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _vp(_raw_stream())


def _check(t, dtype, shape=None, name="tensor"):
    import torch

    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


class DevicePlan:
    """Device copies of a plan's arrays (int32, contiguous) for tg_stitch/tg_unstitch."""

    def __init__(self, rois: np.ndarray, plan: Plan, device="cuda"):
        import torch

        r = np.ascontiguousarray(rois, dtype=np.int32).reshape(-1, 5)
        self.n_rois = r.shape[0]
        self.n_canvases = plan.n_canvases
        self.rois = torch.from_numpy(r).to(device)
        self.place = torch.from_numpy(np.ascontiguousarray(plan.place, np.int32)).to(device)
        self.order = torch.from_numpy(np.ascontiguousarray(plan.order, np.int32)).to(device)
        self.canvas_begin = torch.from_numpy(
            np.ascontiguousarray(plan.canvas_begin, np.int32)).to(device)

    @classmethod
    def from_tensors(cls, rois, place, order, canvas_begin, n_canvases: int) -> "DevicePlan":
        """Wrap existing device tensors (e.g. views of one staging-backed buffer)."""
        self = cls.__new__(cls)
        self.n_rois = int(rois.shape[0])
        self.n_canvases = int(n_canvases)
        self.rois, self.place, self.order, self.canvas_begin = rois, place, order, canvas_begin
        self.check()
        return self

    def check(self):
        import torch

        _check(self.rois, torch.int32, (self.n_rois, 5), "rois")
        _check(self.place, torch.int32, (self.n_rois, 3), "place")
        _check(self.order, torch.int32, (self.n_rois,), "order")
        _check(self.canvas_begin, torch.int32, (self.n_canvases + 1,), "canvas_begin")


def stitch_norm_uses_table(mean, std) -> bool:
    """True when tg_stitch normalises through its binary16 table (no exact fp32 fma
    constants exist for this mean/std), False when it computes each value."""
    m = (_f32 * 3)(*[float(v) for v in mean])
    s = (_f32 * 3)(*[float(v) for v in std])
    rc = int(lib().tg_stitch_norm_uses_table(m, s))
    if rc < 0:
        raise TgError("tg_stitch_norm_uses_table", rc)
    return bool(rc)


def stitch_units(canvas_w: int, canvas_h: int, canvas_count: int) -> int:
    """Number of work units of one tg_stitch launch (the length of a unit order)."""
    n = int(lib().tg_stitch_units(canvas_w, canvas_h, canvas_count))
    if n < 0:
        raise TgError("tg_stitch_units", n)
    return n


def stitch_args(frames, dplan: DevicePlan, canvas_first, canvas_count, canvas_w, canvas_h,
                mean, std, pad, out, unit_order=None) -> StitchArgs:
    import torch

    dplan.check()
    if frames.dim() != 4 or frames.shape[3] != 3:
        raise ValueError("frames must be uint8 [F, H, W, 3]")
    _check(frames, torch.uint8, name="frames")
    if out.dtype not in (torch.float16, torch.int16):
        raise ValueError("out must be float16 (or int16 bit patterns)")
    _check(out, out.dtype, (canvas_count, 3, canvas_h, canvas_w), "out")
    F, H, W, _ = frames.shape
    a = StitchArgs()
    a.frames = frames.data_ptr()
    a.frame_stride = H * W * 3
    a.n_frames, a.frame_w, a.frame_h, a.row_pitch = F, W, H, W * 3
    a.rois, a.place = dplan.rois.data_ptr(), dplan.place.data_ptr()
    a.order, a.canvas_begin = dplan.order.data_ptr(), dplan.canvas_begin.data_ptr()
    a.n_rois, a.n_canvases = dplan.n_rois, dplan.n_canvases
    a.canvas_first, a.canvas_count = canvas_first, canvas_count
    a.canvas_w, a.canvas_h = canvas_w, canvas_h
    a.mean[:] = [float(v) for v in mean]
    a.std[:] = [float(v) for v in std]
    a.pad[:] = [int(v) for v in pad]
    a.out = out.data_ptr()
    a.unit_order = None
    if unit_order is not None:
        n_units = stitch_units(canvas_w, canvas_h, canvas_count) if canvas_count > 0 else 0
        _check(unit_order, torch.int32, name="unit_order")
        if unit_order.numel() < n_units:
            raise ValueError(f"unit_order must hold {n_units} unit ids")
        a.unit_order = unit_order.data_ptr()
    a._keep = (frames, dplan, out, unit_order)  # the struct holds raw pointers: keep their owners alive
    return a


def stitch(frames, dplan: DevicePlan, canvas_first, canvas_count, canvas_w, canvas_h,
           mean, std, pad, out, stream=None, unit_order=None) -> None:
    """Enqueue tg_stitch for canvases [canvas_first, +canvas_count) into `out`
    (`unit_order`: optional device int32 launch order of the units)."""
    a = stitch_args(frames, dplan, canvas_first, canvas_count, canvas_w, canvas_h,
                    mean, std, pad, out, unit_order)
    rc = lib().tg_stitch(ctypes.byref(a), _stream_handle(stream))
    if rc != OK:
        raise TgError("tg_stitch", rc)


def stitch_raw(args: StitchArgs, stream=None) -> int:
    return int(lib().tg_stitch(ctypes.byref(args), _stream_handle(stream)))


def unstitch_workspace_bytes(n_boxes: int, n_rois: int) -> int:
    return int(lib().tg_unstitch_workspace_bytes(n_boxes, n_rois))


class PartitionBuffers:
    """Caller-owned device outputs and scratch for tg_partition."""

    def __init__(self, n_boxes: int, n_frames: int, device="cuda"):
        import torch

        self.n_boxes, self.n_frames = n_boxes, n_frames
        self.patches = torch.empty((max(n_boxes, 1), 5), dtype=torch.int32, device=device)
        self.zone_of_box = torch.empty(max(n_boxes, 1), dtype=torch.int32, device=device)
        self.n_patches = torch.empty(1, dtype=torch.int32, device=device)
        ws = int(lib().tg_partition_workspace_bytes(n_frames))
        self.workspace = torch.empty(max(ws, 8), dtype=torch.uint8, device=device)
        self.workspace_bytes = ws

    def patches_numpy(self) -> np.ndarray:
        n = _device_count("tg_partition", self.n_patches.item())
        return self.patches[:n].cpu().numpy()


def partition_args(boxes, frame_begin, frame_w, frame_h, zones_x, zones_y,
                   bufs: PartitionBuffers, zone_of_box=True) -> PartitionArgs:
    import torch

    _check(boxes, torch.int32, (bufs.n_boxes, 5), "boxes")
    _check(frame_begin, torch.int32, (bufs.n_frames + 1,), "frame_begin")
    a = PartitionArgs()
    a.boxes, a.frame_begin = boxes.data_ptr(), frame_begin.data_ptr()
    a.n_boxes, a.n_frames, a.frame_w, a.frame_h = bufs.n_boxes, bufs.n_frames, frame_w, frame_h
    a.zones_x, a.zones_y = zones_x, zones_y
    a.patches = bufs.patches.data_ptr()
    a.zone_of_box = bufs.zone_of_box.data_ptr() if zone_of_box else None
    a.n_patches = bufs.n_patches.data_ptr()
    a.workspace, a.workspace_bytes = bufs.workspace.data_ptr(), bufs.workspace_bytes
    a._keep = (boxes, frame_begin, bufs)  # the struct holds raw pointers: keep their owners alive
    return a


def partition(boxes, frame_begin, frame_w, frame_h, zones_x, zones_y, bufs: PartitionBuffers,
              stream=None, zone_of_box=True) -> None:
    """Enqueue tg_partition; patches land in `bufs`."""
    a = partition_args(boxes, frame_begin, frame_w, frame_h, zones_x, zones_y, bufs, zone_of_box)
    rc = lib().tg_partition(ctypes.byref(a), _stream_handle(stream))
    if rc != OK:
        raise TgError("tg_partition", rc)


class UnstitchBuffers:
    """Caller-owned device outputs and scratch for tg_unstitch of n_boxes boxes over a plan
    of n_rois RoIs."""

    def __init__(self, n_boxes: int, n_rois: int, device="cuda"):
        import torch

        self.n_boxes, self.n_rois = n_boxes, n_rois
        self.roi_of_box = torch.empty(n_boxes, dtype=torch.int32, device=device)
        self.dets = torch.empty((n_boxes, DET_WORDS), dtype=torch.int32, device=device)
        self.n_out = torch.empty(1, dtype=torch.int32, device=device)
        ws = unstitch_workspace_bytes(n_boxes, n_rois)
        self.workspace = torch.empty(max(ws, 16), dtype=torch.uint8, device=device)
        self.workspace_bytes = ws

    def dets_numpy(self) -> np.ndarray:
        n = _device_count("tg_unstitch", self.n_out.item())
        return self.dets[:n].cpu().numpy().view(DET_DTYPE).reshape(-1)


def unstitch_args(boxes, box_canvas, dplan: DevicePlan, clip, bufs: UnstitchBuffers,
                  rule: int = 0) -> UnstitchArgs:
    import torch

    dplan.check()
    n = bufs.n_boxes
    _check(boxes, torch.float32, (n, 4), "boxes")
    _check(box_canvas, torch.int32, (n,), "box_canvas")
    if bufs.n_rois < dplan.n_rois:
        raise ValueError(f"UnstitchBuffers sized for {bufs.n_rois} RoIs, the plan has {dplan.n_rois}")
    a = UnstitchArgs()
    a.boxes, a.box_canvas, a.n_boxes = boxes.data_ptr(), box_canvas.data_ptr(), n
    a.rois, a.place = dplan.rois.data_ptr(), dplan.place.data_ptr()
    a.order, a.canvas_begin = dplan.order.data_ptr(), dplan.canvas_begin.data_ptr()
    a.n_rois, a.n_canvases, a.clip = dplan.n_rois, dplan.n_canvases, int(bool(clip))
    a.roi_of_box, a.dets, a.n_out = (bufs.roi_of_box.data_ptr(), bufs.dets.data_ptr(),
                                     bufs.n_out.data_ptr())
    a.workspace, a.workspace_bytes = bufs.workspace.data_ptr(), bufs.workspace_bytes
    a.rule = int(rule)
    a._keep = (boxes, box_canvas, dplan, bufs)  # the struct holds raw pointers: keep their owners alive
    return a


def unstitch(boxes, box_canvas, dplan: DevicePlan, clip, bufs: UnstitchBuffers,
             stream=None, rule: int = 0) -> None:
    """Enqueue tg_unstitch; results land in `bufs` (rule 0 centre, 1 largest overlap)."""
    a = unstitch_args(boxes, box_canvas, dplan, clip, bufs, rule)
    rc = lib().tg_unstitch(ctypes.byref(a), _stream_handle(stream))
    if rc != OK:
        raise TgError("tg_unstitch", rc)


def unstitch_raw(args: UnstitchArgs, stream=None) -> int:
    return int(lib().tg_unstitch(ctypes.byref(args), _stream_handle(stream)))


UNSTITCH_NOALLOC_MAX_BOXES = 1 << 24
UNSTITCH_NOALLOC_MAX_ROIS = 1 << 17


def unstitch_noalloc_raw(args: UnstitchArgs, stream=None) -> int:
    """tg_unstitch_noalloc: tg_unstitch on the library's own device scratch (the args'
    workspace fields are ignored); calls that may overlap on one GPU must be serialised."""
    return int(lib().tg_unstitch_noalloc(ctypes.byref(args), _stream_handle(stream)))


class MergeBuffers:
    """Caller-owned device outputs and scratch for tg_merge."""

    def __init__(self, n_max: int, n_frames: int, device="cuda"):
        import torch

        self.n_max, self.n_frames = n_max, n_frames
        self.keep = torch.empty(max(n_max, 1), dtype=torch.int32, device=device)
        self.out = torch.empty((max(n_max, 1), DET_WORDS), dtype=torch.int32, device=device)
        self.n_kept = torch.empty(1, dtype=torch.int32, device=device)
        ws = int(lib().tg_merge_workspace_bytes(n_max, n_frames))
        self.workspace = torch.empty(max(ws, 8), dtype=torch.uint8, device=device)
        self.workspace_bytes = ws

    def kept_numpy(self) -> np.ndarray:
        n = _device_count("tg_merge", self.n_kept.item())
        return self.out[:n].cpu().numpy().view(DET_DTYPE).reshape(-1)


def merge_args(dets, n_dets, scores, n_frames, iou_threshold, cross_only,
               bufs: MergeBuffers) -> MergeArgs:
    """dets: int32 [n_max, 7] device tensor of tg_det (e.g. UnstitchBuffers.dets); n_dets:
    device int32 [1] (e.g. UnstitchBuffers.n_out); scores: device float32 per box."""
    import torch

    _check(dets, torch.int32, (bufs.n_max, DET_WORDS), "dets")
    _check(n_dets, torch.int32, (1,), "n_dets")
    _check(scores, torch.float32, None, "scores")
    a = MergeArgs()
    a.dets, a.n_dets, a.n_max = dets.data_ptr(), n_dets.data_ptr(), bufs.n_max
    a.scores, a.n_scores = scores.data_ptr(), scores.numel()
    a.n_frames, a.iou_threshold, a.cross_only = n_frames, float(iou_threshold), int(bool(cross_only))
    a.keep, a.out = bufs.keep.data_ptr(), bufs.out.data_ptr()
    a.n_kept = bufs.n_kept.data_ptr()
    a.workspace, a.workspace_bytes = bufs.workspace.data_ptr(), bufs.workspace_bytes
    a._keep = (dets, n_dets, scores, bufs)  # the struct holds raw pointers: keep their owners alive
    return a


def merge(dets, n_dets, scores, n_frames, iou_threshold, cross_only, bufs: MergeBuffers,
          stream=None) -> None:
    """Enqueue tg_merge; results land in `bufs`."""
    a = merge_args(dets, n_dets, scores, n_frames, iou_threshold, cross_only, bufs)
    rc = lib().tg_merge(ctypes.byref(a), _stream_handle(stream))
    if rc != OK:
        raise TgError("tg_merge", rc)


# ---- background model and mask -> RoIs --------------------------------------------

def gmm_params(n_mix=5, alpha=0.002, var_threshold=16.0, var_threshold_gen=9.0, var_init=15.0,
               var_min=4.0, var_max=75.0, background_ratio=0.9,
               complexity_reduction=0.05) -> GmmParams:
    return GmmParams(n_mix, alpha, var_threshold, var_threshold_gen, var_init, var_min, var_max,
                     background_ratio, complexity_reduction)


class GmmModel:
    """Device state of the per-pixel background model of n_frames cameras (tg_gmm_update):
    5 n_mix planes of `stride` floats, the component counts and the last mask."""

    def __init__(self, n_frames: int, width: int, height: int, n_mix: int, device="cuda"):
        import torch

        self.n_frames, self.width, self.height, self.n_mix = n_frames, width, height, n_mix
        self.n_px = n_frames * width * height
        self.stride = int(lib().tg_gmm_plane_stride(self.n_px))
        nbytes = int(lib().tg_gmm_state_bytes(self.n_px, n_mix))
        if nbytes == 0:
            raise ValueError("bad model size")
        self.state = torch.zeros(nbytes // 4, dtype=torch.float32, device=device)
        self.modes = torch.zeros(max(self.n_px, 4), dtype=torch.uint8, device=device)
        self.mask = torch.zeros(max(self.n_px, 4), dtype=torch.uint8, device=device)

    def planes(self):
        """State as [n_mix, 5, n_px] (a view): weight, mean r, g, b, variance."""
        return self.state.view(self.n_mix, 5, self.stride)[:, :, : self.n_px]

    def reset(self):
        self.modes.zero_()


def gmm_args(frames, model: GmmModel, params: GmmParams) -> GmmArgs:
    import torch

    _check(frames, torch.uint8, (model.n_frames, model.height, model.width, 3), "frames")
    if params.n_mix != model.n_mix:
        raise ValueError("params.n_mix differs from the model's")
    a = GmmArgs()
    a.frames = frames.data_ptr()
    a.n_frames, a.width, a.height = model.n_frames, model.width, model.height
    a.state, a.modes, a.mask = model.state.data_ptr(), model.modes.data_ptr(), model.mask.data_ptr()
    a.params = params
    a._keep = (frames, model)  # the struct holds raw pointers: keep their owners alive
    return a


def gmm_update(frames, model: GmmModel, params: GmmParams, stream=None) -> None:
    """Enqueue tg_gmm_update: one frame per camera; the mask lands in model.mask."""
    a = gmm_args(frames, model, params)
    rc = lib().tg_gmm_update(ctypes.byref(a), _stream_handle(stream))
    if rc != OK:
        raise TgError("tg_gmm_update", rc)


class MaskRoisBuffers:
    """Caller-owned device outputs and scratch for tg_mask_rois."""

    def __init__(self, n_frames: int, width: int, height: int, max_rois: int,
                 max_components: int, device="cuda"):
        import torch

        self.n_frames, self.width, self.height = n_frames, width, height
        self.max_rois, self.max_components = max_rois, max_components
        self.rois = torch.empty((max(max_rois, 1), 5), dtype=torch.int32, device=device)
        self.areas = torch.empty(max(max_rois, 1), dtype=torch.int32, device=device)
        self.frame_begin = torch.empty(n_frames + 1, dtype=torch.int32, device=device)
        self.counts = torch.empty(2, dtype=torch.int32, device=device)  # n_rois, n_components
        ws = int(lib().tg_mask_rois_workspace_bytes(n_frames, width, height, max_components))
        if ws == 0:
            raise ValueError("bad mask size or max_components")
        self.workspace = torch.empty(ws, dtype=torch.uint8, device=device)
        self.workspace_bytes = ws

    def result(self):
        """(rois int32 [n][5], areas int32 [n], frame_begin, n_rois, n_components)."""
        n_rois, n_comp = (int(v) for v in self.counts.cpu().tolist())
        _device_count("tg_mask_rois", n_rois)
        n = min(n_rois, self.max_rois)
        return (self.rois[:n].cpu().numpy(), self.areas[:n].cpu().numpy(),
                self.frame_begin.cpu().numpy(), n_rois, n_comp)


def mask_rois_args(mask, bufs: MaskRoisBuffers, min_area: int) -> MaskRoisArgs:
    import torch

    _check(mask, torch.uint8, None, "mask")
    if mask.numel() < bufs.n_frames * bufs.width * bufs.height:
        raise ValueError("mask smaller than n_frames * height * width")
    a = MaskRoisArgs()
    a.mask = mask.data_ptr()
    a.n_frames, a.width, a.height, a.min_area = bufs.n_frames, bufs.width, bufs.height, min_area
    a.rois, a.areas, a.max_rois = bufs.rois.data_ptr(), bufs.areas.data_ptr(), bufs.max_rois
    a.frame_begin = bufs.frame_begin.data_ptr()
    a.n_rois = bufs.counts.data_ptr()
    a.n_components = bufs.counts.data_ptr() + 4
    a.max_components = bufs.max_components
    a.workspace, a.workspace_bytes = bufs.workspace.data_ptr(), bufs.workspace_bytes
    a._keep = (mask, bufs)  # the struct holds raw pointers: keep their owners alive
    return a


def mask_rois(mask, bufs: MaskRoisBuffers, min_area: int = 1, stream=None) -> None:
    """Enqueue tg_mask_rois; RoIs land in `bufs`."""
    a = mask_rois_args(mask, bufs, min_area)
    rc = lib().tg_mask_rois(ctypes.byref(a), _stream_handle(stream))
    if rc != OK:
        raise TgError("tg_mask_rois", rc)


# ---- token operators: a transformer over stitched canvases --------------------------

def _type_of(dtype) -> int:
    import torch

    if dtype == torch.float16:
        return F16
    if dtype == torch.bfloat16:
        return BF16
    raise ValueError(f"float16 or bfloat16, got {dtype}")


def _values(t, dtype, dims, name, shape=None):
    """Checks a tensor of values: on the device, of `dtype`, last dimension contiguous."""
    import torch

    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != dims or (t.numel() > 0 and t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name} must have {dims} dimensions, the last one contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _rows(t):
    """Pointer and strides of rows and heads; 0 for one row or head, whose stride may be anything."""
    return (t.data_ptr(), *(t.stride(i) if t.shape[i] > 1 else 0 for i in (0, 1)))


class Adapters:
    """Low-rank adapters on the device: a [n, rank, k], b [n, outputs, rank], scale [n]."""

    def __init__(self, a, b, scale):
        import torch

        _check(a, a.dtype, None, "a")
        if a.dim() != 3:
            raise ValueError("a must be [adapters, rank, k]")
        _type_of(a.dtype)
        self.n, self.rank, self.k = a.shape
        if b.dim() != 3 or b.shape[0] != self.n or b.shape[2] != self.rank:
            raise ValueError("b must be [adapters, outputs, rank]")
        _check(b, a.dtype, None, "b")
        _check(scale, torch.float32, (self.n,), "scale")
        self.a, self.b, self.scale = a, b, scale
        self.outputs = b.shape[1]


class ProjectBuffers:
    """Caller-owned result and scratch of tg_project for n_tokens tokens."""

    def __init__(self, n_tokens: int, k: int, n: int, dtype, adapters: Adapters | None = None,
                 device="cuda"):
        import torch

        self.n_tokens = n_tokens
        self.y = torch.empty((n_tokens, n), dtype=dtype, device=device)
        low = (adapters.n, adapters.rank) if adapters is not None else (0, 0)
        ws = int(lib().tg_project_workspace_bytes(n_tokens, k, n, *low))
        self.workspace = torch.empty(max(ws, 16), dtype=torch.uint8, device=device)
        self.workspace_bytes = ws


def project_args(x, w, bufs: ProjectBuffers, adapters: Adapters | None = None,
                 token_adapter=None) -> ProjectArgs:
    """x [tokens, k], w [outputs, k], rows of any stride; token_adapter: device int32
    [tokens], outside [0, adapters.n) a token has none."""
    import torch

    dt = x.dtype
    type_ = _type_of(dt)
    _values(x, dt, 2, "x")
    n_tokens, k = x.shape
    _values(w, dt, 2, "w")
    n = w.shape[0]
    if w.shape[1] != k:
        raise ValueError(f"w must have {k} columns")
    _values(bufs.y, dt, 2, "y", (n_tokens, n))
    if (adapters is None) != (token_adapter is None):
        raise ValueError("adapters and token_adapter: both or neither")
    a = ProjectArgs()
    a.x, a.x_stride = x.data_ptr(), x.stride(0) if n_tokens > 1 else k
    a.w, a.w_stride = w.data_ptr(), w.stride(0) if n > 1 else k
    a.y, a.y_stride = bufs.y.data_ptr(), bufs.y.stride(0) if n_tokens > 1 else n
    a.n_tokens, a.k, a.n, a.type = n_tokens, k, n, type_
    if adapters is not None:
        _check(token_adapter, torch.int32, (n_tokens,), "token_adapter")
        if adapters.a.dtype != dt or adapters.k != k or adapters.outputs != n:
            raise ValueError("the adapters' type or sizes differ from the projection's")
        a.adapter, a.a, a.b = (token_adapter.data_ptr(), adapters.a.data_ptr(),
                               adapters.b.data_ptr())
        a.scale, a.n_adapters, a.rank = adapters.scale.data_ptr(), adapters.n, adapters.rank
    a.workspace, a.workspace_bytes = bufs.workspace.data_ptr(), bufs.workspace_bytes
    a._keep = (x, w, bufs, adapters, token_adapter)  # the struct holds raw pointers: keep their owners alive
    return a


def project_raw(args: ProjectArgs, stream=None) -> int:
    return int(lib().tg_project(ctypes.byref(args), _stream_handle(stream)))


def project(x, w, bufs: ProjectBuffers, adapters: Adapters | None = None, token_adapter=None,
            stream=None) -> None:
    """Enqueue tg_project: x w^T plus each token's adapter, into bufs.y."""
    rc = project_raw(project_args(x, w, bufs, adapters, token_adapter), stream)
    if rc != OK:
        raise TgError("tg_project", rc)


def rotate_args(q, k, q_weight, k_weight, table, pos, q_out, k_out, v=None, v_out=None, slot=None,
                eps: float = 1e-6, interleaved: bool = False) -> RotateArgs:
    """q [tokens, heads, d], k and v [tokens, kv heads, d], any strides; weights [d] or None;
    table float32 [positions, rot / 2, 2] of cosines and sines; pos int32 [tokens, axes];
    slot: int64 [tokens], rows of k_out and v_out."""
    import torch

    dt = q.dtype
    type_ = _type_of(dt)
    _values(q, dt, 3, "q")
    n_tokens, n_heads, d = q.shape
    _values(k, dt, 3, "k")
    n_kv = k.shape[1]
    if k.shape[0] != n_tokens or k.shape[2] != d:
        raise ValueError(f"k must have shape ({n_tokens}, kv heads, {d})")
    _values(q_out, dt, 3, "q_out", q.shape)
    _values(k_out, dt, 3, "k_out", None if slot is not None else k.shape)
    if tuple(k_out.shape[1:]) != (n_kv, d):
        raise ValueError("k_out must have the heads of k")
    if (v is None) != (v_out is None):
        raise ValueError("v and v_out: both or neither")
    if v is not None:
        _values(v, dt, 3, "v", k.shape)
        _values(v_out, dt, 3, "v_out", k_out.shape)
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None:
            _check(w, dt, (d,), name)
    _check(table, torch.float32, None, "table")
    if table.dim() != 3 or table.shape[2] != 2:
        raise ValueError("table must be [positions, rot / 2, 2]")
    _check(pos, torch.int32, None, "pos")
    if pos.dim() != 2 or pos.shape[0] != n_tokens:
        raise ValueError("pos must be [tokens, axes]")
    a = RotateArgs()
    a.q, a.q_stride, a.q_head_stride = _rows(q)
    a.k, a.k_stride, a.k_head_stride = _rows(k)
    a.q_out, a.q_out_stride, a.q_out_head_stride = _rows(q_out)
    a.k_out, a.k_out_stride, a.k_out_head_stride = _rows(k_out)
    if v is not None:
        a.v, a.v_stride, a.v_head_stride = _rows(v)
        a.v_out, a.v_out_stride, a.v_out_head_stride = _rows(v_out)
    a.q_weight = q_weight.data_ptr() if q_weight is not None else None
    a.k_weight = k_weight.data_ptr() if k_weight is not None else None
    a.table, a.pos = table.data_ptr(), pos.data_ptr()
    if slot is not None:
        _check(slot, torch.int64, (n_tokens,), "slot")
        a.slot, a.n_rows = slot.data_ptr(), k_out.shape[0]
    a.eps, a.n_tokens, a.n_heads, a.n_kv_heads, a.d = float(eps), n_tokens, n_heads, n_kv, d
    a.rot, a.axes, a.interleaved = 2 * table.shape[1], pos.shape[1], int(bool(interleaved))
    a.n_positions, a.type = table.shape[0], type_
    a._keep = (q, k, v, q_weight, k_weight, table, pos, q_out, k_out, v_out, slot)  # the struct holds raw pointers: keep their owners alive
    return a


def rotate_raw(args: RotateArgs, stream=None) -> int:
    return int(lib().tg_rotate(ctypes.byref(args), _stream_handle(stream)))


def rotate(q, k, q_weight, k_weight, table, pos, q_out, k_out, v=None, v_out=None, slot=None,
           eps: float = 1e-6, interleaved: bool = False, stream=None) -> None:
    """Enqueue tg_rotate: norm and rotation of q and k (and a copy of v) into the outputs."""
    rc = rotate_raw(rotate_args(q, k, q_weight, k_weight, table, pos, q_out, k_out, v, v_out, slot,
                                eps, interleaved), stream)
    if rc != OK:
        raise TgError("tg_rotate", rc)


class Sequences:
    """A ragged batch on the device: queries of sequence s are rows q_begin[s] ..
    q_begin[s + 1], its keys kv_len[s] rows from kv_begin[s] on; max_q and max_kv bound the
    lengths. prefix: int32 [n] or None."""

    def __init__(self, q_begin, kv_begin, kv_len, max_q: int, max_kv: int, prefix=None):
        import torch

        self.n = int(kv_len.shape[0])
        _check(q_begin, torch.int32, (self.n + 1,), "q_begin")
        _check(kv_begin, torch.int64, (self.n,), "kv_begin")
        _check(kv_len, torch.int32, (self.n,), "kv_len")
        if prefix is not None:
            _check(prefix, torch.int32, (self.n,), "prefix")
        self.q_begin, self.kv_begin, self.kv_len, self.prefix = q_begin, kv_begin, kv_len, prefix
        self.max_q, self.max_kv = int(max_q), int(max_kv)


class AttendBuffers:
    """Caller-owned scratch of tg_attend for queries like q [rows, heads, d] and keys like k
    [rows, kv heads, d]."""

    def __init__(self, seqs: Sequences, q, k, device="cuda"):
        import torch

        ws = int(lib().tg_attend_workspace_bytes(seqs.n, q.shape[0], seqs.max_q, seqs.max_kv,
                                                 q.shape[1], k.shape[1], q.shape[2]))
        self.workspace = torch.empty(max(ws, 16), dtype=torch.uint8, device=device)
        self.workspace_bytes = ws


def attend_args(q, k, v, seqs: Sequences, out, bufs: AttendBuffers, scale: float,
                cap: float = 0.0, causal: bool = False, q_doc=None, k_doc=None, q_pos=None,
                k_pos=None, slope=None) -> AttendArgs:
    """q and out [rows, heads, d], k and v [key rows, kv heads, d], any strides; q_doc and
    k_doc int32 per row, q_pos and k_pos int32 [rows, 2], slope float32 [heads]."""
    import torch

    dt = q.dtype
    type_ = _type_of(dt)
    _values(q, dt, 3, "q")
    n_q, n_heads, d = q.shape
    _values(k, dt, 3, "k")
    n_k, n_kv, _ = k.shape
    if k.shape[2] != d:
        raise ValueError(f"k must have heads of {d}")
    _values(v, dt, 3, "v", k.shape)
    _values(out, dt, 3, "out", q.shape)
    if (q_doc is None) != (k_doc is None) or (q_pos is None) != (k_pos is None):
        raise ValueError("documents and positions: of queries and keys, or of neither")
    a = AttendArgs()
    a.q, a.q_stride, a.q_head_stride = _rows(q)
    a.k, a.k_stride, a.k_head_stride = _rows(k)
    a.v, a.v_stride, a.v_head_stride = _rows(v)
    a.out, a.out_stride, a.out_head_stride = _rows(out)
    a.q_begin, a.kv_begin, a.kv_len = (seqs.q_begin.data_ptr(), seqs.kv_begin.data_ptr(),
                                       seqs.kv_len.data_ptr())
    a.prefix = seqs.prefix.data_ptr() if seqs.prefix is not None else None
    if q_doc is not None:
        _check(q_doc, torch.int32, (n_q,), "q_doc")
        _check(k_doc, torch.int32, (n_k,), "k_doc")
        a.q_doc, a.k_doc = q_doc.data_ptr(), k_doc.data_ptr()
    if q_pos is not None:
        _check(q_pos, torch.int32, (n_q, 2), "q_pos")
        _check(k_pos, torch.int32, (n_k, 2), "k_pos")
        a.q_pos, a.k_pos = q_pos.data_ptr(), k_pos.data_ptr()
    if slope is not None:
        _check(slope, torch.float32, (n_heads,), "slope")
        a.slope = slope.data_ptr()
    a.scale, a.cap, a.causal = float(scale), float(cap), int(bool(causal))
    a.n_seqs, a.n_q_rows, a.n_k_rows = seqs.n, n_q, n_k
    a.max_q_len, a.max_kv_len = seqs.max_q, seqs.max_kv
    a.n_heads, a.n_kv_heads, a.d, a.type = n_heads, n_kv, d, type_
    a.workspace, a.workspace_bytes = bufs.workspace.data_ptr(), bufs.workspace_bytes
    a._keep = (q, k, v, seqs, out, bufs, q_doc, k_doc, q_pos, k_pos, slope)  # the struct holds raw pointers: keep their owners alive
    return a


def attend_raw(args: AttendArgs, stream=None) -> int:
    return int(lib().tg_attend(ctypes.byref(args), _stream_handle(stream)))


def attend(q, k, v, seqs: Sequences, out, bufs: AttendBuffers, scale: float, cap: float = 0.0,
           causal: bool = False, q_doc=None, k_doc=None, q_pos=None, k_pos=None, slope=None,
           stream=None) -> None:
    """Enqueue tg_attend: attention of q over k and v, into out."""
    rc = attend_raw(attend_args(q, k, v, seqs, out, bufs, scale, cap, causal, q_doc, k_doc, q_pos,
                                k_pos, slope), stream)
    if rc != OK:
        raise TgError("tg_attend", rc)


# ---- serving operators: a step of many requests over one paged cache ----------------

def _here(*tensors) -> None:
    """Checks that tensors are on the current device, whose stream a call is enqueued on."""
    import torch

    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.device.index != device:
            raise ValueError(f"a tensor is on {t.device}, the current device is {device}")


def _row(t):
    """Pointer and stride of rows; one row's stride may be anything."""
    return t.data_ptr(), (t.stride(0) if t.shape[0] > 1 else t.shape[1])


class Pages:
    """The pages of a cache on the device: table int32 [sequences, most pages of one], rows of any
    stride; kv_len int32 [sequences]: rows that each holds; and for tg_pages the stack of free
    pages, int32 [pages], whose first n_free (int32 [1]) are free."""

    def __init__(self, table, kv_len, page_size: int, free=None, n_free=None):
        import torch

        _values(table, torch.int32, 2, "table")
        self.n_seqs, self.max_pages = table.shape
        _check(kv_len, torch.int32, (self.n_seqs,), "kv_len")
        if (free is None) != (n_free is None):
            raise ValueError("free and n_free: both or neither")
        if free is not None:
            _check(free, torch.int32, None, "free")
            _check(n_free, torch.int32, (1,), "n_free")
            if free.dim() != 1:
                raise ValueError("free must be [pages]")
        self.table, self.kv_len, self.page_size = table, kv_len, int(page_size)
        self.free, self.n_free = free, n_free

    @classmethod
    def empty(cls, n_seqs: int, max_pages: int, n_pages: int, page_size: int, device="cuda"):
        """No sequence holds a row, all pages are free; page 0 is taken first."""
        import torch

        make = dict(dtype=torch.int32, device=device)
        return cls(torch.full((n_seqs, max_pages), -1, **make), torch.zeros(n_seqs, **make),
                   page_size, torch.arange(n_pages - 1, -1, -1, **make),
                   torch.full((1,), n_pages, **make))


class PagesBuffers:
    """Caller-owned results and scratch of tg_pages for n_tokens tokens."""

    def __init__(self, pages: Pages, n_tokens: int, device="cuda"):
        import torch

        self.slot = torch.empty(n_tokens, dtype=torch.int64, device=device)
        self.pos = torch.empty((n_tokens, 1), dtype=torch.int32, device=device)
        self.refused = torch.empty(1, dtype=torch.int32, device=device)
        ws = int(lib().tg_pages_workspace_bytes(pages.n_seqs, n_tokens))
        self.workspace = torch.empty(max(ws, 16), dtype=torch.uint8, device=device)
        self.workspace_bytes = ws


def pages_args(pages: Pages, q_begin, bufs: PagesBuffers, release=None,
               after: Pages | None = None) -> PagesArgs:
    """q_begin int32 [sequences + 1], release int32 [sequences] or None. The lengths and the count
    of free pages change in place, or go to those of `after`; table and stack always in place."""
    import torch

    if pages.free is None:
        raise ValueError("pages has no stack of free pages")
    after = pages if after is None else after
    if (after.n_free is None or after.n_seqs != pages.n_seqs
            or after.table.data_ptr() != pages.table.data_ptr()
            or after.free.data_ptr() != pages.free.data_ptr()):
        raise ValueError("after must have the table and the stack of pages")
    _check(q_begin, torch.int32, (pages.n_seqs + 1,), "q_begin")
    if release is not None:
        _check(release, torch.int32, (pages.n_seqs,), "release")
    _check(bufs.slot, torch.int64, None, "slot")
    n_tokens = bufs.slot.shape[0]
    _check(bufs.pos, torch.int32, (n_tokens, 1), "pos")
    _check(bufs.refused, torch.int32, (1,), "refused")
    _here(pages.table, pages.kv_len, pages.free, pages.n_free, q_begin, release, bufs.slot,
          bufs.pos, bufs.refused, bufs.workspace, after.kv_len, after.n_free)
    a = PagesArgs()
    a.q_begin = q_begin.data_ptr()
    a.kv_len, a.kv_len_out = pages.kv_len.data_ptr(), after.kv_len.data_ptr()
    a.release = release.data_ptr() if release is not None else None
    a.table, a.table_stride = _row(pages.table)
    a.free_pages = pages.free.data_ptr()
    a.n_free, a.n_free_out = pages.n_free.data_ptr(), after.n_free.data_ptr()
    a.slot, a.pos, a.refused = (bufs.slot.data_ptr(), bufs.pos.data_ptr(),
                                bufs.refused.data_ptr())
    a.n_seqs, a.n_tokens, a.n_pages = pages.n_seqs, n_tokens, pages.free.shape[0]
    a.page_size, a.max_pages = pages.page_size, pages.max_pages
    a.workspace, a.workspace_bytes = bufs.workspace.data_ptr(), bufs.workspace_bytes
    a._keep = (pages, q_begin, bufs, release, after)  # the struct holds raw pointers: keep their owners alive
    return a


def pages_raw(args: PagesArgs, stream=None) -> int:
    return int(lib().tg_pages(ctypes.byref(args), _stream_handle(stream)))


def pages(pages: Pages, q_begin, bufs: PagesBuffers, release=None, after: Pages | None = None,
          stream=None) -> None:
    """Enqueue tg_pages: pages given back and taken, and a cache row for every new token, into
    bufs.slot and bufs.pos."""
    rc = pages_raw(pages_args(pages, q_begin, bufs, release, after), stream)
    if rc != OK:
        raise TgError("tg_pages", rc)


class AttendPagesBuffers:
    """Caller-owned scratch of tg_attend_pages for queries like q [rows, heads, d], of n_seqs
    sequences (by default as many), and a cache like k [rows, kv heads, d]; no sequence has more
    than max_kv keys."""

    def __init__(self, q, k, max_kv: int, n_seqs: int | None = None, device="cuda"):
        import torch

        self.max_kv = int(max_kv)
        n_seqs = q.shape[0] if n_seqs is None else n_seqs
        ws = int(lib().tg_attend_pages_workspace_bytes(n_seqs, self.max_kv, q.shape[1],
                                                       k.shape[1], q.shape[2]))
        self.workspace = torch.empty(max(ws, 16), dtype=torch.uint8, device=device)
        self.workspace_bytes = ws


def attend_pages_args(q, k, v, pages: Pages, out, bufs: AttendPagesBuffers, scale: float,
                      cap: float = 0.0, window: int = 0, slope=None,
                      q_begin=None) -> AttendPagesArgs:
    """q and out [sequences, heads, d], or with q_begin (int32 [sequences + 1], as for tg_pages)
    [tokens, heads, d]; k and v [cache rows, kv heads, d], any strides; whole pages of cache rows
    count; slope float32 [heads]."""
    import torch

    dt = q.dtype
    type_ = _type_of(dt)
    _values(q, dt, 3, "q", None if q_begin is not None else (pages.n_seqs, *q.shape[1:]))
    n_rows, n_heads, d = q.shape
    _values(k, dt, 3, "k")
    rows, n_kv, _ = k.shape
    if k.shape[2] != d:
        raise ValueError(f"k must have heads of {d}")
    _values(v, dt, 3, "v", k.shape)
    _values(out, dt, 3, "out", q.shape)
    if slope is not None:
        _check(slope, torch.float32, (n_heads,), "slope")
    if q_begin is not None:
        _check(q_begin, torch.int32, (pages.n_seqs + 1,), "q_begin")
    if pages.page_size < 1:
        raise ValueError("page_size must be positive")
    _here(q, k, v, pages.table, pages.kv_len, out, bufs.workspace, slope, q_begin)
    a = AttendPagesArgs()
    a.q, a.q_stride, a.q_head_stride = _rows(q)
    a.k, a.k_stride, a.k_head_stride = _rows(k)
    a.v, a.v_stride, a.v_head_stride = _rows(v)
    a.out, a.out_stride, a.out_head_stride = _rows(out)
    a.table, a.table_stride = _row(pages.table)
    a.kv_len = pages.kv_len.data_ptr()
    a.slope = slope.data_ptr() if slope is not None else None
    a.scale, a.cap, a.window = float(scale), float(cap), int(window)
    if q_begin is not None:
        a.q_begin, a.n_q_rows = q_begin.data_ptr(), n_rows
    a.n_seqs, a.n_pages = pages.n_seqs, rows // pages.page_size
    a.page_size = pages.page_size
    a.max_pages, a.max_kv_len = pages.max_pages, bufs.max_kv
    a.n_heads, a.n_kv_heads, a.d, a.type = n_heads, n_kv, d, type_
    a.workspace, a.workspace_bytes = bufs.workspace.data_ptr(), bufs.workspace_bytes
    a._keep = (q, k, v, pages, out, bufs, slope, q_begin)  # the struct holds raw pointers: keep their owners alive
    return a


def attend_pages_raw(args: AttendPagesArgs, stream=None) -> int:
    return int(lib().tg_attend_pages(ctypes.byref(args), _stream_handle(stream)))


def attend_pages(q, k, v, pages: Pages, out, bufs: AttendPagesBuffers, scale: float,
                 cap: float = 0.0, window: int = 0, slope=None, q_begin=None, stream=None) -> None:
    """Enqueue tg_attend_pages: one query of each sequence over its pages, into out."""
    rc = attend_pages_raw(attend_pages_args(q, k, v, pages, out, bufs, scale, cap, window, slope,
                                            q_begin), stream)
    if rc != OK:
        raise TgError("tg_attend_pages", rc)


def norm_args(x, x_out=None, h=None, y=None, y_norm: int = NORM_NONE, y_weight=None, y_bias=None,
              gate=None, gate_row=None, x_scale: float = 1.0, y_scale: float = 1.0,
              norm: int = NORM_RMS, weight=None, bias=None, eps: float = 1e-6) -> NormArgs:
    """x, y, x_out, h [tokens, n], rows of any stride; weights and biases [n]; gate [gates, n],
    rows of any stride; gate_row int32 [tokens]."""
    import torch

    dt = x.dtype
    type_ = _type_of(dt)
    _values(x, dt, 2, "x")
    n_tokens, n = x.shape
    for t, name in ((y, "y"), (x_out, "x_out"), (h, "h")):
        if t is not None:
            _values(t, dt, 2, name, x.shape)
    for t, name in ((y_weight, "y_weight"), (y_bias, "y_bias"), (weight, "weight"),
                    (bias, "bias")):
        if t is not None:
            _check(t, dt, (n,), name)
    if gate is not None:
        _values(gate, dt, 2, "gate", (gate.shape[0], n))
    if gate_row is not None:
        _check(gate_row, torch.int32, (n_tokens,), "gate_row")
    _here(x, y, x_out, h, y_weight, y_bias, weight, bias, gate, gate_row)
    a = NormArgs()
    a.x, a.x_stride = _row(x)
    if y is not None:
        a.y, a.y_stride = _row(y)
    if x_out is not None:
        a.x_out, a.x_out_stride = _row(x_out)
    if h is not None:
        a.h, a.h_stride = _row(h)
    if gate is not None:
        (a.gate, a.gate_stride), a.n_gates = _row(gate), gate.shape[0]
    for t, name in ((y_weight, "y_weight"), (y_bias, "y_bias"), (weight, "weight"),
                    (bias, "bias"), (gate_row, "gate_row")):
        if t is not None:
            setattr(a, name, t.data_ptr())
    a.y_norm, a.norm, a.eps = int(y_norm), int(norm), float(eps)
    a.x_scale, a.y_scale = float(x_scale), float(y_scale)
    a.n_tokens, a.n, a.type = n_tokens, n, type_
    a._keep = (x, x_out, h, y, y_weight, y_bias, gate, gate_row, weight, bias)  # the struct holds raw pointers: keep their owners alive
    return a


def norm_raw(args: NormArgs, stream=None) -> int:
    return int(lib().tg_norm(ctypes.byref(args), _stream_handle(stream)))


def norm(x, x_out=None, h=None, y=None, y_norm: int = NORM_NONE, y_weight=None, y_bias=None,
         gate=None, gate_row=None, x_scale: float = 1.0, y_scale: float = 1.0,
         norm: int = NORM_RMS, weight=None, bias=None, eps: float = 1e-6, stream=None) -> None:
    """Enqueue tg_norm: x_scale x + y_scale gate N_y(y) into x_out, and its norm into h."""
    rc = norm_raw(norm_args(x, x_out, h, y, y_norm, y_weight, y_bias, gate, gate_row, x_scale,
                            y_scale, norm, weight, bias, eps), stream)
    if rc != OK:
        raise TgError("tg_norm", rc)


def quantize_args(x, q, scale) -> QuantizeArgs:
    """x [rows, k] to q int8 [rows, k] and scale float32 [rows]; rows of any stride."""
    import torch

    type_ = _type_of(x.dtype)
    _values(x, x.dtype, 2, "x")
    _values(q, torch.int8, 2, "q", x.shape)
    _check(scale, torch.float32, (x.shape[0],), "scale")
    _here(x, q, scale)
    a = QuantizeArgs()
    a.x, a.x_stride = _row(x)
    a.q, a.q_stride = _row(q)
    a.scale = scale.data_ptr()
    a.n_rows, a.k, a.type = x.shape[0], x.shape[1], type_
    a._keep = (x, q, scale)  # the struct holds raw pointers: keep their owners alive
    return a


def quantize_raw(args: QuantizeArgs, stream=None) -> int:
    return int(lib().tg_quantize(ctypes.byref(args), _stream_handle(stream)))


def quantize(x, q, scale, stream=None) -> None:
    """Enqueue tg_quantize: rows of x to 8-bit integers and a scale each."""
    rc = quantize_raw(quantize_args(x, q, scale), stream)
    if rc != OK:
        raise TgError("tg_quantize", rc)


def project_i8_args(x, x_scale, w, w_scale, y) -> ProjectI8Args:
    """x int8 [tokens, k], w int8 [outputs, k], y [tokens, outputs], rows of any stride; x_scale
    float32 [tokens], w_scale float32 [outputs]."""
    import torch

    _values(x, torch.int8, 2, "x")
    n_tokens, k = x.shape
    _values(w, torch.int8, 2, "w")
    n = w.shape[0]
    if w.shape[1] != k:
        raise ValueError(f"w must have {k} columns")
    type_ = _type_of(y.dtype)
    _values(y, y.dtype, 2, "y", (n_tokens, n))
    _check(x_scale, torch.float32, (n_tokens,), "x_scale")
    _check(w_scale, torch.float32, (n,), "w_scale")
    _here(x, x_scale, w, w_scale, y)
    a = ProjectI8Args()
    a.x, a.x_stride = _row(x)
    a.w, a.w_stride = _row(w)
    a.y, a.y_stride = _row(y)
    a.x_scale, a.w_scale = x_scale.data_ptr(), w_scale.data_ptr()
    a.n_tokens, a.k, a.n, a.type = n_tokens, k, n, type_
    a._keep = (x, x_scale, w, w_scale, y)  # the struct holds raw pointers: keep their owners alive
    return a


def project_i8_raw(args: ProjectI8Args, stream=None) -> int:
    return int(lib().tg_project_i8(ctypes.byref(args), _stream_handle(stream)))


def project_i8(x, x_scale, w, w_scale, y, stream=None) -> None:
    """Enqueue tg_project_i8: x w^T in 8-bit integers times the scales, into y."""
    rc = project_i8_raw(project_i8_args(x, x_scale, w, w_scale, y), stream)
    if rc != OK:
        raise TgError("tg_project_i8", rc)
