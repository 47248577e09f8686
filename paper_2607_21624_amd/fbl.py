"""ctypes binding of libfbl.so (the C ABI in include/fbl.h).

Argument marshalling only, natively for the plain tensor calls (_fastcall.so):
every step of the attention path runs in the HIP kernels behind the C ABI.  torch is used for device memory (allocating outputs
and the workspace) and for the current stream.  If libfbl.so is missing the
import fails; there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfbl.so")

FBL_OK = 0
FBL_ERR_NULL = 1
FBL_ERR_SHAPE = 2
FBL_ERR_DTYPE = 3
FBL_ERR_LAYOUT = 4
FBL_ERR_ALIGN = 5
FBL_ERR_UNSUPPORTED = 6
FBL_ERR_WORKSPACE = 7
FBL_ERR_HIP = 8
FBL_ERR_ARG = 9

FBL_F32 = 0
FBL_BF16 = 1
FBL_MASK_CAUSAL = 1
FBL_MASK_KEY_PADDING = 2

FBL_BWD_PREP = 1
FBL_BWD_KV = 2
FBL_BWD_Q = 4
FBL_BWD_ALL = 7

FBL_PROJ_FWD = 0
FBL_PROJ_BWD_DATA = 1
FBL_PROJ_BWD_WEIGHT = 2
FBL_GEMM_TILE_AUTO = -1
FBL_GEMM_TILE_128x128 = 0
FBL_GEMM_TILE_128x64 = 1
FBL_GEMM_TILE_64x128 = 2
FBL_GEMM_TILE_64x64 = 3
FBL_TUNE_TIME = 0
FBL_TUNE_GFLOPS_X_MEMEFF = 1

FBL_ACT_NONE = 0
FBL_ACT_RELU = 1
FBL_ACT_GELU = 2
FBL_ACT_GELU_TANH = 3
FBL_ACT_SILU = 4
ACTIVATIONS = {"none": FBL_ACT_NONE, "relu": FBL_ACT_RELU, "gelu": FBL_ACT_GELU, "gelu_tanh": FBL_ACT_GELU_TANH,
               "silu": FBL_ACT_SILU}

FBL_HEAD_KV = 0
FBL_HEAD_VK = 1

FBL_ATTN_FWD = 0
FBL_ATTN_BWD_KV = 1
FBL_ATTN_BWD_DQ = 2
FBL_ATTN_TILE_AUTO = -1

EXPORTED = ("fbl_layout_desc", "fbl_layout_packed_qkv", "fbl_layout_offset", "fbl_layout_map_device", "fbl_attn_fwd",
            "fbl_attn_bwd_workspace", "fbl_attn_bwd_workspace_min", "fbl_attn_bwd", "fbl_attn_bwd_phases",
            "fbl_attn_bwd_noalloc", "fbl_attn_fwd_tiled", "fbl_attn_bwd_tiled", "fbl_attn_bwd_launches", "fbl_attn_tile_count",
            "fbl_attn_tile_info", "fbl_attn_candidates", "fbl_attn_auto_tiles", "fbl_attn_tune", "fbl_attn_tuned_tile",
            "fbl_attn_tune_reset", "fbl_proj", "fbl_proj_dt",
            "fbl_gemm_tile_count", "fbl_gemm_tile_info", "fbl_proj_candidates", "fbl_proj_tune", "fbl_proj_tuned_tile", "fbl_proj_auto_tile",
            "fbl_proj_float_tile", "fbl_proj_tune_reset", "fbl_layer_norm_fwd", "fbl_layer_norm_bwd_workspace",
            "fbl_layer_norm_bwd", "fbl_linear_fwd", "fbl_linear_fwd_workspace", "fbl_linear_bwd_workspace", "fbl_linear_bwd",
            "fbl_linear_loss_workspace", "fbl_linear_ce_fwd", "fbl_linear_ce_bwd", "fbl_linear_kd_fwd", "fbl_linear_kd_bwd",
            "fbl_rotary_turns", "fbl_qk_norm_rotary_fwd", "fbl_qk_norm_rotary_bwd_workspace", "fbl_qk_norm_rotary_bwd",
            "fbl_gated_fwd", "fbl_gated_fwd_workspace", "fbl_gated_bwd_workspace", "fbl_gated_bwd",
            "fbl_grad_norm_workspace", "fbl_grad_norm", "fbl_grad_clip", "fbl_clip_grad_norm", "fbl_status_str")


class Layout(ctypes.Structure):
    """Mirror of fbl_layout."""
    _fields_ = [("dtype", ctypes.c_int32), ("reserved0", ctypes.c_int32), ("tile_d", ctypes.c_int32),
                ("reserved1", ctypes.c_int32),
                ("B", ctypes.c_int64), ("S", ctypes.c_int64), ("H", ctypes.c_int64), ("D", ctypes.c_int64),
                ("sb", ctypes.c_int64), ("ss", ctypes.c_int64), ("sh", ctypes.c_int64), ("sd", ctypes.c_int64)]

    def __repr__(self):
        return (f"Layout(dtype={self.dtype}, B={self.B}, S={self.S}, H={self.H}, D={self.D}, "
                f"sb={self.sb}, ss={self.ss}, sh={self.sh}, sd={self.sd}, tile_d={self.tile_d})")


class Mask(ctypes.Structure):
    """Mirror of fbl_mask."""
    _fields_ = [("kind", ctypes.c_uint32), ("reserved", ctypes.c_uint32), ("kv_len", ctypes.c_void_p)]


FBL_ROTARY_MAX_AXES = 4


class RotaryArgs(ctypes.Structure):
    """Mirror of fbl_rotary."""
    _fields_ = [("turns", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("stride_axis", ctypes.c_int64),
                ("stride_batch", ctypes.c_int64), ("stride_token", ctypes.c_int64), ("dims", ctypes.c_int32),
                ("neighbours", ctypes.c_int32), ("num_axes", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("axes", ctypes.c_uint8 * 64)]


class HeadNormArgs(ctypes.Structure):
    """Mirror of fbl_head_norm."""
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("reserved", ctypes.c_uint32)]


class Grad(ctypes.Structure):
    """Mirror of fbl_grad."""
    _fields_ = [("p", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class FblError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_str(status)} (status {status})")


def _load() -> ctypes.CDLL:
    # torch bundles its own HIP runtime (soname libamdhip64.so.7).  Loading it
    # first makes libfbl.so bind to that same runtime instead of pulling in a
    # second copy from /opt/rocm: one runtime owns the device memory and the
    # streams that torch hands over.
    import torch  # noqa: F401
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libfbl.so not built at {LIB_PATH}; run __graft_entry__.build() "
                          "or python paper_2607_21624_amd/build.py")
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER
    vp = ctypes.c_void_p
    lib.fbl_layout_desc.argtypes = [P(Layout), ctypes.c_int32] + [ctypes.c_int64] * 7
    lib.fbl_layout_desc.restype = ctypes.c_int
    lib.fbl_layout_packed_qkv.argtypes = [P(Layout), P(Layout), P(Layout), P(ctypes.c_int64), P(ctypes.c_int64),
                                          ctypes.c_int32] + [ctypes.c_int64] * 7
    lib.fbl_layout_packed_qkv.restype = ctypes.c_int
    lib.fbl_layout_offset.argtypes = [P(Layout)] + [ctypes.c_int64] * 4
    lib.fbl_layout_offset.restype = ctypes.c_int64
    lib.fbl_layout_map_device.argtypes = [P(Layout), vp, vp]
    lib.fbl_layout_map_device.restype = ctypes.c_int
    lib.fbl_attn_fwd.argtypes = [P(Layout), vp, P(Layout), vp, P(Layout), vp, P(Layout), vp, vp,
                                 ctypes.c_float, Mask, vp]
    lib.fbl_attn_fwd.restype = ctypes.c_int
    lib.fbl_attn_bwd_workspace.argtypes = [P(Layout), P(Layout), P(ctypes.c_size_t)]
    lib.fbl_attn_bwd_workspace.restype = ctypes.c_int
    lib.fbl_attn_bwd_workspace_min.argtypes = [P(Layout), P(Layout), P(ctypes.c_size_t)]
    lib.fbl_attn_bwd_workspace_min.restype = ctypes.c_int
    lib.fbl_attn_bwd.argtypes = [P(Layout), vp, P(Layout), vp, P(Layout), vp, P(Layout), vp, P(Layout), vp,
                                 vp, ctypes.c_float, Mask, P(Layout), vp, P(Layout), vp, P(Layout), vp,
                                 vp, ctypes.c_size_t, vp]
    lib.fbl_attn_bwd.restype = ctypes.c_int
    lib.fbl_attn_bwd_phases.argtypes = [ctypes.c_uint32] + lib.fbl_attn_bwd.argtypes
    lib.fbl_attn_bwd_phases.restype = ctypes.c_int
    lib.fbl_attn_bwd_noalloc.argtypes = lib.fbl_attn_bwd.argtypes[:19] + [vp]
    lib.fbl_attn_bwd_noalloc.restype = ctypes.c_int
    lib.fbl_attn_fwd_tiled.argtypes = lib.fbl_attn_fwd.argtypes[:11] + [ctypes.c_int32, vp]
    lib.fbl_attn_fwd_tiled.restype = ctypes.c_int
    lib.fbl_attn_bwd_tiled.argtypes = [ctypes.c_uint32] + lib.fbl_attn_bwd.argtypes[:21] + [ctypes.c_int32,
                                                                                         ctypes.c_int32, vp]
    lib.fbl_attn_bwd_tiled.restype = ctypes.c_int
    lib.fbl_attn_tile_count.argtypes = []
    lib.fbl_attn_tile_count.restype = ctypes.c_int32
    lib.fbl_attn_tile_info.argtypes = [ctypes.c_int32, ctypes.c_int64, P(ctypes.c_int32)]
    lib.fbl_attn_tile_info.restype = ctypes.c_int
    lib.fbl_attn_candidates.argtypes = [ctypes.c_uint32, P(Layout), P(Layout), P(ctypes.c_int32), ctypes.c_int32,
                                        P(ctypes.c_int32)]
    lib.fbl_attn_candidates.restype = ctypes.c_int
    lib.fbl_attn_auto_tiles.argtypes = [P(Layout), P(Layout), ctypes.c_uint32, P(ctypes.c_int32)]
    lib.fbl_attn_auto_tiles.restype = ctypes.c_int
    lib.fbl_attn_bwd_launches.argtypes = [ctypes.c_uint32, P(Layout), P(Layout), ctypes.c_uint32, ctypes.c_size_t,
                                          ctypes.c_int32, ctypes.c_int32, P(ctypes.c_int32)]
    lib.fbl_attn_bwd_launches.restype = ctypes.c_int
    lib.fbl_attn_tune.argtypes = ([P(Layout), vp, P(Layout), vp, P(Layout), vp, P(Layout), vp, vp, P(Layout), vp,
                                   ctypes.c_float, Mask, P(Layout), vp, P(Layout), vp, P(Layout), vp, vp,
                                   ctypes.c_size_t, ctypes.c_uint32, ctypes.c_int32, P(ctypes.c_float),
                                   P(ctypes.c_int32), vp])
    lib.fbl_attn_tune.restype = ctypes.c_int
    lib.fbl_attn_tuned_tile.argtypes = [ctypes.c_uint32, P(Layout), P(Layout), ctypes.c_uint32]
    lib.fbl_attn_tuned_tile.restype = ctypes.c_int32
    lib.fbl_attn_tune_reset.argtypes = []
    lib.fbl_attn_tune_reset.restype = None
    lib.fbl_proj.argtypes = [ctypes.c_uint32] + [ctypes.c_int64] * 3 + [vp, ctypes.c_int64, vp, ctypes.c_int64, vp,
                                                                        ctypes.c_int64, ctypes.c_int32, vp]
    lib.fbl_proj.restype = ctypes.c_int
    lib.fbl_proj_dt.argtypes = [ctypes.c_uint32, ctypes.c_int32] + [ctypes.c_int64] * 3 + [vp, ctypes.c_int64, vp,
                                                                                   ctypes.c_int64, vp, ctypes.c_int64,
                                                                                   ctypes.c_int32, vp]
    lib.fbl_proj_dt.restype = ctypes.c_int
    lib.fbl_gemm_tile_count.argtypes = []
    lib.fbl_gemm_tile_count.restype = ctypes.c_int32
    lib.fbl_gemm_tile_info.argtypes = [ctypes.c_int32, P(ctypes.c_int32)]
    lib.fbl_gemm_tile_info.restype = ctypes.c_int
    lib.fbl_proj_candidates.argtypes = [ctypes.c_uint32] + [ctypes.c_int64] * 3 + [P(ctypes.c_int32), ctypes.c_int32,
                                                                                 P(ctypes.c_int32)]
    lib.fbl_proj_candidates.restype = ctypes.c_int
    lib.fbl_proj_tune.argtypes = lib.fbl_proj.argtypes[:10] + [ctypes.c_uint32, ctypes.c_int32, P(ctypes.c_float),
                                                              P(ctypes.c_int32), vp]
    lib.fbl_proj_tune.restype = ctypes.c_int
    lib.fbl_proj_tuned_tile.argtypes = [ctypes.c_uint32] + [ctypes.c_int64] * 3
    lib.fbl_proj_tuned_tile.restype = ctypes.c_int32
    lib.fbl_proj_auto_tile.argtypes = [ctypes.c_uint32] + [ctypes.c_int64] * 3 + [ctypes.POINTER(ctypes.c_int32)]
    lib.fbl_proj_auto_tile.restype = ctypes.c_int
    lib.fbl_proj_float_tile.argtypes = [ctypes.c_uint32] + [ctypes.c_int64] * 3 + [ctypes.POINTER(ctypes.c_int32)]
    lib.fbl_proj_float_tile.restype = ctypes.c_int
    lib.fbl_proj_tune_reset.argtypes = []
    lib.fbl_proj_tune_reset.restype = None
    i32, i64, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    size, sizep = ctypes.c_size_t, P(ctypes.c_size_t)
    lib.fbl_layer_norm_fwd.argtypes = [i32, i64, i64, vp, i64, vp, vp, f32, vp, i64, vp, vp, vp]
    lib.fbl_layer_norm_fwd.restype = ctypes.c_int
    lib.fbl_layer_norm_bwd_workspace.argtypes = [i32, i64, i64, sizep]
    lib.fbl_layer_norm_bwd_workspace.restype = ctypes.c_int
    lib.fbl_layer_norm_bwd.argtypes = [i32, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, vp, size, vp]
    lib.fbl_layer_norm_bwd.restype = ctypes.c_int
    u32 = ctypes.c_uint32
    lib.fbl_linear_fwd.argtypes = [i32, u32, i64, i64, i64, vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, i64, i32, vp, size, vp]
    lib.fbl_linear_fwd_workspace.argtypes = [i32, i64, i64, i64, sizep]
    lib.fbl_linear_fwd_workspace.restype = ctypes.c_int
    lib.fbl_linear_fwd.restype = ctypes.c_int
    lib.fbl_linear_bwd_workspace.argtypes = [i32, i64, i64, i64, sizep]
    lib.fbl_linear_bwd_workspace.restype = ctypes.c_int
    lib.fbl_linear_bwd.argtypes = [i32, u32, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, u32, vp, i64, vp, i64, vp,
                                   vp, i64, vp, vp, size, vp]
    lib.fbl_linear_bwd.restype = ctypes.c_int
    lib.fbl_linear_loss_workspace.argtypes = [i32, u32] + [i64] * 5 + [sizep]
    lib.fbl_linear_loss_workspace.restype = ctypes.c_int
    lib.fbl_linear_ce_fwd.argtypes = [i32, u32, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, size, vp]
    lib.fbl_linear_ce_fwd.restype = ctypes.c_int
    lib.fbl_linear_ce_bwd.argtypes = [i32, u32, i64, i64, i64, vp, i64, vp, vp, i64, vp, i64, vp, i64, vp, vp, i64, vp, i64,
                                      vp, size, vp]
    lib.fbl_linear_ce_bwd.restype = ctypes.c_int
    lib.fbl_linear_kd_fwd.argtypes = [i32, u32, i64, i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, vp, i64, f32, vp, vp, vp,
                                      vp, vp, vp, size, vp]
    lib.fbl_linear_kd_fwd.restype = ctypes.c_int
    lib.fbl_linear_kd_bwd.argtypes = [i32, u32, i64, i64, i64, i64, vp, i64, vp, vp, i64, vp, i64, vp, i64, f32, vp, vp, vp,
                                      i64, vp, i64, vp, size, vp]
    lib.fbl_linear_kd_bwd.restype = ctypes.c_int
    lib.fbl_rotary_turns.argtypes = [P(ctypes.c_double), i64, P(ctypes.c_uint64)]
    lib.fbl_rotary_turns.restype = ctypes.c_int
    L, R, H = P(Layout), P(RotaryArgs), P(HeadNormArgs)
    lib.fbl_qk_norm_rotary_fwd.argtypes = [L, vp, L, vp, R, H, L, vp, L, vp, vp]
    lib.fbl_qk_norm_rotary_fwd.restype = ctypes.c_int
    lib.fbl_qk_norm_rotary_bwd_workspace.argtypes = [L, L, sizep]
    lib.fbl_qk_norm_rotary_bwd_workspace.restype = ctypes.c_int
    lib.fbl_qk_norm_rotary_bwd.argtypes = [L, vp, L, vp, L, vp, L, vp, R, H, L, vp, L, vp, vp, vp, vp, size, vp]
    lib.fbl_qk_norm_rotary_bwd.restype = ctypes.c_int
    lib.fbl_gated_fwd.argtypes = [i32, u32, i64, i64, i64, vp, i64, vp, i64, vp, vp, i64, vp, i64, i32, vp, size, vp]
    lib.fbl_gated_fwd.restype = ctypes.c_int
    lib.fbl_gated_fwd_workspace.argtypes = [i32, i64, i64, i64, sizep]
    lib.fbl_gated_fwd_workspace.restype = ctypes.c_int
    lib.fbl_gated_bwd_workspace.argtypes = [i32, i64, i64, i64, sizep]
    lib.fbl_gated_bwd_workspace.restype = ctypes.c_int
    lib.fbl_gated_bwd.argtypes = [i32, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i32, vp, size, vp]
    lib.fbl_gated_bwd.restype = ctypes.c_int
    lib.fbl_grad_norm_workspace.argtypes = [i64, sizep]
    lib.fbl_grad_norm_workspace.restype = ctypes.c_int
    lib.fbl_grad_norm.argtypes = [i64, P(Grad), vp, vp, size, vp]
    lib.fbl_grad_norm.restype = ctypes.c_int
    lib.fbl_grad_clip.argtypes = [i64, P(Grad), vp, f32, vp]
    lib.fbl_grad_clip.restype = ctypes.c_int
    lib.fbl_clip_grad_norm.argtypes = [i64, P(Grad), f32, vp, vp, size, vp]
    lib.fbl_clip_grad_norm.restype = ctypes.c_int
    lib.fbl_status_str.argtypes = [ctypes.c_int]
    lib.fbl_status_str.restype = ctypes.c_char_p
    return lib


LIB = _load()

# The plain calls of these functions run natively
# (csrc/fastcall.cpp): each does the whole call, or nothing and returns None --
# any argument that is not a plain one, any error -- and the Python below then
# makes the call with every check.
_NATIVE = ("attn_fwd", "attn_bwd", "attn_fwd_packed", "attn_bwd_packed", "proj", "layer_norm_fwd", "layer_norm_bwd",
           "linear_fwd", "linear_bwd", "linear_ce_fwd", "linear_ce_bwd", "linear_kd_fwd", "linear_kd_bwd", "qk_norm_rotary_fwd",
           "qk_norm_rotary_bwd", "gated_fwd", "gated_bwd", "grad_norm", "clip_grad_norm")


def _load_native():
    """The _fastcall module, or a stand-in that handles no call.  It is compiled
    against one torch and one Python: without it, or with one of another build, the
    Python path makes every call (the same kernels, 10 .. 16 us of host time more)."""
    import sys
    import torch
    try:
        from . import _fastcall  # after _load: it needs libfbl.so's runtime
        wants = (torch.__version__.split("+")[0], "%d.%d" % sys.version_info[:2])
        if _fastcall.built_for != wants:
            raise ImportError(f"_fastcall.so was built for torch {_fastcall.built_for[0]} and Python "
                              f"{_fastcall.built_for[1]}, running {wants[0]} and {wants[1]}")
        return _fastcall
    except ImportError as e:
        import warnings
        warnings.warn(f"native call path unavailable, calls take the Python path: {e}", RuntimeWarning)
        no = staticmethod(lambda *args: None)
        return type("NoNative", (), dict.fromkeys(_NATIVE, no))


_FAST = _load_native()


def status_str(status: int) -> str:
    return LIB.fbl_status_str(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != FBL_OK:
        raise FblError(status, where)


# ------------------------------------------------------------------ layouts
def fbl_layout_desc(dtype: int, B: int, S: int, H: int, D: int, row_stride: int = 0, batch_stride: int = 0,
                    tile_d: int = 0) -> Layout:
    out = Layout()
    _check(LIB.fbl_layout_desc(ctypes.byref(out), dtype, B, S, H, D, row_stride, batch_stride, tile_d),
           "fbl_layout_desc")
    return out


def fbl_layout_desc_status(dtype: int, B: int, S: int, H: int, D: int, row_stride: int = 0,
                           batch_stride: int = 0, tile_d: int = 0) -> Tuple[int, Layout]:
    """Like fbl_layout_desc but returns (status, layout) instead of raising."""
    out = Layout()
    st = LIB.fbl_layout_desc(ctypes.byref(out), dtype, B, S, H, D, row_stride, batch_stride, tile_d)
    return st, out


def fbl_layout_packed_qkv(dtype: int, B: int, S: int, Hq: int, Hkv: int, D: int, batch_stride: int = 0,
                          tile_d: int = 0):
    """Descriptors of Q, K, V inside one packed [B, S, (Hq + 2 Hkv) D] projection
    output: returns (lq, lk, lv, k_off, v_off), offsets in elements."""
    lq, lk, lv = Layout(), Layout(), Layout()
    ko, vo = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(LIB.fbl_layout_packed_qkv(ctypes.byref(lq), ctypes.byref(lk), ctypes.byref(lv), ctypes.byref(ko),
                                     ctypes.byref(vo), dtype, B, S, Hq, Hkv, D, batch_stride, tile_d),
           "fbl_layout_packed_qkv")
    return lq, lk, lv, int(ko.value), int(vo.value)


def fbl_layout_offset(l: Layout, b: int, h: int, s: int, i: int) -> int:
    return LIB.fbl_layout_offset(ctypes.byref(l), b, h, s, i)


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def fbl_layout_map_device(l: Layout, out, stream=None) -> None:
    _check(LIB.fbl_layout_map_device(ctypes.byref(l), _ptr(out), _stream(stream)), "fbl_layout_map_device")


def _mask(causal: bool, kv_len) -> Mask:
    kind = (FBL_MASK_CAUSAL if causal else 0) | (FBL_MASK_KEY_PADDING if kv_len is not None else 0)
    return Mask(kind, 0, _ptr(kv_len))


def fbl_attn_fwd_raw(lq, q, lk, k, lv, v, lo, o, lse, scale, mask: Mask, stream=None,
                     tile: int = FBL_ATTN_TILE_AUTO) -> int:
    """Direct call of fbl_attn_fwd (tile AUTO) or fbl_attn_fwd_tiled; returns the status code."""
    ref = lambda l: ctypes.byref(l) if l is not None else None
    args = (ref(lq), _ptr(q), ref(lk), _ptr(k), ref(lv), _ptr(v), ref(lo), _ptr(o), _ptr(lse), float(scale), mask)
    st = _stream(stream) if stream != 0 else None
    if tile == FBL_ATTN_TILE_AUTO:
        return LIB.fbl_attn_fwd(*args, st)
    return LIB.fbl_attn_fwd_tiled(*args, int(tile), st)


def fbl_attn_bwd_workspace(lq: Layout, lk: Layout) -> int:
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_attn_bwd_workspace(ctypes.byref(lq), ctypes.byref(lk), ctypes.byref(n)), "fbl_attn_bwd_workspace")
    return int(n.value)


def fbl_attn_bwd_workspace_min(lq: Layout, lk: Layout) -> int:
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_attn_bwd_workspace_min(ctypes.byref(lq), ctypes.byref(lk), ctypes.byref(n)),
           "fbl_attn_bwd_workspace_min")
    return int(n.value)


def fbl_attn_bwd_raw(lq, q, lk, k, lv, v, lo, o, ldo, do, lse, scale, mask: Mask, ldq, dq, ldk, dk, ldv, dv,
                     ws, ws_bytes, stream=None, phases: int = FBL_BWD_ALL, kv_tile: int = FBL_ATTN_TILE_AUTO,
                     dq_tile: int = FBL_ATTN_TILE_AUTO) -> int:
    """Direct call of fbl_attn_bwd (phases == FBL_BWD_ALL, AUTO tiles), fbl_attn_bwd_phases (AUTO
    tiles) or fbl_attn_bwd_tiled (an explicit tile); returns the status."""
    ref = lambda l: ctypes.byref(l) if l is not None else None
    args = (ref(lq), _ptr(q), ref(lk), _ptr(k), ref(lv), _ptr(v), ref(lo), _ptr(o), ref(ldo), _ptr(do), _ptr(lse),
            float(scale), mask, ref(ldq), _ptr(dq), ref(ldk), _ptr(dk), ref(ldv), _ptr(dv), _ptr(ws), int(ws_bytes))
    st = _stream(stream) if stream != 0 else None
    if kv_tile != FBL_ATTN_TILE_AUTO or dq_tile != FBL_ATTN_TILE_AUTO:
        return LIB.fbl_attn_bwd_tiled(phases, *args, int(kv_tile), int(dq_tile), st)
    if phases == FBL_BWD_ALL:
        return LIB.fbl_attn_bwd(*args, st)
    return LIB.fbl_attn_bwd_phases(phases, *args, st)


# ------------------------------------------------------- torch-tensor helpers
def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return FBL_BF16
    if t.dtype == torch.float32:
        return FBL_F32
    raise FblError(FBL_ERR_DTYPE, f"unsupported tensor dtype {t.dtype}")


_LAYOUTS = {}


def _layout(t, H: int) -> Layout:
    """layout_of for the calls below, cached per (dtype, shape, strides, H): the
    descriptor only depends on those, and building it costs a library call per
    tensor per launch.  The cached objects are passed read-only (const) and
    never handed out."""
    key = (t.dtype, tuple(t.shape), t.stride(), H)
    l = _LAYOUTS.get(key)
    if l is None:
        l = layout_of(t, H)
        if len(_LAYOUTS) < 4096:
            _LAYOUTS[key] = l
    return l


def layout_of(t, H: int) -> Layout:
    """Descriptor of a token-major [B, S, H*D] tensor (or a strided view of one:
    inner stride 1, arbitrary row and batch strides).  No data is touched."""
    if t.dim() != 3:
        raise FblError(FBL_ERR_SHAPE, "expected a [B, S, H*D] tensor")
    B, S, HD = t.shape
    if HD % H:
        raise FblError(FBL_ERR_SHAPE, f"last dim {HD} not divisible by heads {H}")
    if t.stride(2) != 1:
        raise FblError(FBL_ERR_LAYOUT, "innermost stride must be 1")
    return fbl_layout_desc(_dtype_code(t), B, S, H, HD // H, row_stride=t.stride(1),
                           batch_stride=t.stride(0) if B > 1 else 0)


def _check_kv_len(kv_len, B: int, where: str) -> None:
    """kv_len must be an int32 tensor of at least B entries with unit stride:
    the kernels read kv_len[b] as a 32-bit integer from device memory."""
    if kv_len is None:
        return
    import torch
    if not isinstance(kv_len, torch.Tensor):
        raise FblError(FBL_ERR_ARG, f"{where}: kv_len must be a torch tensor")
    if kv_len.dtype != torch.int32:
        raise FblError(FBL_ERR_DTYPE, f"{where}: kv_len must be int32, got {kv_len.dtype}")
    if kv_len.dim() != 1 or (kv_len.numel() > 1 and kv_len.stride(0) != 1):
        raise FblError(FBL_ERR_LAYOUT, f"{where}: kv_len must be a 1-D tensor with unit stride")
    if kv_len.numel() < B:
        raise FblError(FBL_ERR_SHAPE, f"{where}: kv_len has {kv_len.numel()} entries, needs {B}")


def _check_lse(lse, B: int, Hq: int, S: int, where: str) -> None:
    """lse must be a contiguous float32 [B, Hq, S_q] tensor: the kernels read and
    write it as B*Hq*S_q consecutive floats."""
    if lse is None:
        return
    import torch
    if not isinstance(lse, torch.Tensor):
        raise FblError(FBL_ERR_ARG, f"{where}: lse must be a torch tensor")
    if lse.dtype != torch.float32:
        raise FblError(FBL_ERR_DTYPE, f"{where}: lse must be float32, got {lse.dtype}")
    if tuple(lse.shape) != (B, Hq, S):
        raise FblError(FBL_ERR_SHAPE, f"{where}: lse has shape {tuple(lse.shape)}, needs {(B, Hq, S)}")
    if not lse.is_contiguous():
        raise FblError(FBL_ERR_LAYOUT, f"{where}: lse must be contiguous")


def _check_workspace(ws, where: str) -> None:
    """The workspace is handed over as one span of numel * element_size bytes."""
    if ws is None:
        return
    import torch
    if not isinstance(ws, torch.Tensor):
        raise FblError(FBL_ERR_ARG, f"{where}: workspace must be a torch tensor")
    if not ws.is_contiguous():
        raise FblError(FBL_ERR_LAYOUT, f"{where}: workspace must be contiguous")


def _check_device(where: str, stream, **tensors) -> None:
    """Every tensor argument lives on one GPU, the device the launch stream
    belongs to: the kernels dereference each pointer on that device."""
    import torch
    dev = None
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise FblError(FBL_ERR_ARG, f"{where}: {name} is on {t.device}, not on a GPU")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise FblError(FBL_ERR_ARG, f"{where}: {name} is on {t.device}, the other tensors on {dev}")
    if dev is None or isinstance(stream, int) or stream == 0:
        return
    sdev = torch.cuda.current_device() if stream is None else stream.device.index
    if sdev != dev.index:
        raise FblError(FBL_ERR_ARG, f"{where}: tensors are on {dev}, the stream on cuda:{sdev}")


def attn_fwd(q, k, v, Hq: int, Hkv: int, scale: Optional[float] = None, causal: bool = False, kv_len=None,
             out=None, lse=None, stream=None, tile: int = FBL_ATTN_TILE_AUTO):
    """Forward on token-major tensors.  Returns (O, LSE); O has q's shape and dtype
    (allocated contiguous unless `out` is given), LSE is float32 [B, Hq, S]."""
    done = _FAST.attn_fwd(q, k, v, Hq, Hkv, scale, causal, kv_len, out, lse, stream, tile)
    if done is not None:
        return done
    import torch
    _check_kv_len(kv_len, q.shape[0], "attn_fwd")
    _check_device("attn_fwd", stream, q=q, k=k, v=v, kv_len=kv_len, out=out, lse=lse)
    if q.dim() == 3:
        _check_lse(lse, q.shape[0], Hq, q.shape[1], "attn_fwd")
    lq, lk, lv = _layout(q, Hq), _layout(k, Hkv), _layout(v, Hkv)
    if scale is None:
        scale = 1.0 / math.sqrt(lq.D)
    B, S = q.shape[0], q.shape[1]
    if out is None:
        out = torch.empty((B, S, q.shape[2]), dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((B, Hq, S), dtype=torch.float32, device=q.device)
    lo = _layout(out, Hq)
    _check(fbl_attn_fwd_raw(lq, q, lk, k, lv, v, lo, out, lse, scale, _mask(causal, kv_len), stream, tile),
           "fbl_attn_fwd")
    return out, lse


def attn_bwd(q, k, v, o, do, lse, Hq: int, Hkv: int, scale: Optional[float] = None, causal: bool = False,
             kv_len=None, dq=None, dk=None, dv=None, workspace=None, stream=None, phases: int = FBL_BWD_ALL,
             kv_tile: int = FBL_ATTN_TILE_AUTO, dq_tile: int = FBL_ATTN_TILE_AUTO):
    """Backward.  Returns (dQ, dK, dV) with the shapes/dtypes of q, k, v."""
    done = _FAST.attn_bwd(q, k, v, o, do, lse, Hq, Hkv, scale, causal, kv_len, dq, dk, dv, workspace, stream, phases,
                          kv_tile, dq_tile)
    if done is not None:
        return done
    import torch
    _check_kv_len(kv_len, q.shape[0], "attn_bwd")
    _check_device("attn_bwd", stream, q=q, k=k, v=v, o=o, do=do, lse=lse, kv_len=kv_len, dq=dq, dk=dk, dv=dv,
                  workspace=workspace)
    if q.dim() == 3:
        _check_lse(lse, q.shape[0], Hq, q.shape[1], "attn_bwd")
    _check_workspace(workspace, "attn_bwd")
    lq, lk, lv = _layout(q, Hq), _layout(k, Hkv), _layout(v, Hkv)
    lo, ldo = _layout(o, Hq), _layout(do, Hq)
    if scale is None:
        scale = 1.0 / math.sqrt(lq.D)
    if dq is None:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if dk is None:
        dk = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    if dv is None:
        dv = torch.empty(v.shape, dtype=v.dtype, device=v.device)
    if workspace is None:
        need = fbl_attn_bwd_workspace(lq, lk)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    ldq, ldk, ldv = _layout(dq, Hq), _layout(dk, Hkv), _layout(dv, Hkv)
    _check(fbl_attn_bwd_raw(lq, q, lk, k, lv, v, lo, o, ldo, do, lse, scale, _mask(causal, kv_len), ldq, dq, ldk,
                            dk, ldv, dv, workspace, workspace.numel() * workspace.element_size(), stream,
                            phases, kv_tile, dq_tile), "fbl_attn_bwd")
    return dq, dk, dv


# ------------------------------------------------------- attention tiles
def attn_tiles(D: int):
    """Every attention tile configuration at head dim D:
    {id: dict(pass, rows, cols, waves, per_wave, occupancy, lds_bytes, legal)}."""
    keys = ("pass", "rows", "cols", "waves", "per_wave", "occupancy", "lds_bytes", "legal")
    out = {}
    for t in range(LIB.fbl_attn_tile_count()):
        info = (ctypes.c_int32 * 8)()
        _check(LIB.fbl_attn_tile_info(t, D, info), "fbl_attn_tile_info")
        out[t] = dict(zip(keys, list(info)))
    return out


def attn_candidates(pass_: int, lq: Layout, lk: Layout):
    """Candidate tile ids of one attention pass for these shapes (C1/C2/C3)."""
    n = ctypes.c_int32()
    cap = LIB.fbl_attn_tile_count()
    ids = (ctypes.c_int32 * cap)()
    _check(LIB.fbl_attn_candidates(pass_, ctypes.byref(lq), ctypes.byref(lk), ids, cap, ctypes.byref(n)),
           "fbl_attn_candidates")
    return list(ids[:n.value])


def attn_auto_tiles(lq: Layout, lk: Layout, mask_kind: int):
    """(forward, kv, dQ) tile ids FBL_ATTN_TILE_AUTO resolves to, where a pass
    runs a tile (small untuned calls and one-launch backwards run none)."""
    t = (ctypes.c_int32 * 3)()
    _check(LIB.fbl_attn_auto_tiles(ctypes.byref(lq), ctypes.byref(lk), mask_kind, t), "fbl_attn_auto_tiles")
    return tuple(t)


def attn_bwd_launches(lq: Layout, lk: Layout, mask_kind: int, ws_bytes: int, phases: int = FBL_BWD_ALL,
                      kv_tile: int = FBL_ATTN_TILE_AUTO, dq_tile: int = FBL_ATTN_TILE_AUTO) -> int:
    """Kernel launches a backward call with these shapes, mask bits, workspace
    size and tiles enqueues (1: the one-launch backward)."""
    n = ctypes.c_int32()
    _check(LIB.fbl_attn_bwd_launches(phases, ctypes.byref(lq), ctypes.byref(lk), mask_kind, ws_bytes, kv_tile,
                                     dq_tile, ctypes.byref(n)), "fbl_attn_bwd_launches")
    return n.value


def attn_tune(q, k, v, do, Hq: int, Hkv: int, scale: Optional[float] = None, causal: bool = False, kv_len=None,
              o=None, lse=None, dq=None, dk=None, dv=None, workspace=None, objective: int = FBL_TUNE_TIME,
              reps: int = 10, stream=None):
    """Measured tile selection for this attention shape (fbl_attn_tune).  Returns
    ((fwd, kv, dq) chosen ids, {id: average ms}, outputs (o, lse, dq, dk, dv)
    computed with the chosen tiles).  Among tiles only: a small shape, whose
    untuned calls run other kernels, is usually faster left untuned."""
    import torch
    _check_kv_len(kv_len, q.shape[0], "attn_tune")
    _check_device("attn_tune", stream, q=q, k=k, v=v, do=do, kv_len=kv_len, o=o, lse=lse, dq=dq, dk=dk, dv=dv,
                  workspace=workspace)
    if q.dim() == 3:
        _check_lse(lse, q.shape[0], Hq, q.shape[1], "attn_tune")
    _check_workspace(workspace, "attn_tune")
    lq, lk, lv, ldo = _layout(q, Hq), _layout(k, Hkv), _layout(v, Hkv), _layout(do, Hq)
    if scale is None:
        scale = 1.0 / math.sqrt(lq.D)
    B, S = q.shape[0], q.shape[1]
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device) if o is None else o
    lse = torch.empty((B, Hq, S), dtype=torch.float32, device=q.device) if lse is None else lse
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
    dv = torch.empty(v.shape, dtype=v.dtype, device=v.device) if dv is None else dv
    if workspace is None:
        workspace = torch.empty(fbl_attn_bwd_workspace(lq, lk), dtype=torch.uint8, device=q.device)
    lo, ldq, ldk, ldv = _layout(o, Hq), _layout(dq, Hq), _layout(dk, Hkv), _layout(dv, Hkv)
    cap = LIB.fbl_attn_tile_count()
    ms = (ctypes.c_float * cap)()
    best = (ctypes.c_int32 * 3)()
    ref = ctypes.byref
    _check(LIB.fbl_attn_tune(ref(lq), _ptr(q), ref(lk), _ptr(k), ref(lv), _ptr(v), ref(lo), _ptr(o), _ptr(lse),
                             ref(ldo), _ptr(do), float(scale), _mask(causal, kv_len), ref(ldq), _ptr(dq), ref(ldk),
                             _ptr(dk), ref(ldv), _ptr(dv), _ptr(workspace),
                             workspace.numel() * workspace.element_size(), objective, reps, ms, best,
                             _stream(stream) if stream != 0 else None), "fbl_attn_tune")
    return tuple(best), {t: ms[t] for t in range(cap) if ms[t] >= 0}, (o, lse, dq, dk, dv)


def attn_tuned_tile(pass_: int, lq: Layout, lk: Layout, mask_kind: int) -> int:
    """The tile fbl_attn_tune chose for this pass and shape in this process, or -1."""
    return LIB.fbl_attn_tuned_tile(pass_, ctypes.byref(lq), ctypes.byref(lk), mask_kind)


def attn_tune_reset() -> None:
    LIB.fbl_attn_tune_reset()


NOALLOC_SCRATCH_BYTES = 64 << 20  # FBL_NOALLOC_SCRATCH_BYTES


def fbl_attn_bwd_noalloc_raw(lq, q, lk, k, lv, v, lo, o, ldo, do, lse, scale, mask: Mask, ldq, dq, ldk, dk, ldv,
                             dv, stream=None) -> int:
    """Direct call of fbl_attn_bwd_noalloc; returns the status."""
    ref = lambda l: ctypes.byref(l) if l is not None else None
    return LIB.fbl_attn_bwd_noalloc(ref(lq), _ptr(q), ref(lk), _ptr(k), ref(lv), _ptr(v), ref(lo), _ptr(o), ref(ldo),
                                    _ptr(do), _ptr(lse), float(scale), mask, ref(ldq), _ptr(dq), ref(ldk), _ptr(dk),
                                    ref(ldv), _ptr(dv), _stream(stream) if stream != 0 else None)


def attn_bwd_noalloc(q, k, v, o, do, lse, Hq: int, Hkv: int, dq, dk, dv, scale: Optional[float] = None,
                     causal: bool = False, kv_len=None, stream=None):
    """Backward through fbl_attn_bwd_noalloc: the library's own device scratch
    replaces the workspace, so nothing is allocated; dq, dk, dv are the
    caller's preallocated outputs (shapes and dtypes of q, k, v)."""
    _check_kv_len(kv_len, q.shape[0], "attn_bwd_noalloc")
    _check_device("attn_bwd_noalloc", stream, q=q, k=k, v=v, o=o, do=do, lse=lse, kv_len=kv_len, dq=dq, dk=dk,
                  dv=dv)
    if q.dim() == 3:
        _check_lse(lse, q.shape[0], Hq, q.shape[1], "attn_bwd_noalloc")
    lq, lk, lv = _layout(q, Hq), _layout(k, Hkv), _layout(v, Hkv)
    lo, ldo = _layout(o, Hq), _layout(do, Hq)
    ldq, ldk, ldv = _layout(dq, Hq), _layout(dk, Hkv), _layout(dv, Hkv)
    if scale is None:
        scale = 1.0 / math.sqrt(lq.D)
    _check(fbl_attn_bwd_noalloc_raw(lq, q, lk, k, lv, v, lo, o, ldo, do, lse, scale, _mask(causal, kv_len), ldq, dq,
                                    ldk, dk, ldv, dv, stream), "fbl_attn_bwd_noalloc")
    return dq, dk, dv


# ------------------------------------------------- packed QKV projection output
def _packed(qkv, Hq: int, Hkv: int):
    import torch
    if qkv.dim() != 3 or qkv.stride(2) != 1 or qkv.stride(1) != qkv.shape[2]:
        raise FblError(FBL_ERR_LAYOUT, "expected a [B, S, (Hq + 2 Hkv) D] tensor with contiguous rows")
    B, S, W = qkv.shape
    if W % (Hq + 2 * Hkv):
        raise FblError(FBL_ERR_SHAPE, f"row width {W} not divisible by Hq + 2 Hkv = {Hq + 2 * Hkv}")
    D = W // (Hq + 2 * Hkv)
    lq, lk, lv, ko, vo = fbl_layout_packed_qkv(_dtype_code(qkv), B, S, Hq, Hkv, D,
                                               batch_stride=qkv.stride(0) if B > 1 else 0)
    es = qkv.element_size()
    base = qkv.data_ptr()
    return lq, lk, lv, base, base + ko * es, base + vo * es


def attn_fwd_packed(qkv, Hq: int, Hkv: int, scale: Optional[float] = None, causal: bool = False, kv_len=None,
                    out=None, lse=None, stream=None):
    """Forward on a packed QKV projection output [B, S, (Hq + 2 Hkv) D]: Q, K and
    V are read in place through fbl_layout_packed_qkv descriptors.  Returns
    (O [B, S, Hq D], LSE [B, Hq, S])."""
    done = _FAST.attn_fwd_packed(qkv, Hq, Hkv, scale, causal, kv_len, out, lse, stream)
    if done is not None:
        return done
    import torch
    _check_kv_len(kv_len, qkv.shape[0], "attn_fwd_packed")
    _check_device("attn_fwd_packed", stream, qkv=qkv, kv_len=kv_len, out=out, lse=lse)
    if qkv.dim() == 3:
        _check_lse(lse, qkv.shape[0], Hq, qkv.shape[1], "attn_fwd_packed")
    lq, lk, lv, pq, pk, pv = _packed(qkv, Hq, Hkv)
    if scale is None:
        scale = 1.0 / math.sqrt(lq.D)
    B, S = qkv.shape[0], qkv.shape[1]
    if out is None:
        out = torch.empty((B, S, Hq * lq.D), dtype=qkv.dtype, device=qkv.device)
    if lse is None:
        lse = torch.empty((B, Hq, S), dtype=torch.float32, device=qkv.device)
    lo = _layout(out, Hq)
    _check(fbl_attn_fwd_raw(lq, pq, lk, pk, lv, pv, lo, out, lse, scale, _mask(causal, kv_len), stream),
           "fbl_attn_fwd")
    return out, lse


def attn_bwd_packed(qkv, o, do, lse, Hq: int, Hkv: int, scale: Optional[float] = None, causal: bool = False,
                    kv_len=None, dqkv=None, workspace=None, stream=None):
    """Backward on a packed QKV projection output: dQ, dK, dV are written into
    one packed gradient tensor shaped like ``qkv`` (allocated unless given)."""
    done = _FAST.attn_bwd_packed(qkv, o, do, lse, Hq, Hkv, scale, causal, kv_len, dqkv, workspace, stream)
    if done is not None:
        return done
    import torch
    _check_kv_len(kv_len, qkv.shape[0], "attn_bwd_packed")
    _check_device("attn_bwd_packed", stream, qkv=qkv, o=o, do=do, lse=lse, kv_len=kv_len, dqkv=dqkv,
                  workspace=workspace)
    if qkv.dim() == 3:
        _check_lse(lse, qkv.shape[0], Hq, qkv.shape[1], "attn_bwd_packed")
    _check_workspace(workspace, "attn_bwd_packed")
    lq, lk, lv, pq, pk, pv = _packed(qkv, Hq, Hkv)
    if scale is None:
        scale = 1.0 / math.sqrt(lq.D)
    if dqkv is None:
        dqkv = torch.empty(qkv.shape, dtype=qkv.dtype, device=qkv.device)
    if dqkv.shape != qkv.shape or dqkv.stride() != qkv.stride() or dqkv.dtype != qkv.dtype:
        raise FblError(FBL_ERR_SHAPE, "dqkv must have qkv's shape, strides and dtype")
    _, _, _, gq, gk, gv = _packed(dqkv, Hq, Hkv)
    lo, ldo = _layout(o, Hq), _layout(do, Hq)
    if workspace is None:
        workspace = torch.empty(fbl_attn_bwd_workspace(lq, lk), dtype=torch.uint8, device=qkv.device)
    _check(fbl_attn_bwd_raw(lq, pq, lk, pk, lv, pv, lo, o, ldo, do, lse, scale, _mask(causal, kv_len), lq, gq, lk,
                            gk, lv, gv, workspace, workspace.numel() * workspace.element_size(), stream),
           "fbl_attn_bwd")
    return dqkv


# ------------------------------------------------------- projection products
def fbl_proj_raw(op, M, K, N, a, lda, b, ldb, c, ldc, tile=FBL_GEMM_TILE_AUTO, stream=None) -> int:
    """Direct call of fbl_proj; returns the status code."""
    return LIB.fbl_proj(op, M, K, N, _ptr(a), lda, _ptr(b), ldb, _ptr(c), ldc, tile,
                        _stream(stream) if stream != 0 else None)


def _rows(t, name):
    if t.dim() != 2 or t.stride(1) != 1:
        raise FblError(FBL_ERR_LAYOUT, f"{name}: expected a 2-D row-major tensor (inner stride 1)")
    return t.shape[0], t.shape[1], t.stride(0)


def _proj_shape(op, a, b, out=None):
    """(M, K, N, result shape, lda, ldb) of a product.  Both operands state one of its
    extents and `out`, where given, has the result's shape: the library takes addresses
    and extents alone, so what disagrees here would be read or written past its end."""
    ra, wa, lda = _rows(a, "a")
    rb, wb, ldb = _rows(b, "b")
    if op == FBL_PROJ_FWD:
        M, K, N, shape, other = ra, wa, wb, (ra, wb), rb == wa
    elif op == FBL_PROJ_BWD_DATA:
        M, N, K, shape, other = ra, wa, rb, (ra, rb), wb == wa
    else:
        M, K, N, shape, other = ra, wa, wb, (wa, wb), rb == ra
    if not other:
        raise FblError(FBL_ERR_SHAPE, f"proj: operands {(ra, wa)} and {(rb, wb)} do not agree for op {op}")
    if out is not None and tuple(out.shape) != shape:
        raise FblError(FBL_ERR_SHAPE, f"proj: out has shape {tuple(out.shape)}, the result is {shape}")
    return M, K, N, shape, lda, ldb


def proj(op: int, a, b, out=None, tile: int = FBL_GEMM_TILE_AUTO, stream=None):
    """One projection product on 2-D bf16 or fp32 tensors (row-major, any row stride):
    FBL_PROJ_FWD (a = X [M, K], b = W [K, N]) -> Y [M, N];
    FBL_PROJ_BWD_DATA (a = dY [M, N], b = W [K, N]) -> dX [M, K];
    FBL_PROJ_BWD_WEIGHT (a = X [M, K], b = dY [M, N]) -> dW [K, N]."""
    done = _FAST.proj(op, a, b, out, tile, stream)
    if done is not None:
        return done
    import torch
    _check_device("proj", stream, a=a, b=b, out=out)
    M, K, N, shape, lda, ldb = _proj_shape(op, a, b, out)
    if out is None:
        out = torch.empty(shape, dtype=a.dtype, device=a.device)
    _, _, ldc = _rows(out, "out")
    if not (a.dtype == b.dtype == out.dtype):
        raise FblError(FBL_ERR_DTYPE, f"proj: operand dtypes differ ({a.dtype}, {b.dtype}, {out.dtype})")
    if a.dtype == torch.float32:
        _check(LIB.fbl_proj_dt(op, FBL_F32, M, K, N, _ptr(a), lda, _ptr(b), ldb, _ptr(out), ldc, tile,
                               _stream(stream) if stream != 0 else None), "fbl_proj_dt")
    else:
        _check(fbl_proj_raw(op, M, K, N, a, lda, b, ldb, out, ldc, tile, stream), "fbl_proj")
    return out


def gemm_tiles():
    """Every tile configuration: {id: dict(bm, bn, bk, stages, wm, wn, wk, lds_bytes)}."""
    keys = ("bm", "bn", "bk", "stages", "wm", "wn", "wk", "lds_bytes")
    out = {}
    for t in range(LIB.fbl_gemm_tile_count()):
        info = (ctypes.c_int32 * 8)()
        _check(LIB.fbl_gemm_tile_info(t, info), "fbl_gemm_tile_info")
        out[t] = dict(zip(keys, list(info)))
    return out


def proj_candidates(op: int, M: int, K: int, N: int):
    """Candidate tile ids of one product shape (the C1/C2/C3 filters)."""
    n = ctypes.c_int32()
    cap = LIB.fbl_gemm_tile_count()
    ids = (ctypes.c_int32 * cap)()
    _check(LIB.fbl_proj_candidates(op, M, K, N, ids, cap, ctypes.byref(n)), "fbl_proj_candidates")
    return list(ids[:n.value])


def proj_tune(op: int, a, b, out, objective: int = FBL_TUNE_TIME, reps: int = 10, stream=None):
    """Measured tile selection for one product (fbl_proj_tune).  Returns
    (chosen id, {id: average ms} over the candidates); `out` then holds the
    product computed with the chosen tile.  Where proj_auto_tile is no candidate,
    the untuned choice may be the faster one."""
    _check_device("proj_tune", stream, a=a, b=b, out=out)
    M, K, N, _, lda, ldb = _proj_shape(op, a, b, out)
    _, _, ldc = _rows(out, "out")
    cap = LIB.fbl_gemm_tile_count()
    ms = (ctypes.c_float * cap)()
    best = ctypes.c_int32(-1)
    _check(LIB.fbl_proj_tune(op, M, K, N, _ptr(a), lda, _ptr(b), ldb, _ptr(out), ldc, objective, reps, ms,
                             ctypes.byref(best), _stream(stream) if stream != 0 else None), "fbl_proj_tune")
    return best.value, {t: ms[t] for t in range(cap) if ms[t] >= 0}


def proj_tuned_tile(op: int, M: int, K: int, N: int) -> int:
    """The tile fbl_proj_tune chose for this shape in this process, or -1."""
    return LIB.fbl_proj_tuned_tile(op, M, K, N)


def proj_auto_tile(op: int, M: int, K: int, N: int) -> int:
    """The tile id FBL_GEMM_TILE_AUTO resolves to for this bf16 product."""
    t = ctypes.c_int32(-1)
    _check(LIB.fbl_proj_auto_tile(op, M, K, N, ctypes.byref(t)), "fbl_proj_auto_tile")
    return t.value


def proj_float_tile(op: int, M: int, K: int, N: int):
    """The tile an fp32 product runs: dict(bm, bn, bk, waves, wk, workgroups)."""
    info = (ctypes.c_int32 * 6)()
    _check(LIB.fbl_proj_float_tile(op, M, K, N, info), "fbl_proj_float_tile")
    return dict(zip(("bm", "bn", "bk", "waves", "wk", "workgroups"), list(info)))


def proj_tune_reset() -> None:
    LIB.fbl_proj_tune_reset()


# ---------------------------------------------------------------- layer norm
def _matrix(t, where: str, name: str, shape=None, like=None):
    """Row stride of a 2-D tensor with unit inner stride, of `shape` and of `like`'s dtype
    where given.  (The stride of a single row means nothing: its width, in whole 16-byte chunks.)"""
    if t.dim() != 2:
        raise FblError(FBL_ERR_SHAPE, f"{where}: {name} must be 2-D, got shape {tuple(t.shape)}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise FblError(FBL_ERR_SHAPE, f"{where}: {name} has shape {tuple(t.shape)}, needs {tuple(shape)}")
    if like is not None and t.dtype != like.dtype:
        raise FblError(FBL_ERR_DTYPE, f"{where}: {name} is {t.dtype}, needs {like.dtype}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise FblError(FBL_ERR_LAYOUT, f"{where}: {name} needs inner stride 1, got strides {t.stride()}")
    return t.stride(0) if t.shape[0] > 1 else -(-t.shape[1] // 8) * 8


def _vector(t, where: str, name: str, n: int, dtype):
    """A contiguous 1-D tensor of n entries of `dtype`, or None."""
    if t is None:
        return
    if t.dtype != dtype:
        raise FblError(FBL_ERR_DTYPE, f"{where}: {name} is {t.dtype}, needs {dtype}")
    if tuple(t.shape) != (n,):
        raise FblError(FBL_ERR_SHAPE, f"{where}: {name} has shape {tuple(t.shape)}, needs {(n,)}")
    if n > 1 and t.stride(0) != 1:
        raise FblError(FBL_ERR_LAYOUT, f"{where}: {name} must be contiguous")


def _empty(shape, dtype, like, stream, result: bool = True):
    """New memory for work on `stream` (None: the current one).  Another stream's comes from that stream's own pool:
    a block of the current stream's may still be in use by work that is queued there.  A
    result is known to the current stream too, whose program reads it."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    here = torch.cuda.current_stream(like.device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=like.device) if stream else torch.cuda.default_stream(like.device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=like.device)
    if result:
        t.record_stream(here)
    return t


def _scratch(workspace, need: int, where: str, like, stream):
    """(workspace, its bytes): the caller's, or one allocated for this call."""
    import torch
    _check_workspace(workspace, where)
    if workspace is None:
        workspace = _empty(need, torch.uint8, like, stream, result=False)
    return workspace, workspace.numel() * workspace.element_size()


def _call(name: str, like, stream, *args) -> None:
    """One call of the library on `stream`, with like's device current (a stream given may be another's than the
    program's current one)."""
    import torch
    f, args = getattr(LIB, name), args + (_stream(stream) if stream != 0 else None,)
    if stream is not None and like.device.index != torch.cuda.current_device():
        with torch.cuda.device(like.device):
            status = f(*args)
    else:
        status = f(*args)
    _check(status, name)


def layer_norm_fwd(x, weight=None, bias=None, eps: float = 1e-5, out=None, mean=None, rstd=None, stream=None):
    """Layer norm of the rows of x [M, N] (any row stride): returns (y, mean, rstd), mean
    and rstd float32 [M].  weight and bias [N], in x's dtype, may be None."""
    done = _FAST.layer_norm_fwd(x, weight, bias, eps, out, mean, rstd, stream)
    if done is not None:
        return done
    import torch
    where = "layer_norm_fwd"
    _check_device(where, stream, x=x, weight=weight, bias=bias, out=out, mean=mean, rstd=rstd)
    ldx = _matrix(x, where, "x")
    M, N = x.shape
    dt = _dtype_code(x)
    _vector(weight, where, "weight", N, x.dtype)
    _vector(bias, where, "bias", N, x.dtype)
    if out is None:
        out = _empty((M, N), x.dtype, x, stream)
    ldy = _matrix(out, where, "out", (M, N), x)
    if mean is None:
        mean = _empty(M, torch.float32, x, stream)
    if rstd is None:
        rstd = _empty(M, torch.float32, x, stream)
    _vector(mean, where, "mean", M, torch.float32)
    _vector(rstd, where, "rstd", M, torch.float32)
    _call("fbl_layer_norm_fwd", x, stream, dt, M, N, _ptr(x), ldx, _ptr(weight), _ptr(bias), float(eps), _ptr(out),
          ldy, _ptr(mean), _ptr(rstd))
    return out, mean, rstd


def layer_norm_bwd_workspace(x) -> int:
    """Bytes of layer_norm_bwd's workspace for rows like x's."""
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_layer_norm_bwd_workspace(_dtype_code(x), *x.shape, ctypes.byref(n)), "fbl_layer_norm_bwd_workspace")
    return int(n.value)


def layer_norm_bwd(dy, x, mean, rstd, weight=None, dx=None, dweight=None, dbias=None, workspace=None, stream=None,
                   need_weight: bool = True, need_bias: bool = True):
    """Gradients of layer_norm_fwd's rows: returns (dx, dweight, dbias), the last two
    None where not needed.  mean and rstd are the forward's."""
    done = _FAST.layer_norm_bwd(dy, x, mean, rstd, weight, dx, dweight,
                                   dbias, workspace, stream, need_weight, need_bias)
    if done is not None:
        return done
    import torch
    where = "layer_norm_bwd"
    _check_device(where, stream, dy=dy, x=x, mean=mean, rstd=rstd, weight=weight, dx=dx, dweight=dweight, dbias=dbias,
                  workspace=workspace)
    ldx = _matrix(x, where, "x")
    M, N = x.shape
    dt = _dtype_code(x)
    lddy = _matrix(dy, where, "dy", (M, N), x)
    _vector(mean, where, "mean", M, torch.float32)
    _vector(rstd, where, "rstd", M, torch.float32)
    _vector(weight, where, "weight", N, x.dtype)
    if dx is None:
        dx = _empty((M, N), x.dtype, x, stream)
    lddx = _matrix(dx, where, "dx", (M, N), x)
    if dweight is None and need_weight:
        dweight = _empty(N, x.dtype, x, stream)
    if dbias is None and need_bias:
        dbias = _empty(N, x.dtype, x, stream)
    _vector(dweight, where, "dweight", N, x.dtype)
    _vector(dbias, where, "dbias", N, x.dtype)
    ws, ws_bytes = None, 0
    if dweight is not None or dbias is not None:
        need = 0 if workspace is not None else layer_norm_bwd_workspace(x)
        ws, ws_bytes = _scratch(workspace, need, where, x, stream)
    _call("fbl_layer_norm_bwd", x, stream, dt, M, N, _ptr(dy), lddy, _ptr(x), ldx, _ptr(weight), _ptr(mean),
          _ptr(rstd), _ptr(dx), lddx, _ptr(dweight), _ptr(dbias), _ptr(ws), ws_bytes)
    return dx, dweight, dbias


# ------------------------------------- linear layers: bias, activation, residual
def _act_code(act, where: str) -> int:
    code = ACTIVATIONS.get(act)
    if code is None:
        raise FblError(FBL_ERR_ARG, f"{where}: no activation {act!r}, there are {', '.join(ACTIVATIONS)}")
    return code


def linear_fwd_workspace(x, w) -> int:
    """Bytes of linear_fwd's workspace for x [M, K] and w [K, N]: 0 but for a few tokens."""
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_linear_fwd_workspace(_dtype_code(x), *x.shape, w.shape[1], ctypes.byref(n)), "fbl_linear_fwd_workspace")
    return int(n.value)


def linear_fwd(x, w, bias=None, act: str = "none", residual=None, out=None, z=None, tile: int = FBL_GEMM_TILE_AUTO,
               workspace=None, stream=None):
    """y = act(x w + bias) + residual for x [M, K], w [K, N], bias [N], residual [M, N] (any row
    strides, one storage type), act one of ACTIVATIONS.  z [M, N], where given, receives the
    pre-activation, which linear_bwd needs for every act but "none".  workspace: linear_fwd_workspace bytes, allocated
    where they are needed and it is None.  Returns y."""
    done = _FAST.linear_fwd(x, w, bias, act, residual, out, z, tile, workspace, stream)
    if done is not None:
        return done
    import torch
    where = "linear_fwd"
    _check_device(where, stream, x=x, w=w, bias=bias, residual=residual, out=out, z=z, workspace=workspace)
    ldx = _matrix(x, where, "x")
    M, K = x.shape
    dt, code = _dtype_code(x), _act_code(act, where)
    ldw = _matrix(w, where, "w", None, x)
    N = w.shape[1]
    if w.shape[0] != K:
        raise FblError(FBL_ERR_SHAPE, f"{where}: x {tuple(x.shape)} and w {tuple(w.shape)} do not agree")
    _vector(bias, where, "bias", N, x.dtype)
    ldr = 0 if residual is None else _matrix(residual, where, "residual", (M, N), x)
    ldz = 0 if z is None else _matrix(z, where, "z", (M, N), x)
    if out is None:
        out = _empty((M, N), x.dtype, x, stream)
    ldy = _matrix(out, where, "out", (M, N), x)
    ws, ws_bytes = None, 0
    need = linear_fwd_workspace(x, w) if workspace is None and M <= 128 and tile == FBL_GEMM_TILE_AUTO else 0
    if workspace is not None or need:
        ws, ws_bytes = _scratch(workspace, need, where, x, stream)
    _call("fbl_linear_fwd", x, stream, dt, code, M, K, N, _ptr(x), ldx, _ptr(w), ldw, _ptr(bias), _ptr(residual), ldr,
          _ptr(out), ldy, _ptr(z), ldz, tile, _ptr(ws), ws_bytes)
    return out


def linear_bwd_workspace(x, w) -> int:
    """Bytes of linear_bwd's workspace for x [M, K] and w [K, N]."""
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_linear_bwd_workspace(_dtype_code(x), *x.shape, w.shape[1], ctypes.byref(n)), "fbl_linear_bwd_workspace")
    return int(n.value)


def linear_bwd(dy, x, w, z=None, act: str = "none", dx=None, dw=None, dbias=None, workspace=None, stream=None,
               need_dx: bool = True, need_dw: bool = True, need_bias: bool = True, x_act: str = "none", x_z=None, dxbias=None):
    """Gradients of linear_fwd: returns (dx, dw, dbias), each None where not needed.  z is the
    forward's pre-activation (None for act "none"); the residual's gradient is dy.  Where x
    itself is x_act(x_z), dx can be the gradient of x_z; dxbias [K], where given, receives the
    sums of dx over its rows, then the gradient of the bias in x_z."""
    done = _FAST.linear_bwd(dy, x, w, z, act, dx, dw, dbias, workspace, stream, need_dx, need_dw, need_bias, x_act, x_z,
                            dxbias)
    if done is not None:
        return done
    import torch
    where = "linear_bwd"
    _check_device(where, stream, dy=dy, x=x, w=w, z=z, dx=dx, dw=dw, dbias=dbias, workspace=workspace, x_z=x_z,
                  dxbias=dxbias)
    ldx = _matrix(x, where, "x")
    M, K = x.shape
    dt, code, xcode = _dtype_code(x), _act_code(act, where), _act_code(x_act, where)
    ldw = _matrix(w, where, "w", None, x)
    N = w.shape[1]
    if w.shape[0] != K:
        raise FblError(FBL_ERR_SHAPE, f"{where}: x {tuple(x.shape)} and w {tuple(w.shape)} do not agree")
    lddy = _matrix(dy, where, "dy", (M, N), x)
    ldz = 0 if z is None else _matrix(z, where, "z", (M, N), x)
    ldxz = 0 if x_z is None else _matrix(x_z, where, "x_z", (M, K), x)
    if dx is None and need_dx:
        dx = _empty((M, K), x.dtype, x, stream)
    if dw is None and need_dw:
        dw = _empty((K, N), x.dtype, x, stream)
    if dbias is None and need_bias:
        dbias = _empty(N, x.dtype, x, stream)
    lddx = 0 if dx is None else _matrix(dx, where, "dx", (M, K), x)
    lddw = 0 if dw is None else _matrix(dw, where, "dw", (K, N), x)
    _vector(dbias, where, "dbias", N, x.dtype)
    _vector(dxbias, where, "dxbias", K, x.dtype)
    ws, ws_bytes = None, 0
    if code != FBL_ACT_NONE or dbias is not None or dxbias is not None or workspace is not None \
            or (dx is not None and M <= 128) or (dw is not None and K * N <= 1 << 19):
        need = 0 if workspace is not None else linear_bwd_workspace(x, w)
        ws, ws_bytes = _scratch(workspace, need, where, x, stream)
    _call("fbl_linear_bwd", x, stream, dt, code, M, K, N, _ptr(dy), lddy, _ptr(x), ldx, _ptr(w), ldw, _ptr(z), ldz,
          xcode, _ptr(x_z), ldxz, _ptr(dx), lddx, _ptr(dxbias), _ptr(dw), lddw, _ptr(dbias), _ptr(ws), ws_bytes)
    return dx, dw, dbias


# ------------------------------------------------------------------ gated layers
def _gated_width(w, where: str) -> int:
    if w.dim() != 2 or w.shape[1] % 2:
        raise FblError(FBL_ERR_SHAPE, f"{where}: w has shape {tuple(w.shape)}, needs [K, 2 F], gate then up columns")
    return w.shape[1] // 2


def gated_fwd_workspace(x, w) -> int:
    """Bytes of gated_fwd's workspace for x [M, K] and w [K, 2F]: 0 but for a few tokens."""
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_gated_fwd_workspace(_dtype_code(x), *x.shape, _gated_width(w, "gated_fwd_workspace"), ctypes.byref(n)),
           "fbl_gated_fwd_workspace")
    return int(n.value)


def gated_fwd(x, w, bias=None, act: str = "silu", out=None, factors=None, tile: int = FBL_GEMM_TILE_AUTO, workspace=None,
              stream=None):
    """h = act(gate) * up with (gate, up) = x w + bias for x [M, K], w [K, 2F] and bias [2F], gate then up columns (any row
    strides, one storage type), act one of ACTIVATIONS.  factors [M, 2F], where given, receives h's derivatives by gate
    and by up, which gated_bwd needs (bfloat16: in a form of the library's own, two bytes a value).  workspace:
    gated_fwd_workspace bytes, allocated where they are needed and it is None.  Returns h [M, F]."""
    done = _FAST.gated_fwd(x, w, bias, act, out, factors, tile, workspace, stream)
    if done is not None:
        return done
    import torch
    where = "gated_fwd"
    _check_device(where, stream, x=x, w=w, bias=bias, out=out, factors=factors, workspace=workspace)
    ldx = _matrix(x, where, "x")
    M, K = x.shape
    dt, code = _dtype_code(x), _act_code(act, where)
    ldw = _matrix(w, where, "w", None, x)
    F = _gated_width(w, where)
    if w.shape[0] != K:
        raise FblError(FBL_ERR_SHAPE, f"{where}: x {tuple(x.shape)} and w {tuple(w.shape)} do not agree")
    _vector(bias, where, "bias", 2 * F, x.dtype)
    ldf = 0 if factors is None else _matrix(factors, where, "factors", (M, 2 * F), x)
    if out is None:
        out = _empty((M, F), x.dtype, x, stream)
    ldh = _matrix(out, where, "out", (M, F), x)
    ws, ws_bytes = None, 0
    need = gated_fwd_workspace(x, w) if workspace is None and M <= 128 and tile == FBL_GEMM_TILE_AUTO else 0
    if workspace is not None or need:
        ws, ws_bytes = _scratch(workspace, need, where, x, stream)
    _call("fbl_gated_fwd", x, stream, dt, code, M, K, F, _ptr(x), ldx, _ptr(w), ldw, _ptr(bias), _ptr(out), ldh,
          _ptr(factors), ldf, tile, _ptr(ws), ws_bytes)
    return out


def gated_bwd_workspace(dy, w_down) -> int:
    """Bytes of gated_bwd's workspace for dy [M, N] and w_down [F, N]."""
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_gated_bwd_workspace(_dtype_code(dy), dy.shape[0], *w_down.shape, ctypes.byref(n)),
           "fbl_gated_bwd_workspace")
    return int(n.value)


def gated_bwd(dy, w_down, factors, dz=None, dbias=None, tile: int = FBL_GEMM_TILE_AUTO, workspace=None, stream=None,
              need_bias: bool = True):
    """Gradient of a gated layer's pre-activations from that of the block's result: dy [M, N], w_down [F, N] and the
    forward's factors [M, 2F] give dz [M, 2F] and the sums of dz over its rows, dbias [2F].  Returns (dz, dbias), dbias
    None where not needed.  dx and dw are linear_bwd's of dz."""
    done = _FAST.gated_bwd(dy, w_down, factors, dz, dbias, tile, workspace, stream, need_bias)
    if done is not None:
        return done
    import torch
    where = "gated_bwd"
    _check_device(where, stream, dy=dy, w_down=w_down, factors=factors, dz=dz, dbias=dbias, workspace=workspace)
    lddy = _matrix(dy, where, "dy")
    M, N = dy.shape
    dt = _dtype_code(dy)
    ldwd = _matrix(w_down, where, "w_down", None, dy)
    F = w_down.shape[0]
    if w_down.shape[1] != N:
        raise FblError(FBL_ERR_SHAPE, f"{where}: dy {tuple(dy.shape)} and w_down {tuple(w_down.shape)} do not agree")
    ldf = _matrix(factors, where, "factors", (M, 2 * F), dy)
    if dz is None:
        dz = _empty((M, 2 * F), dy.dtype, dy, stream)
    lddz = _matrix(dz, where, "dz", (M, 2 * F), dy)
    if dbias is None and need_bias:
        dbias = _empty(2 * F, dy.dtype, dy, stream)
    _vector(dbias, where, "dbias", 2 * F, dy.dtype)
    ws, ws_bytes = None, 0
    if dbias is not None or workspace is not None or M <= 128:
        need = 0 if workspace is not None else gated_bwd_workspace(dy, w_down)
        ws, ws_bytes = _scratch(workspace, need, where, dy, stream)
    _call("fbl_gated_bwd", dy, stream, dt, M, F, N, _ptr(dy), lddy, _ptr(w_down), ldwd, _ptr(factors), ldf, _ptr(dz), lddz,
          _ptr(dbias), tile, _ptr(ws), ws_bytes)
    return dz, dbias


# ------------------------------------- losses of a linear head over a vocabulary
def _head(w, x, where: str, name: str = "w"):
    """(order, row stride) of a head's weight [K, V]: stored by rows of V, or, as the
    transposed view of a table, by rows of K."""
    if w.dim() != 2:
        raise FblError(FBL_ERR_SHAPE, f"{where}: {name} must be 2-D, got shape {tuple(w.shape)}")
    if w.dtype != x.dtype:
        raise FblError(FBL_ERR_DTYPE, f"{where}: {name} is {w.dtype}, needs {x.dtype}")
    K, V = w.shape
    if K != x.shape[1]:
        raise FblError(FBL_ERR_SHAPE, f"{where}: x {tuple(x.shape)} and {name} {tuple(w.shape)} do not agree")
    if w.stride(1) == 1 and (K == 1 or w.stride(0) >= V):
        return FBL_HEAD_KV, (w.stride(0) if K > 1 else max(w.stride(0), V))
    if w.stride(0) == 1 or K == 1:
        return FBL_HEAD_VK, (w.stride(1) if V > 1 else max(w.stride(1), K))
    raise FblError(FBL_ERR_LAYOUT, f"{where}: {name} [K, V] needs rows of V or, as a table's transposed view, of K, got "
                                   f"strides {w.stride()}")


def linear_loss_workspace(x, w, top: int = 1) -> int:
    """Bytes of the workspace of linear_ce_fwd and _bwd (top 1) or linear_kd_fwd and _bwd."""
    order, ldw = _head(w, x, "linear_loss_workspace")
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_linear_loss_workspace(_dtype_code(x), order, *x.shape, w.shape[1], top, ldw, ctypes.byref(n)),
           "fbl_linear_loss_workspace")
    return int(n.value)


def _new_f32(t, n: int, like, where: str, name: str, stream):
    import torch
    if t is None:
        t = _empty(n, torch.float32, like, stream)
    _vector(t, where, name, n, torch.float32)
    return t


def _loss_scratch(workspace, x, w, top: int, where: str, stream):
    need = 0 if workspace is not None else linear_loss_workspace(x, w, top)
    return _scratch(workspace, need, where, x, stream)


def _mean_ptr(mean, where: str):
    import torch
    if mean is None:
        return None
    if mean.dtype != torch.float32 or mean.numel() != 1:
        raise FblError(FBL_ERR_SHAPE, f"{where}: mean must be one float32")
    return _ptr(mean)


def _dloss(dloss, M: int, where: str) -> int:
    """Stride of the loss' gradient: one number, or one a row."""
    import torch
    if dloss.dtype != torch.float32:
        raise FblError(FBL_ERR_DTYPE, f"{where}: dloss is {dloss.dtype}, needs torch.float32")
    if dloss.dim() == 0 or tuple(dloss.shape) == (1,) and M != 1:
        return 0
    if tuple(dloss.shape) != (M,):
        raise FblError(FBL_ERR_SHAPE, f"{where}: dloss has shape {tuple(dloss.shape)}, needs () or {(M,)}")
    return dloss.stride(0)


def _head_grads(x, w, dx, dw, need_dx: bool, need_dw: bool, order: int, where: str, stream):
    """(dx, its row stride, dw, its row stride): the given ones, or new ones where needed."""
    import torch
    if dx is None and need_dx:
        dx = _empty(x.shape, x.dtype, x, stream)
    lddx = 0 if dx is None else _matrix(dx, where, "dx", x.shape, x)
    if dw is None and need_dw:
        K, V = w.shape
        dw = (_empty((V, K), x.dtype, x, stream).t() if order == FBL_HEAD_VK else
              _empty((K, V), x.dtype, x, stream))
    lddw = 0
    if dw is not None:
        if tuple(dw.shape) != tuple(w.shape):
            raise FblError(FBL_ERR_SHAPE, f"{where}: dw has shape {tuple(dw.shape)}, needs {tuple(w.shape)}")
        dorder, lddw = _head(dw, x, where, "dw")
        if dorder != order:
            raise FblError(FBL_ERR_LAYOUT, f"{where}: dw must be stored by the same rows as w")
    return dx, lddx, dw, lddw


def linear_ce_fwd(x, w, labels, ignore_index: int = -100, loss=None, lse=None, total=None, mean=None, workspace=None,
                  stream=None):
    """Softmax cross entropy of the logits x w, which are never kept: x [M, K], w [K, V] (rows of V,
    or the transposed view of a [V, K] table), labels int64 [M].  Returns (loss, lse, total): each row's loss and
    log-sum-exp, float32 [M], and [their sum, the number of rows that count].  Rows labelled
    ignore_index do not count; a label outside the vocabulary makes its row's loss nan.  mean: one float32 that
    receives total[0] / total[1]."""
    done = _FAST.linear_ce_fwd(x, w, labels, ignore_index, loss, lse, total, mean, workspace, stream)
    if done is not None:
        return done
    import torch
    where = "linear_ce_fwd"
    _check_device(where, stream, x=x, w=w, labels=labels, loss=loss, lse=lse, total=total, mean=mean, workspace=workspace)
    ldx = _matrix(x, where, "x")
    M, K = x.shape
    dt = _dtype_code(x)
    order, ldw = _head(w, x, where)
    _vector(labels, where, "labels", M, torch.int64)
    loss, lse = _new_f32(loss, M, x, where, "loss", stream), _new_f32(lse, M, x, where, "lse", stream)
    total = _new_f32(total, 2, x, where, "total", stream)
    ws, ws_bytes = _loss_scratch(workspace, x, w, 1, where, stream)
    _call("fbl_linear_ce_fwd", x, stream, dt, order, M, K, w.shape[1], _ptr(x), ldx, _ptr(w), ldw, _ptr(labels),
          ignore_index, _ptr(loss), _ptr(lse), _ptr(total), _mean_ptr(mean, where), _ptr(ws), ws_bytes)
    return loss, lse, total


def linear_ce_bwd(dloss, x, w, labels, lse, total=None, ignore_index: int = -100, dx=None, dw=None, workspace=None,
                  stream=None, need_dx: bool = True, need_dw: bool = True):
    """Gradients (dx, dw) of linear_ce_fwd, each None where not needed; dw is stored as w is.  dloss,
    float32, is the gradient of each row's loss ([M], or one number for all), or with the
    forward's total that of the mean over the rows that count."""
    done = _FAST.linear_ce_bwd(dloss, x, w, labels, lse, total, ignore_index,
                                  dx, dw, workspace, stream, need_dx, need_dw)
    if done is not None:
        return done
    import torch
    where = "linear_ce_bwd"
    _check_device(where, stream, dloss=dloss, x=x, w=w, labels=labels, lse=lse, total=total, dx=dx, dw=dw,
                  workspace=workspace)
    ldx = _matrix(x, where, "x")
    M, K = x.shape
    dt = _dtype_code(x)
    order, ldw = _head(w, x, where)
    _vector(labels, where, "labels", M, torch.int64)
    _vector(lse, where, "lse", M, torch.float32)
    _vector(total, where, "total", 2, torch.float32)
    gstride = _dloss(dloss, M, where)
    dx, lddx, dw, lddw = _head_grads(x, w, dx, dw, need_dx, need_dw, order, where, stream)
    ws, ws_bytes = _loss_scratch(workspace, x, w, 1, where, stream)
    _call("fbl_linear_ce_bwd", x, stream, dt, order, M, K, w.shape[1], _ptr(dloss), gstride, _ptr(total), _ptr(x),
          ldx, _ptr(w), ldw, _ptr(labels), ignore_index, _ptr(lse), _ptr(dx), lddx, _ptr(dw), lddw, _ptr(ws),
          ws_bytes)
    return dx, dw


def _teacher(index, logits, x, where: str):
    """(top, row strides of index and logits, logits' dtype code)."""
    import torch
    if index.dim() != 2 or index.shape[0] != x.shape[0]:
        raise FblError(FBL_ERR_SHAPE, f"{where}: index has shape {tuple(index.shape)}, needs ({x.shape[0]}, top)")
    if index.dtype != torch.int64:
        raise FblError(FBL_ERR_DTYPE, f"{where}: index is {index.dtype}, needs torch.int64")
    ldi = _matrix(index, where, "index")
    if logits is None:
        return index.shape[1], ldi, 0, 0
    ldl = _matrix(logits, where, "logits", index.shape)
    return index.shape[1], ldi, ldl, _dtype_code(logits)


def linear_kd_fwd(x, w, index, logits, temperature: float = 1.0, loss=None, lse=None, prob=None, total=None, mean=None,
                  workspace=None, stream=None):
    """Distillation from a teacher's top logits on the student's logits x w, which are never kept: index int64 and
    logits (float32 or bfloat16) [M, top] are the teacher's, loss[m] = T^2 sum p (log p - log q) with p = softmax(logits /
    T) over the row's entries and q = softmax(x w / T) over the vocabulary.  A negative index is an absent entry; a
    row without entries does not count.  The teacher is a constant: there is no gradient of its logits.  Returns (loss,
    lse, prob, total); prob float32 [M, top]."""
    done = _FAST.linear_kd_fwd(x, w, index, logits, temperature, loss, lse, prob, total, mean, workspace, stream)
    if done is not None:
        return done
    import torch
    where = "linear_kd_fwd"
    _check_device(where, stream, x=x, w=w, index=index, logits=logits, loss=loss, lse=lse, prob=prob, total=total, mean=mean,
                  workspace=workspace)
    ldx = _matrix(x, where, "x")
    M, K = x.shape
    dt = _dtype_code(x)
    order, ldw = _head(w, x, where)
    top, ldi, ldl, ldt = _teacher(index, logits, x, where)
    loss, lse = _new_f32(loss, M, x, where, "loss", stream), _new_f32(lse, M, x, where, "lse", stream)
    total = _new_f32(total, 2, x, where, "total", stream)
    if prob is None:
        prob = _empty((M, top), torch.float32, x, stream)
    _contiguous(prob, where, "prob", (M, top))
    ws, ws_bytes = _loss_scratch(workspace, x, w, top, where, stream)
    _call("fbl_linear_kd_fwd", x, stream, dt, order, M, K, w.shape[1], top, _ptr(x), ldx, _ptr(w), ldw, _ptr(index),
          ldi, ldt, _ptr(logits), ldl, float(temperature), _ptr(prob), _ptr(loss), _ptr(lse), _ptr(total),
          _mean_ptr(mean, where), _ptr(ws), ws_bytes)
    return loss, lse, prob, total


def _contiguous(t, where: str, name: str, shape):
    import torch
    if t.dtype != torch.float32:
        raise FblError(FBL_ERR_DTYPE, f"{where}: {name} is {t.dtype}, needs torch.float32")
    if tuple(t.shape) != tuple(shape):
        raise FblError(FBL_ERR_SHAPE, f"{where}: {name} has shape {tuple(t.shape)}, needs {tuple(shape)}")
    if not t.is_contiguous():
        raise FblError(FBL_ERR_LAYOUT, f"{where}: {name} must be contiguous")


def linear_kd_bwd(dloss, x, w, index, prob, lse, temperature: float = 1.0, total=None, dx=None, dw=None, workspace=None,
                  stream=None, need_dx: bool = True, need_dw: bool = True):
    """Gradients (dx, dw) of linear_kd_fwd from its prob and lse; the rest as linear_ce_bwd."""
    done = _FAST.linear_kd_bwd(dloss, x, w, index, prob, lse, temperature, total,
                                  dx, dw, workspace, stream, need_dx, need_dw)
    if done is not None:
        return done
    import torch
    where = "linear_kd_bwd"
    _check_device(where, stream, dloss=dloss, x=x, w=w, index=index, prob=prob, lse=lse, total=total, dx=dx, dw=dw,
                  workspace=workspace)
    ldx = _matrix(x, where, "x")
    M, K = x.shape
    dt = _dtype_code(x)
    order, ldw = _head(w, x, where)
    top, ldi, _, _ = _teacher(index, None, x, where)
    _contiguous(prob, where, "prob", (M, top))
    _vector(lse, where, "lse", M, torch.float32)
    _vector(total, where, "total", 2, torch.float32)
    gstride = _dloss(dloss, M, where)
    dx, lddx, dw, lddw = _head_grads(x, w, dx, dw, need_dx, need_dw, order, where, stream)
    ws, ws_bytes = _loss_scratch(workspace, x, w, top, where, stream)
    _call("fbl_linear_kd_bwd", x, stream, dt, order, M, K, w.shape[1], top, _ptr(dloss), gstride, _ptr(total),
          _ptr(x), ldx, _ptr(w), ldw, _ptr(index), ldi, float(temperature), _ptr(prob), _ptr(lse), _ptr(dx), lddx,
          _ptr(dw), lddw, _ptr(ws), ws_bytes)
    return dx, dw


# ---------------------- norms of queries and keys for each head, and their rotation
def rotary_frequencies(dims: int, base: float = 10000.0):
    """Radians a position of each of dims / 2 pairs: base ** (-2 j / dims)."""
    return [base ** (-2.0 * j / dims) for j in range(dims // 2)]


def rotary_turns(frequencies, device="cuda"):
    """The plan of a rotation that a program makes once: int64 [dims / 2] on `device`, the frequencies (radians a
    position, any sequence of floats) as turns of 64-bit fixed point."""
    import torch
    f = [float(x) for x in frequencies]
    out = (ctypes.c_uint64 * max(len(f), 1))()
    _check(LIB.fbl_rotary_turns((ctypes.c_double * max(len(f), 1))(*f), len(f), out), "fbl_rotary_turns")
    return torch.tensor([x - (1 << 64) if x >> 63 else x for x in out], dtype=torch.int64, device=device)


def _rotary(turns, positions, axes, neighbours: bool, B: int, S: int, where: str):
    """fbl_rotary of a call, None where nothing turns.  Both are read by address: what does not agree with
    the tensors would be read past its end."""
    import torch
    if turns is None:
        if positions is not None or axes is not None:
            raise FblError(FBL_ERR_ARG, f"{where}: positions and axes need turns")
        return None
    if turns.dtype != torch.int64:
        raise FblError(FBL_ERR_DTYPE, f"{where}: turns is {turns.dtype}, needs torch.int64")
    if turns.dim() != 1 or not turns.is_contiguous():
        raise FblError(FBL_ERR_LAYOUT, f"{where}: turns must be one contiguous dimension of dims / 2, as rotary_turns makes it")
    r = RotaryArgs(turns=turns.data_ptr(), dims=2 * turns.numel(), neighbours=bool(neighbours), num_axes=1)
    if turns.numel() > 64:
        raise FblError(FBL_ERR_SHAPE, f"{where}: {turns.numel()} pairs do not fit a head of at most 128")
    if axes is not None:
        axes = [int(a) for a in axes]
        if len(axes) != turns.numel():
            raise FblError(FBL_ERR_SHAPE, f"{where}: {len(axes)} axes for {turns.numel()} pairs")
        if positions is None or positions.dim() != 3:
            raise FblError(FBL_ERR_SHAPE, f"{where}: axes need positions [axes, B, S]")
        if axes and not 0 <= min(axes) <= max(axes) < min(positions.shape[0], FBL_ROTARY_MAX_AXES):
            raise FblError(FBL_ERR_ARG, f"{where}: axes must be 0 .. {min(positions.shape[0], FBL_ROTARY_MAX_AXES) - 1}")
        r.axes[:len(axes)] = axes
    if positions is not None:
        if positions.dtype != torch.int64:
            raise FblError(FBL_ERR_DTYPE, f"{where}: positions is {positions.dtype}, needs torch.int64")
        want = {1: (S,), 2: (B, S), 3: (*positions.shape[:1], B, S)}.get(positions.dim())
        if want is None or tuple(positions.shape) != want or positions.shape[0] == 0:
            raise FblError(FBL_ERR_SHAPE, f"{where}: positions has shape {tuple(positions.shape)}, needs {(S,)}, {(B, S)} or "
                                          f"{('axes', B, S)}")
        if positions.dim() == 3:
            if axes is None and positions.shape[0] > 1:
                raise FblError(FBL_ERR_ARG, f"{where}: positions of {positions.shape[0]} axes need axes, the axis of each pair")
            if positions.shape[0] > FBL_ROTARY_MAX_AXES:
                raise FblError(FBL_ERR_ARG, f"{where}: {positions.shape[0]} axes, there are at most {FBL_ROTARY_MAX_AXES}")
            r.num_axes = positions.shape[0]
        st = positions.stride()
        r.positions = positions.data_ptr()
        r.stride_token = st[-1]
        r.stride_batch = st[-2] if positions.dim() >= 2 else 0
        r.stride_axis = st[0] if positions.dim() == 3 else 0
    return r


def _head_norm(q_weight, k_weight, eps, D: int, dtype, where: str):
    """fbl_head_norm of a call, None without a norm."""
    if eps is None:
        if q_weight is not None or k_weight is not None:
            raise FblError(FBL_ERR_ARG, f"{where}: weights need a norm: give eps")
        return None
    _vector(q_weight, where, "q_weight", D, dtype)
    _vector(k_weight, where, "k_weight", D, dtype)
    return HeadNormArgs(q_weight=_ptr(q_weight), k_weight=_ptr(k_weight), eps=float(eps))


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _heads_out(out, like, stream):
    """`out`, or a new contiguous tensor of like's shape."""
    return _empty(like.shape, like.dtype, like, stream) if out is None else out


def qk_norm_rotary_fwd(q, k, Hq: int, Hkv: int, turns=None, positions=None, axes=None, neighbours: bool = False,
                       q_weight=None, k_weight=None, eps: Optional[float] = None, q_out=None, k_out=None, stream=None):
    """Norms of each head of q [B, S, Hq d] and k [B, S, Hkv d] (k may be None) and their rotation by position, d 32, 64 or
    128: returns (q', k').  eps: of the norm, x / sqrt(mean(x^2) + eps) * weight, None for none; the weights
    [d] may be None.  turns: rotary_turns of dims / 2 frequencies, None for no rotation; positions: int64 [S], [B, S] or
    [axes, B, S], None for 0 .. S - 1; axes: with several, the axis of each pair.  The pairs are the halves of the first
    dims values, or neighbours.  q_out and k_out may be q and k themselves."""
    done = _FAST.qk_norm_rotary_fwd(q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight, eps, q_out, k_out,
                                    stream)
    if done is not None:
        return done
    where = "qk_norm_rotary_fwd"
    _check_device(where, stream, q=q, k=k, turns=turns, positions=positions, q_weight=q_weight, k_weight=k_weight,
                  q_out=q_out, k_out=k_out)
    lq, lk = _layout(q, Hq), None if k is None else _layout(k, Hkv)
    B, S = q.shape[:2]
    rot = _rotary(turns, positions, axes, neighbours, B, S, where)
    norm = _head_norm(q_weight, k_weight, eps, lq.D, q.dtype, where)
    q_out = _heads_out(q_out, q, stream)
    if k is not None:
        k_out = _heads_out(k_out, k, stream)
    lqo, lko = _layout(q_out, Hq), None if k_out is None else _layout(k_out, Hkv)
    _call("fbl_qk_norm_rotary_fwd", q, stream, _ref(lq), _ptr(q), _ref(lk), _ptr(k), _ref(rot), _ref(norm), _ref(lqo),
          _ptr(q_out), _ref(lko), _ptr(k_out))
    return q_out, k_out


def qk_norm_rotary_bwd_workspace(q, k, Hq: int, Hkv: int) -> int:
    """Bytes of qk_norm_rotary_bwd's workspace where a weight's gradient is wanted."""
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_qk_norm_rotary_bwd_workspace(_ref(_layout(q, Hq)), _ref(None if k is None else _layout(k, Hkv)),
                                                ctypes.byref(n)), "fbl_qk_norm_rotary_bwd_workspace")
    return int(n.value)


def qk_norm_rotary_bwd(dq_out, dk_out, q, k, Hq: int, Hkv: int, turns=None, positions=None, axes=None,
                       neighbours: bool = False, q_weight=None, k_weight=None, eps: Optional[float] = None, dq=None, dk=None,
                       dq_weight=None, dk_weight=None, workspace=None, stream=None, need_weights: bool = True):
    """Gradients of qk_norm_rotary_fwd from those of its results (dk_out None without keys): returns (dq, dk, dq_weight,
    dk_weight), the weights' None where there is no weight or need_weights is False.  q and k are the forward's inputs,
    needed with a norm (else they may be None).  dq and dk may be dq_out and dk_out themselves."""
    done = _FAST.qk_norm_rotary_bwd(dq_out, dk_out, q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight, eps,
                                    dq, dk, dq_weight, dk_weight, workspace, stream, need_weights)
    if done is not None:
        return done
    where = "qk_norm_rotary_bwd"
    if eps is None:
        q = k = None
    elif q is None or (k is None) != (dk_out is None):
        raise FblError(FBL_ERR_NULL, f"{where}: a norm's backward needs the forward's inputs")
    _check_device(where, stream, dq_out=dq_out, dk_out=dk_out, q=q, k=k, turns=turns, positions=positions, q_weight=q_weight,
                  k_weight=k_weight, dq=dq, dk=dk, dq_weight=dq_weight, dk_weight=dk_weight, workspace=workspace)
    lgq, lgk = _layout(dq_out, Hq), None if dk_out is None else _layout(dk_out, Hkv)
    lq, lk = None if q is None else _layout(q, Hq), None if k is None else _layout(k, Hkv)
    B, S = dq_out.shape[:2]
    rot = _rotary(turns, positions, axes, neighbours, B, S, where)
    norm = _head_norm(q_weight, k_weight, eps, lgq.D, dq_out.dtype, where)
    dq = _heads_out(dq, dq_out, stream)
    if dk_out is not None:
        dk = _heads_out(dk, dk_out, stream)
    if need_weights:
        if dq_weight is None and q_weight is not None:
            dq_weight = _empty(lgq.D, dq_out.dtype, dq_out, stream)
        if dk_weight is None and k_weight is not None and dk_out is not None:
            dk_weight = _empty(lgq.D, dq_out.dtype, dq_out, stream)
    _vector(dq_weight, where, "dq_weight", lgq.D, dq_out.dtype)
    _vector(dk_weight, where, "dk_weight", lgq.D, dq_out.dtype)
    ws, ws_bytes = None, 0
    if dq_weight is not None or dk_weight is not None:
        need = 0 if workspace is not None else qk_norm_rotary_bwd_workspace(dq_out, dk_out, Hq, Hkv)
        ws, ws_bytes = _scratch(workspace, need, where, dq_out, stream)
    ldq, ldk = _layout(dq, Hq), None if dk is None else _layout(dk, Hkv)
    _call("fbl_qk_norm_rotary_bwd", dq_out, stream, _ref(lgq), _ptr(dq_out), _ref(lgk), _ptr(dk_out), _ref(lq), _ptr(q),
          _ref(lk), _ptr(k), _ref(rot), _ref(norm), _ref(ldq), _ptr(dq), _ref(ldk), _ptr(dk), _ptr(dq_weight),
          _ptr(dk_weight), _ptr(ws), ws_bytes)
    return dq, dk, dq_weight, dk_weight


# ------------------------------------------------- the global norm of gradients
def _dense(t) -> bool:
    """Whether a tensor's values lie in one piece of memory, in any order of its dimensions."""
    if t.is_contiguous():
        return True
    step = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n > 1):
        if stride != step:
            return False
        step *= size
    return True


def _grad_list(grads, out, where: str):
    """(fbl_grad array, the first tensor) of a list of gradients and of the tensors that receive them."""
    import torch
    grads = list(grads)
    out = grads if out is None else list(out)
    if not grads:
        raise FblError(FBL_ERR_SHAPE, f"{where}: no gradients")
    if len(out) != len(grads):
        raise FblError(FBL_ERR_SHAPE, f"{where}: {len(out)} outputs for {len(grads)} gradients")
    a = (Grad * len(grads))()
    first = grads[0]
    for i, (g, o) in enumerate(zip(grads, out)):
        for name, t in (("grads", g), ("out", o)):
            if not isinstance(t, torch.Tensor) or t.layout != torch.strided:
                raise FblError(FBL_ERR_ARG, f"{where}: {name}[{i}] must be a plain tensor")
            if not t.is_cuda or t.device != first.device:
                raise FblError(FBL_ERR_ARG, f"{where}: {name}[{i}] is on {t.device}, all must be on one GPU"
                                            + (f", grads[0] is on {first.device}" if first.is_cuda else ""))
        if not _dense(g):
            raise FblError(FBL_ERR_LAYOUT, f"{where}: grads[{i}] has gaps, shape {tuple(g.shape)} strides {g.stride()}")
        if o is not g:
            if o.dtype != g.dtype:
                raise FblError(FBL_ERR_DTYPE, f"{where}: out[{i}] is {o.dtype}, needs {g.dtype}")
            if o.shape != g.shape or any(x != y for x, y, n in zip(o.stride(), g.stride(), g.shape) if n > 1):
                raise FblError(FBL_ERR_SHAPE, f"{where}: out[{i}] has shape {tuple(o.shape)} strides {o.stride()}, needs "
                                              f"{tuple(g.shape)} {g.stride()}")
        a[i].p, a[i].out, a[i].n, a[i].dtype = g.data_ptr(), o.data_ptr(), g.numel(), _dtype_code(g)
    return a, first


def _norm_out(norm, like, where: str, stream):
    import torch
    if norm is None:
        return _empty((), torch.float32, like, stream)
    if norm.dtype != torch.float32 or norm.numel() != 1:
        raise FblError(FBL_ERR_SHAPE, f"{where}: norm must be one float32")
    return norm


def grad_norm_workspace(grads) -> int:
    """Bytes of grad_norm's and clip_grad_norm's workspace."""
    n = ctypes.c_size_t(0)
    _check(LIB.fbl_grad_norm_workspace(len(grads), ctypes.byref(n)), "fbl_grad_norm_workspace")
    return int(n.value)


def grad_norm(grads, norm=None, workspace=None, stream=None):
    """The norm of all values of a list of tensors (float32 and bfloat16, each in one piece of memory): one
    float32 on their device."""
    done = _FAST.grad_norm(grads, norm, workspace, stream)
    if done is not None:
        return done
    where = "grad_norm"
    a, like = _grad_list(grads, None, where)
    norm = _norm_out(norm, like, where, stream)
    _check_device(where, stream, grads=like, norm=norm, workspace=workspace)
    ws, ws_bytes = _scratch(workspace, 0 if workspace is not None else grad_norm_workspace(a), where, like, stream)
    _call("fbl_grad_norm", like, stream, len(a), a, _ptr(norm), _ptr(ws), ws_bytes)
    return norm


def clip_grads(grads, norm, limit: float, out=None, stream=None) -> None:
    """Every gradient times min(1, limit / (norm + 1e-6)), in place or into the tensors of `out`; norm is one float32 on
    their device (grad_norm's, or the program's own)."""
    where = "clip_grads"
    if norm is None:
        raise FblError(FBL_ERR_NULL, f"{where}: needs the norm; clip_grad_norm takes it by itself")
    a, like = _grad_list(grads, out, where)
    norm = _norm_out(norm, like, where, stream)
    _check_device(where, stream, grads=like, norm=norm)
    _call("fbl_grad_clip", like, stream, len(a), a, _ptr(norm), float(limit))


def clip_grad_norm(grads, limit: float, out=None, norm=None, workspace=None, stream=None):
    """grad_norm and clip_grads by it in one call: returns the norm of the gradients as they were."""
    done = _FAST.clip_grad_norm(grads, limit, out, norm, workspace, stream)
    if done is not None:
        return done
    where = "clip_grad_norm"
    a, like = _grad_list(grads, out, where)
    norm = _norm_out(norm, like, where, stream)
    _check_device(where, stream, grads=like, norm=norm, workspace=workspace)
    ws, ws_bytes = _scratch(workspace, 0 if workspace is not None else grad_norm_workspace(a), where, like, stream)
    _call("fbl_clip_grad_norm", like, stream, len(a), a, float(limit), _ptr(norm), _ptr(ws), ws_bytes)
    return norm
