"""ctypes loader for libxdit.so (the HIP library built from csrc/).

The library is loaded from this package directory only; there is no fallback.
If it has not been built, loading raises XditError (build it with
``python -m paper_2411_01738_amd.build``).
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIBRARY = os.path.join(HERE, "libxdit.so")

# Status codes of include/xdit.h
XDIT_OK = 0
STATUS = {
    0: "XDIT_OK", -1: "XDIT_ERR_NULL", -2: "XDIT_ERR_DTYPE", -3: "XDIT_ERR_SHAPE",
    -4: "XDIT_ERR_RANGE", -5: "XDIT_ERR_LAYOUT", -6: "XDIT_ERR_ALIAS",
    -7: "XDIT_ERR_UNSUPPORTED", -8: "XDIT_ERR_HIP",
}
XDIT_BF16, XDIT_F32, XDIT_I64 = 0, 1, 2
NORMS = {"none": 0, "rms": 1, "layer": 2}
LAYOUTS = {"interleaved": 0, "half": 1}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "ramp": 3}
XDIT_MAX_AXES = 4
XDIT_ACCUM_DQ, XDIT_ACCUM_DKV = 1, 2
XDIT_MAX_PARTIALS = 64
XDIT_MAX_RANGES = 2
XDIT_MAX_SPLITS = 16

_vp = ctypes.c_void_p
_i64 = ctypes.c_int64
_i32 = ctypes.c_int32
_f64 = ctypes.c_double


class RopeScaling(ctypes.Structure):
    """xdit_rope_scaling"""
    _fields_ = [("kind", _i32), ("factor", _f64), ("orig_len", _f64), ("fast", _f64), ("slow", _f64), ("magnitude", _f64)]


class Qk(ctypes.Structure):
    """xdit_qk"""
    _fields_ = [("batch", _i64), ("tokens", _i64), ("q_heads", _i64), ("k_heads", _i64), ("head_dim", _i64),
                ("dtype", _i32), ("norm", _i32), ("eps", _f64), ("wq", _vp), ("wk", _vp), ("bq", _vp), ("bk", _vp),
                ("weight_dtype", _i32), ("layout", _i32), ("rot_dim", _i64), ("cos", _vp), ("sin", _vp),
                ("table_per_batch", _i32), ("strides", ctypes.POINTER(_i64))]


SIGNATURES = {
    "xdit_patch_attn": (ctypes.c_int, [_vp, _vp, _i64, _i64, _vp, _vp, _vp, _i64, _i64, _i64, _i64,
                                       _i32]),
    "xdit_patch_attn_ranges": (ctypes.c_int, [_vp, _i64, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp,
                                              _i64, _i64, _i64, _i64, _i32]),
    "xdit_chunk_attn": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _i64, _i32]),
    "xdit_split_workspace_bytes": (_i64, [_i64, _i64, _i64, _i64, _i64, _i32, _i32]),
    "xdit_chunk_attn_split": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _i32, _vp, _i64, _i64, _i64,
                                             _i64, _i64, _i64, _i32]),
    "xdit_chunk_attn_split_noalloc": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _i32, _i64, _i64, _i64,
                                                     _i64, _i64, _i32]),
    "xdit_noalloc_scratch_bytes": (_i64, []),
    "xdit_patch_attn_split": (ctypes.c_int, [_vp, _i64, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp,
                                             _i32, _vp, _i64, _i64, _i64, _i64, _i64, _i32]),
    "xdit_chunk_attn_accum": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _i64,
                                             _i32]),
    "xdit_chunk_attn_accum_split": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _i32, _vp, _i64, _i64,
                                                   _i64, _i64, _i64, _i64, _i32]),
    "xdit_lse_merge": (ctypes.c_int, [_vp, _vp, _i32, _vp, _vp, _i64, _i64, _i64, _i64, _i32]),
    "xdit_kv_update": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp, _i64, _i64, _i64, _i64, _i32]),
    "xdit_stage_step": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _vp,
                                       _vp, _i64, _i64, _i64, _i64, _i64, _i32]),
    "xdit_chunk_attn_bwd_workspace_bytes": (_i64, [_i64, _i64, _i64, _i64, _i64, _i32]),
    "xdit_chunk_attn_bwd": (ctypes.c_int, [_vp] * 10 + [_i32, _vp, _i64] + [_i64] * 5 + [_i32]),
    "xdit_rope_table": (ctypes.c_int, [_vp, _i32, _i64, _i32, _vp, _f64, ctypes.POINTER(RopeScaling), _vp, _vp]),
    "xdit_rope": (ctypes.c_int, [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64, _i64, _i32, _i32, _i32, _i32]),
    "xdit_qk_norm_rope": (ctypes.c_int, [ctypes.POINTER(Qk), _vp, _vp, _vp, _vp]),
    "xdit_qk_norm_rope_bwd_workspace_bytes": (_i64, [_i64, _i64, _i64, _i64, _i64, _i32]),
    "xdit_qk_norm_rope_bwd": (ctypes.c_int, [ctypes.POINTER(Qk), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                             _i64]),
    "xdit_stage_step_qk": (ctypes.c_int, [ctypes.POINTER(Qk), _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _vp,
                                          _vp, _i64, _i64, _i64, _i64, _i64, _i32]),
    "xdit_set_stream": (ctypes.c_int, [_vp]),
    "xdit_get_stream": (_vp, []),
    "xdit_last_error": (ctypes.c_char_p, []),
    "xdit_version": (ctypes.c_char_p, []),
}


class XditError(RuntimeError):
    def __init__(self, code: int, message: str):
        self.code = code
        super().__init__(f"{STATUS.get(code, code)}: {message}")


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library with argument types set (loaded once)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIBRARY):
            raise XditError(-8, f"{LIBRARY} is missing: build it with "
                                "`python -m paper_2411_01738_amd.build`")
        handle = ctypes.CDLL(LIBRARY)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def check(code: int) -> None:
    if code != XDIT_OK:
        raise XditError(code, lib().xdit_last_error().decode())
