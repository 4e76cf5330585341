"""ctypes declarations of the C ABI in include/dc.h (argument marshalling only)."""
from __future__ import annotations

import ctypes as C
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdrivecache.so")

DC_OK, DC_ERR_ARG, DC_ERR_SHAPE, DC_ERR_DTYPE, DC_ERR_HIP, DC_ERR_WORKSPACE, DC_ERR_STATE = 0, -1, -2, -3, -4, -5, -6
DC_F32, DC_BF16 = 0, 1
DC_MAX_BATCH = 64

vp = C.c_void_p


class ModelCfg(C.Structure):
    _fields_ = [("n_blocks", C.c_int32), ("hidden", C.c_int32), ("heads", C.c_int32),
                ("head_dim", C.c_int32), ("mlp_hidden", C.c_int32), ("lat_c", C.c_int32),
                ("lat_t", C.c_int32), ("lat_h", C.c_int32), ("lat_w", C.c_int32),
                ("patch", C.c_int32), ("n_txt", C.c_int32), ("dtype", C.c_int32),
                ("ln_eps", C.c_float)]


class BlockWeights(C.Structure):
    _fields_ = [("w_qkv", vp), ("b_qkv", vp), ("w_o", vp), ("b_o", vp), ("w_1", vp), ("b_1", vp),
                ("w_2", vp), ("b_2", vp), ("mod_offset", vp)]


class ModelWeights(C.Structure):
    _fields_ = [("w_pe", vp), ("b_pe", vp), ("pos", vp), ("w_t1", vp), ("b_t1", vp), ("w_t2", vp),
                ("b_t2", vp), ("w_m", vp), ("b_m", vp), ("head_mod", vp), ("w_head", vp),
                ("b_head", vp), ("blocks", C.POINTER(BlockWeights))]


class SchedProblem(C.Structure):
    _fields_ = [("K", C.c_int32), ("h_max", C.c_int32), ("n_cap", C.c_int32),
                ("legal", C.POINTER(C.c_uint8)), ("segment", C.POINTER(C.c_int32)),
                ("n_pose", C.c_int32), ("pose_xy", C.POINTER(C.c_double)),
                ("pose_yaw", C.POINTER(C.c_double)), ("L0", C.c_double), ("Th0", C.c_double),
                ("L1", C.c_double), ("Th1", C.c_double), ("eps", C.c_double),
                ("q0", C.POINTER(C.c_double)), ("q1", C.POINTER(C.c_double)),
                ("d0", C.POINTER(C.c_double)), ("d1", C.POINTER(C.c_double)),
                ("tau_q", C.c_int64), ("start_step", C.c_int32), ("spent_q", C.c_int64),
                ("spent_n", C.c_int32)]


class Schedule(C.Structure):
    _fields_ = [("reuse", C.POINTER(C.c_uint8)), ("chat_q", C.POINTER(C.c_int64)),
                ("dbar", C.POINTER(C.c_double)), ("n_reuse", C.c_int32), ("cost_q", C.c_int64),
                ("L", C.c_double), ("Theta", C.c_double), ("zL", C.c_double), ("zTh", C.c_double),
                ("D", C.c_double), ("in_support", C.c_int32)]


class Buffers(C.Structure):
    _fields_ = [("x", vp), ("txt", vp), ("h_in", vp), ("h", vp), ("resid", vp), ("u_ref", vp),
                ("mod", vp), ("sums", vp), ("ws", vp), ("ws_bytes", C.c_size_t)]


class SamplerOpts(C.Structure):
    _fields_ = [("drift_metric", C.c_int32), ("w_low", C.POINTER(ModelWeights)), ("k_switch", C.c_int32),
                ("mod_low", vp), ("cfg", C.c_int32), ("guidance", C.c_float), ("txt_null", vp)]


class RopeAxes(C.Structure):
    _fields_ = [("dim", C.c_int32 * 3), ("theta", C.c_double), ("start", C.c_double * 3),
                ("step", C.c_double * 3)]


class QkCfg(C.Structure):
    _fields_ = [("q_weight", vp), ("k_weight", vp), ("eps", C.c_float), ("cos_sin", vp),
                ("interleaved", C.c_int32)]


class LinearI8Args(C.Structure):
    _fields_ = [("rows", C.c_int32), ("out_features", C.c_int32), ("in_features", C.c_int32),
                ("x", vp), ("x_scale", vp), ("ld_x", C.c_int64), ("w", vp), ("w_scale", vp),
                ("ld_w", C.c_int64), ("bias", vp), ("gelu", C.c_int32), ("gate", vp), ("residual", vp),
                ("ld_residual", C.c_int64), ("out", vp), ("out_dtype", C.c_int32), ("ld_out", C.c_int64)]


class QuantizeF8Args(C.Structure):
    _fields_ = [("rows", C.c_int32), ("cols", C.c_int32), ("x", vp), ("x_dtype", C.c_int32), ("ld_x", C.c_int64),
                ("block_rows", C.c_int32), ("q", vp), ("ld_q", C.c_int64), ("scale", vp), ("scale_row", C.c_int64),
                ("scale_block", C.c_int64)]


class RmsNormF8Args(C.Structure):
    _fields_ = [("rows", C.c_int32), ("cols", C.c_int32), ("x", vp), ("x_dtype", C.c_int32), ("ld_x", C.c_int64),
                ("residual", vp), ("residual_dtype", C.c_int32), ("ld_residual", C.c_int64), ("sum", vp),
                ("sum_dtype", C.c_int32), ("ld_sum", C.c_int64), ("weight", vp), ("eps", C.c_float), ("q", vp),
                ("ld_q", C.c_int64), ("scale", vp), ("scale_row", C.c_int64), ("scale_block", C.c_int64)]


class LinearF8Args(C.Structure):
    _fields_ = [("rows", C.c_int32), ("out_features", C.c_int32), ("in_features", C.c_int32), ("x", vp),
                ("ld_x", C.c_int64), ("x_scale", vp), ("x_scale_row", C.c_int64), ("x_scale_block", C.c_int64),
                ("w", vp), ("ld_w", C.c_int64), ("w_scale", vp), ("w_scale_row", C.c_int64),
                ("w_scale_block", C.c_int64), ("bias", vp), ("gelu", C.c_int32), ("gate", vp), ("residual", vp),
                ("ld_residual", C.c_int64), ("out", vp), ("out_dtype", C.c_int32), ("ld_out", C.c_int64)]


class BlockWeightsI8(C.Structure):
    _fields_ = [("w_qkv", vp), ("s_qkv", vp), ("w_o", vp), ("s_o", vp), ("w_1", vp), ("s_1", vp),
                ("w_2", vp), ("s_2", vp)]


class BlockExt(C.Structure):
    _fields_ = [("qk", C.POINTER(QkCfg)), ("i8", C.POINTER(BlockWeightsI8))]


class SamplerExt(C.Structure):
    _fields_ = [("blocks", C.POINTER(BlockExt)), ("blocks_low", C.POINTER(BlockExt)),
                ("cache_bits", C.c_int32), ("cache_scales", vp)]


P = C.POINTER
i32p = P(C.c_int32)

SIGNATURES = {
    "dc_last_error": (C.c_char_p, []),
    "dc_workspace_bytes": (C.c_size_t, [P(ModelCfg), C.c_int32]),
    "dc_time_modulation": (C.c_int32, [P(ModelCfg), P(ModelWeights), P(C.c_double), C.c_int32, vp, vp,
                                       C.c_size_t, vp]),
    "dc_patch_embed": (C.c_int32, [P(ModelCfg), P(ModelWeights), vp, vp, vp, i32p, C.c_int32, vp,
                                   C.c_size_t, vp]),
    "dc_block_forward": (C.c_int32, [P(ModelCfg), P(BlockWeights), vp, vp, i32p, C.c_int32, vp,
                                     C.c_size_t, vp]),
    "dc_cache_store": (C.c_int32, [P(ModelCfg), vp, vp, vp, i32p, C.c_int32, vp]),
    "dc_cache_apply": (C.c_int32, [P(ModelCfg), vp, vp, vp, i32p, C.c_int32, vp]),
    "dc_drift_l1": (C.c_int32, [P(ModelCfg), vp, vp, vp, C.c_int32, vp, i32p, C.c_int32, vp,
                                C.c_size_t, vp]),
    "dc_drift_l1_noalloc": (C.c_int32, [P(ModelCfg), vp, vp, vp, C.c_int32, vp, i32p, C.c_int32, vp]),
    "dc_head_euler": (C.c_int32, [P(ModelCfg), P(ModelWeights), vp, vp, vp, C.c_float, i32p,
                                  C.c_int32, vp, C.c_size_t, vp]),
    "dc_calibrate_workspace_bytes": (C.c_size_t, [P(ModelCfg), C.c_int32]),
    "dc_calibrate_tables": (C.c_int32, [P(ModelCfg), P(ModelWeights), vp, vp, P(C.c_double), C.c_int32,
                                        C.c_int32, C.c_double, P(C.c_double), P(C.c_double), vp,
                                        C.c_size_t, vp]),
    "dc_rope_table": (C.c_int32, [P(ModelCfg), P(RopeAxes), vp, vp, vp]),
    "dc_qk_norm_rope": (C.c_int32, [P(ModelCfg), P(QkCfg), vp, C.c_int64, vp, C.c_int64, C.c_float, i32p,
                                    C.c_int32, vp]),
    "dc_quantize_rows": (C.c_int32, [vp, C.c_int32, C.c_int64, C.c_int32, C.c_int32, vp, C.c_int64, vp, vp]),
    "dc_linear_i8": (C.c_int32, [P(LinearI8Args), vp]),
    "dc_quantize_f8": (C.c_int32, [P(QuantizeF8Args), vp]),
    "dc_rms_norm_f8": (C.c_int32, [P(RmsNormF8Args), vp]),
    "dc_linear_f8": (C.c_int32, [P(LinearF8Args), vp]),
    "dc_cache_store_q": (C.c_int32, [P(ModelCfg), C.c_int32, vp, vp, vp, vp, i32p, C.c_int32, vp]),
    "dc_cache_apply_q": (C.c_int32, [P(ModelCfg), C.c_int32, vp, vp, vp, vp, i32p, C.c_int32, vp]),
    "dc_block_ext_workspace_bytes": (C.c_size_t, [P(ModelCfg), C.c_int32]),
    "dc_block_forward_ext": (C.c_int32, [P(ModelCfg), P(BlockWeights), P(BlockExt), vp, vp, i32p, C.c_int32,
                                         vp, C.c_size_t, vp]),
    "dc_schedule_dp": (C.c_int32, [P(SchedProblem), P(Schedule)]),
    "dc_select_tau": (C.c_int32, [P(SchedProblem), C.c_int32, C.c_double, P(C.c_int64)]),
    "dc_motion_statistics": (C.c_int32, [P(C.c_double), P(C.c_double), C.c_int32, P(C.c_double),
                                         P(C.c_double)]),
    "dc_select_anchors": (C.c_int32, [P(C.c_double), P(C.c_double), C.c_int32, C.c_double,
                                      P(C.c_double), P(C.c_int32)]),
    "dc_sampler_create": (C.c_int32, [P(ModelCfg), P(ModelWeights), C.c_int32, P(SchedProblem),
                                      P(C.c_double), P(Buffers), C.c_int32, vp, P(vp)]),
    "dc_sampler_create_ex": (C.c_int32, [P(ModelCfg), P(ModelWeights), C.c_int32, P(SchedProblem),
                                         P(C.c_double), P(Buffers), P(SamplerOpts), vp, P(vp)]),
    "dc_sampler_create_ext": (C.c_int32, [P(ModelCfg), P(ModelWeights), C.c_int32, P(SchedProblem),
                                          P(C.c_double), P(Buffers), P(SamplerOpts), P(SamplerExt), vp,
                                          P(vp)]),
    "dc_denoise_step": (C.c_int32, [vp, C.c_int32, vp, P(C.c_uint8), P(C.c_double)]),
    "dc_sampler_plan": (C.c_int32, [vp, C.c_int32, P(C.c_uint8), i32p, P(C.c_int64)]),
    "dc_sampler_destroy": (None, [vp]),
    "dc_profile_enable": (C.c_int32, [C.c_uint32]),
    "dc_profile_read": (C.c_int32, [C.c_int32, P(C.c_int64), P(C.c_double)]),
    "dc_profile_reset": (C.c_int32, []),
}

KERNEL_CLASSES = ("attention", "gemm_qkv", "gemm_out", "gemm_up", "gemm_down", "ln_modulate",
                  "patch_embed", "drift", "cache_store", "cache_apply", "head", "head_reuse",
                  "qk_norm_rope", "quantize")

_lib = None


class DriveCacheError(RuntimeError):
    def __init__(self, fn, code, msg):
        super().__init__(f"{fn} failed with status {code}: {msg}")
        self.code = code


def load() -> C.CDLL:
    """Load libdrivecache.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with python -m paper_2608_16354_amd.build")
        lib = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            f = getattr(lib, name)
            f.restype = res
            f.argtypes = args
        _lib = lib
    return _lib


_binding = None


def binding():
    """The tensor binding (binding.cpp) on the loaded library; raises if it has not been built."""
    global _binding
    if _binding is None:
        lib = load()
        import torch  # noqa: F401  (the libraries that the binding is linked against)
        try:
            from . import _binding as b
        except ImportError as e:
            raise ImportError("_binding.so is missing or does not fit this torch: build it with "
                              "python -m paper_2608_16354_amd.build") from e
        b.init(*[C.cast(getattr(lib, n), vp).value for n in (
            "dc_rope_table", "dc_qk_norm_rope", "dc_quantize_rows", "dc_linear_i8", "dc_cache_store_q",
            "dc_cache_apply_q", "dc_quantize_f8", "dc_rms_norm_f8", "dc_linear_f8")])
        _binding = b
    return _binding


def check(fn: str, code: int):
    if code != DC_OK:
        msg = load().dc_last_error().decode(errors="replace")
        raise DriveCacheError(fn, code, msg)
