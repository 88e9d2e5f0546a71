"""Thin ctypes binding of libogc_mlp.so (include/ogc_mlp.h, ogc_mha.h, ogc_decoder.h, ogc_mx.h, ogc_sample.h): argument marshalling only.

Every step of the path runs in the library's HIP kernels.  PyTorch appears here only as the owner
of device memory and streams.  There is no CPU fallback: if the shared library is missing, loading
it raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

OGC_F32, OGC_BF16, OGC_I8, OGC_F8 = 0, 1, 2, 3
OGC_ACT_NONE, OGC_ACT_RELU, OGC_ACT_GELU_TANH, OGC_ACT_SIGMOID = 0, 1, 2, 3
OGC_OUT_SAME, OGC_OUT_F32 = 0, 1
OGC_MODE_AUTO, OGC_MODE_PER_LAYER, OGC_MODE_FUSED, OGC_MODE_COOP = 0, 1, 2, 3
OGC_LAYOUT_PLAIN, OGC_LAYOUT_BLOCKED = 0, 1
OGC_SOFTMAX_STABLE, OGC_SOFTMAX_FAST = 0, 1
OGC_ROPE_HALF, OGC_ROPE_INTERLEAVED = 0, 1
OGC_MX4, OGC_MX8 = 0, 1
OGC_NORM_SAME, OGC_NORM_MX4, OGC_NORM_MX8 = 0, 1, 2
OGC_GATE_NONE, OGC_GATE_SILU = 0, 1
OGC_OK = 0
DTYPES = {"f32": OGC_F32, "bf16": OGC_BF16, "i8": OGC_I8, "f8": OGC_F8}

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libogc_mlp.so")

EXPORTS = [
    "ogc_mlp_plan", "ogc_mlp_packed_bytes", "ogc_mlp_workspace_bytes", "ogc_mlp_chosen_mode",
    "ogc_mlp_buffer_assignment", "ogc_mlp_prepack_weights", "ogc_mlp_run", "ogc_mlp_destroy",
    "ogc_status_string", "ogc_mlp_kernel_name", "ogc_mlp_num_launches", "ogc_mlp_run_profiled", "ogc_mlp_blocked_bytes", "ogc_mlp_estimated_us", "ogc_mlp_mode_estimates",
    "ogc_mlp_run_static", "ogc_mlp_static_workspace_limit", "ogc_mlp_plan_with_overrides", "ogc_mlp_check", "ogc_mlp_test_barrier", "ogc_mlp_cluster_layout",
    "ogc_mlp_run_clocked", "ogc_mlp_clock_words_per_launch",
    "ogc_quantize_e4m3", "ogc_dequantize_e4m3",
    "ogc_mha_validate", "ogc_mha_run", "ogc_mha_kernel_name", "ogc_mha_i8_validate", "ogc_mha_run_i8", "ogc_mha_i8_kernel_name",
    "ogc_rope_validate", "ogc_rope_run", "ogc_kv4_validate", "ogc_kv4_cache_bytes", "ogc_kv4_write", "ogc_kv4_read",
    "ogc_kv4_attention_validate", "ogc_kv4_attention_workspace_bytes", "ogc_kv4_attention_run",
    "ogc_prompt_validate", "ogc_prompt_run", "ogc_prompt_kernel_name",
    "ogc_mx_bytes", "ogc_norm_validate", "ogc_norm_run", "ogc_mx_validate", "ogc_mx_write", "ogc_mx_read",
    "ogc_mx_product_validate", "ogc_mx_product_workspace_bytes", "ogc_mx_product_run", "ogc_mx_product_kernel_name",
    "ogc_sample_validate", "ogc_sample_workspace_bytes", "ogc_sample_run",
]
OGC_ERR_TIMEOUT = -8


class ogc_layer_desc(ctypes.Structure):
    _fields_ = [("k", ctypes.c_int32), ("n", ctypes.c_int32), ("has_bias", ctypes.c_int32), ("act", ctypes.c_int32),
                ("in_scale", ctypes.c_float), ("in_zp", ctypes.c_int32), ("out_scale", ctypes.c_float),
                ("out_zp", ctypes.c_int32), ("out", ctypes.c_int32)]


class ogc_mlp_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("m", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("layers", ctypes.POINTER(ogc_layer_desc)), ("ld_x", ctypes.c_int32), ("ld_y", ctypes.c_int32),
                ("residual", ctypes.c_int32), ("mode", ctypes.c_int32), ("x_layout", ctypes.c_int32),
                ("y_layout", ctypes.c_int32)]


class ogc_plan_overrides(ctypes.Structure):
    _fields_ = [("tile", ctypes.c_int32), ("ksplit_log2", ctypes.c_int32), ("cluster_split", ctypes.c_int32),
                ("cluster_ksplit", ctypes.c_int32), ("cluster_whole", ctypes.c_int32)]


class ogc_mha_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("seq", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("softmax", ctypes.c_int32), ("scale", ctypes.c_float),
                ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
                ("o_stride", ctypes.c_int64 * 3), ("query_groups", ctypes.c_int32)]


class ogc_mha_quant(ctypes.Structure):
    _fields_ = [("q_scale", ctypes.c_float), ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float), ("o_scale", ctypes.c_float)]


class ogc_rope_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("tokens", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("norm", ctypes.c_int32),
                ("eps", ctypes.c_float), ("magnitude", ctypes.c_float), ("q_stride", ctypes.c_int64 * 2),
                ("k_stride", ctypes.c_int64 * 2), ("qo_stride", ctypes.c_int64 * 2), ("ko_stride", ctypes.c_int64 * 2)]


class ogc_kv4_desc(ctypes.Structure):
    _fields_ = [("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("pages", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("table_width", ctypes.c_int32)]


class ogc_kv4_rows(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("rows", ctypes.c_int32), ("max_rows", ctypes.c_int32), ("k_stride", ctypes.c_int64 * 2),
                ("v_stride", ctypes.c_int64 * 2)]


class ogc_kv4_attention_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("rows", ctypes.c_int32), ("max_rows", ctypes.c_int32),
                ("max_keys", ctypes.c_int32), ("scale", ctypes.c_float), ("q_stride", ctypes.c_int64 * 2), ("o_stride", ctypes.c_int64 * 2)]


class ogc_prompt_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("q_rows", ctypes.c_int32), ("k_rows", ctypes.c_int32), ("max_q", ctypes.c_int32),
                ("max_k", ctypes.c_int32), ("scale", ctypes.c_float), ("causal", ctypes.c_int32), ("q_stride", ctypes.c_int64 * 2),
                ("k_stride", ctypes.c_int64 * 2), ("v_stride", ctypes.c_int64 * 2), ("o_stride", ctypes.c_int64 * 2)]


class ogc_norm_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("rows", ctypes.c_int32), ("channels", ctypes.c_int32), ("out", ctypes.c_int32),
                ("eps", ctypes.c_float), ("x_stride", ctypes.c_int64), ("residual_stride", ctypes.c_int64), ("sum_stride", ctypes.c_int64),
                ("y_stride", ctypes.c_int64)]


class ogc_mx_rows(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("format", ctypes.c_int32), ("rows", ctypes.c_int32), ("channels", ctypes.c_int32),
                ("gate", ctypes.c_int32), ("stride", ctypes.c_int64)]


class ogc_mx_product_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("x_format", ctypes.c_int32), ("w_format", ctypes.c_int32), ("m", ctypes.c_int32),
                ("n", ctypes.c_int32), ("k", ctypes.c_int32), ("has_bias", ctypes.c_int32), ("y_stride", ctypes.c_int64)]


class ogc_sample_desc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("stride", ctypes.c_int64)]


class OgcError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s: %s (%d)" % (what, status_string(status), status))


_lib = None


def lib():
    """Loads the shared library (fails loudly if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                "%s not found: build it with `python -m paper_2301_01333_amd.build` (there is no fallback path)" % LIB_PATH)
        try:  # PyTorch brings a HIP runtime of its own: loaded after this library, it would be a second one, whose streams and memory launches do not know
            import torch  # noqa: F401
        except ImportError:
            pass
        l = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        l.ogc_mlp_plan.argtypes = [ctypes.POINTER(ogc_mlp_desc), ctypes.POINTER(vp)]
        l.ogc_mlp_plan.restype = i32
        l.ogc_mlp_plan_with_overrides.argtypes = [ctypes.POINTER(ogc_mlp_desc), ctypes.POINTER(ogc_plan_overrides), ctypes.POINTER(vp)]
        l.ogc_mlp_plan_with_overrides.restype = i32
        l.ogc_mlp_check.argtypes = [vp, vp, vp]
        l.ogc_mlp_check.restype = i32
        l.ogc_mlp_test_barrier.argtypes = [vp, i32, i32]
        l.ogc_mlp_test_barrier.restype = i32
        l.ogc_mlp_cluster_layout.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_uint32), ctypes.POINTER(sz)]
        l.ogc_mlp_cluster_layout.restype = i32
        l.ogc_mlp_packed_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        l.ogc_mlp_packed_bytes.restype = i32
        l.ogc_mlp_workspace_bytes.argtypes = [vp, ctypes.POINTER(sz)]
        l.ogc_mlp_workspace_bytes.restype = i32
        l.ogc_mlp_blocked_bytes.argtypes = [vp, i32, ctypes.POINTER(sz)]
        l.ogc_mlp_blocked_bytes.restype = i32
        l.ogc_mlp_chosen_mode.argtypes = [vp, ctypes.POINTER(i32)]
        l.ogc_mlp_chosen_mode.restype = i32
        l.ogc_mlp_buffer_assignment.argtypes = [vp, i32, ctypes.POINTER(i32), ctypes.POINTER(sz)]
        l.ogc_mlp_buffer_assignment.restype = i32
        l.ogc_mlp_prepack_weights.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), vp, vp]
        l.ogc_mlp_prepack_weights.restype = i32
        l.ogc_mlp_run.argtypes = [vp, vp, vp, vp, vp, vp]
        l.ogc_mlp_run.restype = i32
        l.ogc_mlp_run_static.argtypes = [vp, vp, vp, vp, vp]
        l.ogc_mlp_run_static.restype = i32
        l.ogc_mlp_static_workspace_limit.argtypes = []
        l.ogc_mlp_static_workspace_limit.restype = sz
        l.ogc_mlp_num_launches.argtypes = [vp, ctypes.POINTER(i32)]
        l.ogc_mlp_num_launches.restype = i32
        l.ogc_mlp_run_clocked.argtypes = [vp, vp, vp, vp, vp, vp, vp]
        l.ogc_mlp_run_clocked.restype = i32
        l.ogc_mlp_clock_words_per_launch.argtypes = []
        l.ogc_mlp_clock_words_per_launch.restype = ctypes.c_size_t
        l.ogc_mlp_run_profiled.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.POINTER(ctypes.c_float)]
        l.ogc_mlp_run_profiled.restype = i32
        l.ogc_mlp_destroy.argtypes = [vp]
        l.ogc_mlp_destroy.restype = None
        l.ogc_status_string.argtypes = [i32]
        l.ogc_status_string.restype = ctypes.c_char_p
        l.ogc_mlp_kernel_name.argtypes = [vp, i32]
        l.ogc_mlp_kernel_name.restype = ctypes.c_char_p
        l.ogc_mlp_estimated_us.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_float)]
        l.ogc_mlp_estimated_us.restype = i32
        l.ogc_mlp_mode_estimates.argtypes = [vp, ctypes.POINTER(ctypes.c_float)]
        l.ogc_mlp_mode_estimates.restype = i32
        l.ogc_quantize_e4m3.argtypes = [vp, vp, sz, ctypes.c_float, vp]
        l.ogc_quantize_e4m3.restype = i32
        l.ogc_dequantize_e4m3.argtypes = [vp, vp, sz, ctypes.c_float, vp]
        l.ogc_dequantize_e4m3.restype = i32
        l.ogc_mha_validate.argtypes = [ctypes.POINTER(ogc_mha_desc)]
        l.ogc_mha_validate.restype = i32
        l.ogc_mha_run.argtypes = [ctypes.POINTER(ogc_mha_desc), vp, vp, vp, vp, vp, vp]
        l.ogc_mha_run.restype = i32
        l.ogc_mha_kernel_name.argtypes = [ctypes.POINTER(ogc_mha_desc), i32]
        l.ogc_mha_kernel_name.restype = ctypes.c_char_p
        l.ogc_mha_i8_validate.argtypes = [ctypes.POINTER(ogc_mha_desc), ctypes.POINTER(ogc_mha_quant)]
        l.ogc_mha_i8_validate.restype = i32
        l.ogc_mha_run_i8.argtypes = [ctypes.POINTER(ogc_mha_desc), ctypes.POINTER(ogc_mha_quant), vp, vp, vp, vp, vp, vp]
        l.ogc_mha_run_i8.restype = i32
        l.ogc_mha_i8_kernel_name.argtypes = [ctypes.POINTER(ogc_mha_desc)]
        l.ogc_mha_i8_kernel_name.restype = ctypes.c_char_p
        rope, cache, rows, asks, prompt = (ctypes.POINTER(t) for t in (ogc_rope_desc, ogc_kv4_desc, ogc_kv4_rows, ogc_kv4_attention_desc,
                                                                       ogc_prompt_desc))
        for name, args in (("ogc_rope_validate", [rope]), ("ogc_rope_run", [rope] + 9 * [vp]),
                           ("ogc_kv4_validate", [cache, rows]), ("ogc_kv4_cache_bytes", [cache, ctypes.POINTER(sz)]),
                           ("ogc_kv4_write", [cache, rows] + 7 * [vp]), ("ogc_kv4_read", [cache, rows] + 7 * [vp]),
                           ("ogc_kv4_attention_validate", [cache, asks]),
                           ("ogc_kv4_attention_workspace_bytes", [cache, asks, ctypes.POINTER(sz)]),
                           ("ogc_kv4_attention_run", [cache, asks] + 8 * [vp]),
                           ("ogc_prompt_validate", [prompt]), ("ogc_prompt_run", [prompt] + 7 * [vp])):
            getattr(l, name).argtypes, getattr(l, name).restype = args, i32
        l.ogc_prompt_kernel_name.argtypes, l.ogc_prompt_kernel_name.restype = [prompt], ctypes.c_char_p
        norm, mx, product, sample = (ctypes.POINTER(t) for t in (ogc_norm_desc, ogc_mx_rows, ogc_mx_product_desc, ogc_sample_desc))
        size = ctypes.POINTER(sz)
        for name, args in (("ogc_mx_bytes", [i32, i32, i32, size, size]), ("ogc_norm_validate", [norm]), ("ogc_norm_run", [norm] + 7 * [vp]),
                           ("ogc_mx_validate", [mx]), ("ogc_mx_write", [mx] + 4 * [vp]), ("ogc_mx_read", [mx] + 4 * [vp]),
                           ("ogc_mx_product_validate", [product]), ("ogc_mx_product_workspace_bytes", [product, size]),
                           ("ogc_mx_product_run", [product] + 8 * [vp]),
                           ("ogc_sample_validate", [sample]), ("ogc_sample_workspace_bytes", [sample, size]),
                           ("ogc_sample_run", [sample] + 10 * [vp])):
            getattr(l, name).argtypes, getattr(l, name).restype = args, i32
        l.ogc_mx_product_kernel_name.argtypes, l.ogc_mx_product_kernel_name.restype = [product], ctypes.c_char_p
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().ogc_status_string(int(status)).decode()


def _check(status: int, what: str) -> None:
    if status != OGC_OK:
        raise OgcError(status, what)


# ---- one function per entry point, same names ---------------------------------------------------
def _desc(dtype, m, layers, ld_x, ld_y, residual, mode, x_layout, y_layout):
    arr = (ogc_layer_desc * max(len(layers), 1))()
    for i, ly in enumerate(layers):
        arr[i] = ogc_layer_desc(int(ly["k"]), int(ly["n"]), int(ly.get("has_bias", 0)), int(ly.get("act", 0)),
                                float(ly.get("in_scale", 0.0)), int(ly.get("in_zp", 0)), float(ly.get("out_scale", 0.0)),
                                int(ly.get("out_zp", 0)), int(ly.get("out", 0)))
    desc = ogc_mlp_desc(int(dtype), int(m), len(layers), arr, int(ld_x), int(ld_y), int(residual), int(mode), int(x_layout),
                        int(y_layout))
    return desc, arr


def ogc_mlp_plan(dtype: int, m: int, layers: Sequence[dict], ld_x: int, ld_y: int, residual: int = 0, mode: int = 0,
                 x_layout: int = 0, y_layout: int = 0) -> int:
    """layers: dicts with k, n, has_bias, act, in_scale, in_zp, out_scale, out_zp, out.  Returns the plan handle."""
    desc, _keep = _desc(dtype, m, layers, ld_x, ld_y, residual, mode, x_layout, y_layout)
    handle = ctypes.c_void_p()
    _check(lib().ogc_mlp_plan(ctypes.byref(desc), ctypes.byref(handle)), "ogc_mlp_plan")
    return handle.value


def ogc_mlp_plan_with_overrides(dtype: int, m: int, layers: Sequence[dict], ld_x: int, ld_y: int, residual: int = 0,
                                mode: int = 0, x_layout: int = 0, y_layout: int = 0, overrides: Optional[dict] = None) -> int:
    """overrides: dict with any of tile, ksplit_log2, cluster_split, cluster_ksplit, cluster_whole (missing or None = -1,
    the cost model's choice); None passes a NULL pointer."""
    desc, _keep = _desc(dtype, m, layers, ld_x, ld_y, residual, mode, x_layout, y_layout)
    ov = None
    if overrides is not None:
        unknown = set(overrides) - {f for f, _ in ogc_plan_overrides._fields_}
        if unknown:
            raise KeyError("unknown plan overrides: %s" % sorted(unknown))
        ov = ogc_plan_overrides(*[-1 if overrides.get(f) is None else int(overrides[f]) for f, _ in ogc_plan_overrides._fields_])
    handle = ctypes.c_void_p()
    _check(lib().ogc_mlp_plan_with_overrides(ctypes.byref(desc), ctypes.byref(ov) if ov is not None else None,
                                             ctypes.byref(handle)), "ogc_mlp_plan_with_overrides")
    return handle.value


def ogc_mlp_check(plan: int, packed_ptr: int, stream: int = 0) -> int:
    """Returns the status (OGC_OK or OGC_ERR_TIMEOUT); raises on any other error."""
    st = int(lib().ogc_mlp_check(plan, packed_ptr, stream))
    if st not in (OGC_OK, OGC_ERR_TIMEOUT):
        raise OgcError(st, "ogc_mlp_check")
    return st


def ogc_mlp_test_barrier(plan: int, budget: int, extra_target: int) -> None:
    _check(lib().ogc_mlp_test_barrier(plan, int(budget), int(extra_target)), "ogc_mlp_test_barrier")


def ogc_mlp_cluster_layout(plan: int):
    """(members per row tile, k-split variant?, whole-layer mask, tile stride in bytes)."""
    m, k, w, st = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_uint32(), ctypes.c_size_t()
    _check(lib().ogc_mlp_cluster_layout(plan, ctypes.byref(m), ctypes.byref(k), ctypes.byref(w), ctypes.byref(st)),
           "ogc_mlp_cluster_layout")
    return m.value, k.value, w.value, st.value


def ogc_mlp_packed_bytes(plan: int) -> int:
    v = ctypes.c_size_t()
    _check(lib().ogc_mlp_packed_bytes(plan, ctypes.byref(v)), "ogc_mlp_packed_bytes")
    return v.value


def ogc_mlp_workspace_bytes(plan: int) -> int:
    v = ctypes.c_size_t()
    _check(lib().ogc_mlp_workspace_bytes(plan, ctypes.byref(v)), "ogc_mlp_workspace_bytes")
    return v.value


def ogc_mlp_blocked_bytes(plan: int, which: int) -> int:
    v = ctypes.c_size_t()
    _check(lib().ogc_mlp_blocked_bytes(plan, int(which), ctypes.byref(v)), "ogc_mlp_blocked_bytes")
    return v.value


def ogc_mlp_chosen_mode(plan: int) -> int:
    v = ctypes.c_int32()
    _check(lib().ogc_mlp_chosen_mode(plan, ctypes.byref(v)), "ogc_mlp_chosen_mode")
    return v.value


def ogc_mlp_buffer_assignment(plan: int, layer: int):
    s, o = ctypes.c_int32(), ctypes.c_size_t()
    _check(lib().ogc_mlp_buffer_assignment(plan, int(layer), ctypes.byref(s), ctypes.byref(o)), "ogc_mlp_buffer_assignment")
    return s.value, o.value


def _ptr_array(ptrs: Optional[Sequence[Optional[int]]], n: int):
    if ptrs is None:
        return None
    arr = (ctypes.c_void_p * max(n, 1))()
    for i in range(n):
        arr[i] = ptrs[i] if ptrs[i] else None
    return arr


def ogc_mlp_prepack_weights(plan: int, w_ptrs, bias_ptrs, w_scale_ptrs, packed_ptr: int, stream: int = 0) -> None:
    n = len(w_ptrs)
    _check(lib().ogc_mlp_prepack_weights(plan, _ptr_array(w_ptrs, n), _ptr_array(bias_ptrs, n), _ptr_array(w_scale_ptrs, n),
                                         packed_ptr, stream), "ogc_mlp_prepack_weights")


def ogc_mlp_run(plan: int, x_ptr: int, y_ptr: int, packed_ptr: int, workspace_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_mlp_run(plan, x_ptr, y_ptr, packed_ptr, workspace_ptr or None, stream), "ogc_mlp_run")


def ogc_mlp_run_static(plan: int, x_ptr: int, y_ptr: int, packed_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_mlp_run_static(plan, x_ptr, y_ptr, packed_ptr, stream), "ogc_mlp_run_static")


def ogc_quantize_e4m3(x: int, out: int, n: int, scale: float, stream: int = 0) -> None:
    _check(lib().ogc_quantize_e4m3(x, out, n, scale, stream), "ogc_quantize_e4m3")


def ogc_dequantize_e4m3(x: int, out: int, n: int, scale: float, stream: int = 0) -> None:
    _check(lib().ogc_dequantize_e4m3(x, out, n, scale, stream), "ogc_dequantize_e4m3")


def ogc_mlp_static_workspace_limit() -> int:
    return int(lib().ogc_mlp_static_workspace_limit())


def ogc_mlp_num_launches(plan: int) -> int:
    v = ctypes.c_int32()
    _check(lib().ogc_mlp_num_launches(plan, ctypes.byref(v)), "ogc_mlp_num_launches")
    return v.value


def ogc_mlp_run_clocked(plan: int, x_ptr: int, y_ptr: int, packed_ptr: int, workspace_ptr: int, clocks_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_mlp_run_clocked(plan, x_ptr, y_ptr, packed_ptr, workspace_ptr or None, stream, clocks_ptr), "ogc_mlp_run_clocked")


def ogc_mlp_clock_words_per_launch() -> int:
    return int(lib().ogc_mlp_clock_words_per_launch())


def ogc_mlp_run_profiled(plan: int, x_ptr: int, y_ptr: int, packed_ptr: int, workspace_ptr: int, stream: int = 0):
    """Returns the list of per-launch durations in milliseconds."""
    n = ogc_mlp_num_launches(plan)
    ms = (ctypes.c_float * n)()
    _check(lib().ogc_mlp_run_profiled(plan, x_ptr, y_ptr, packed_ptr, workspace_ptr or None, stream, ms), "ogc_mlp_run_profiled")
    return [float(v) for v in ms]


def ogc_mlp_estimated_us(plan: int, layer: int) -> float:
    v = ctypes.c_float()
    _check(lib().ogc_mlp_estimated_us(plan, int(layer), ctypes.byref(v)), "ogc_mlp_estimated_us")
    return v.value


def ogc_mlp_mode_estimates(plan: int):
    """(per layer, fused, cooperative) estimates of the whole chain in microseconds; -1 where not admissible."""
    v = (ctypes.c_float * 3)()
    _check(lib().ogc_mlp_mode_estimates(plan, v), "ogc_mlp_mode_estimates")
    return tuple(float(x) for x in v)


def ogc_mlp_destroy(plan: int) -> None:
    lib().ogc_mlp_destroy(plan)


def ogc_mlp_kernel_name(plan: int, layer: int) -> str:
    r = lib().ogc_mlp_kernel_name(plan, int(layer))
    return r.decode() if r else ""


def mha_desc(dtype: int, batch: int, heads: int, seq: int, head_dim: int, scale: float, softmax: int = OGC_SOFTMAX_STABLE,
             q_stride=None, k_stride=None, v_stride=None, o_stride=None, query_groups: int = 0) -> ogc_mha_desc:
    """Strides default to the [batch, seq, heads*head_dim] layout."""
    plain = (seq * heads * head_dim, head_dim, heads * head_dim)
    arrs = [(ctypes.c_int64 * 3)(*[int(v) for v in (st if st is not None else plain)])
            for st in (q_stride, k_stride, v_stride, o_stride)]
    return ogc_mha_desc(int(dtype), int(batch), int(heads), int(seq), int(head_dim), int(softmax), float(scale), *arrs,
                        int(query_groups))


def ogc_mha_validate(desc: ogc_mha_desc) -> int:
    return int(lib().ogc_mha_validate(ctypes.byref(desc)))


def ogc_mha_run(desc: ogc_mha_desc, q_ptr: int, k_ptr: int, v_ptr: int, mask_ptr: int, o_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_mha_run(ctypes.byref(desc), q_ptr or None, k_ptr or None, v_ptr or None, mask_ptr or None, o_ptr or None,
                             stream), "ogc_mha_run")


def ogc_mha_i8_validate(desc: ogc_mha_desc, quant: ogc_mha_quant) -> int:
    return int(lib().ogc_mha_i8_validate(ctypes.byref(desc), ctypes.byref(quant)))


def ogc_mha_run_i8(desc: ogc_mha_desc, quant: ogc_mha_quant, q_ptr: int, k_ptr: int, v_ptr: int, mask_ptr: int, o_ptr: int,
                   stream: int = 0) -> None:
    _check(lib().ogc_mha_run_i8(ctypes.byref(desc), ctypes.byref(quant), q_ptr or None, k_ptr or None, v_ptr or None,
                                mask_ptr or None, o_ptr or None, stream), "ogc_mha_run_i8")


def ogc_mha_i8_kernel_name(desc: ogc_mha_desc) -> str:
    r = lib().ogc_mha_i8_kernel_name(ctypes.byref(desc))
    return r.decode() if r else ""


def ogc_mha_kernel_name(desc: ogc_mha_desc, has_mask: bool = True) -> str:
    r = lib().ogc_mha_kernel_name(ctypes.byref(desc), int(bool(has_mask)))
    return r.decode() if r else ""


# ---- a decoder's attention block (include/ogc_decoder.h); strides are (row, head), in elements
def _two(stride):
    return (ctypes.c_int64 * 2)(int(stride[0]), int(stride[1]))


def rope_desc(dtype: int, tokens: int, q_heads: int, kv_heads: int, head_dim: int, rot_dim: int, layout: int, norm: int, eps: float,
              magnitude: float, q_stride, k_stride, qo_stride, ko_stride) -> ogc_rope_desc:
    return ogc_rope_desc(int(dtype), int(tokens), int(q_heads), int(kv_heads), int(head_dim), int(rot_dim), int(layout), int(norm),
                         float(eps), float(magnitude), _two(q_stride), _two(k_stride), _two(qo_stride), _two(ko_stride))


def ogc_rope_validate(desc: ogc_rope_desc) -> int:
    return int(lib().ogc_rope_validate(desc))


def ogc_rope_run(desc: ogc_rope_desc, q_ptr: int, k_ptr: int, q_weight_ptr: int, k_weight_ptr: int, positions_ptr: int,
                 frequencies_ptr: int, q_out_ptr: int, k_out_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_rope_run(desc, q_ptr, k_ptr, q_weight_ptr, k_weight_ptr, positions_ptr, frequencies_ptr, q_out_ptr, k_out_ptr,
                              stream), "ogc_rope_run")


def kv4_desc(kv_heads: int, head_dim: int, page_size: int, pages: int, batch: int, table_width: int) -> ogc_kv4_desc:
    return ogc_kv4_desc(int(kv_heads), int(head_dim), int(page_size), int(pages), int(batch), int(table_width))


def kv4_rows(dtype: int, rows: int, max_rows: int, k_stride, v_stride) -> ogc_kv4_rows:
    return ogc_kv4_rows(int(dtype), int(rows), int(max_rows), _two(k_stride), _two(v_stride))


def ogc_kv4_validate(cache: ogc_kv4_desc, rows: ogc_kv4_rows) -> int:
    return int(lib().ogc_kv4_validate(cache, rows))


def ogc_kv4_cache_bytes(cache: ogc_kv4_desc) -> int:
    v = ctypes.c_size_t()
    _check(lib().ogc_kv4_cache_bytes(cache, ctypes.byref(v)), "ogc_kv4_cache_bytes")
    return v.value


def ogc_kv4_write(cache: ogc_kv4_desc, rows: ogc_kv4_rows, k_ptr: int, v_ptr: int, cu_ptr: int, start_ptr: int, table_ptr: int,
                  cache_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_kv4_write(cache, rows, k_ptr, v_ptr, cu_ptr, start_ptr, table_ptr, cache_ptr, stream), "ogc_kv4_write")


def ogc_kv4_read(cache: ogc_kv4_desc, rows: ogc_kv4_rows, cache_ptr: int, cu_ptr: int, start_ptr: int, table_ptr: int, k_ptr: int,
                 v_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_kv4_read(cache, rows, cache_ptr, cu_ptr, start_ptr, table_ptr, k_ptr, v_ptr, stream), "ogc_kv4_read")


def kv4_attention_desc(dtype: int, q_heads: int, rows: int, max_rows: int, max_keys: int, scale: float, q_stride,
                       o_stride) -> ogc_kv4_attention_desc:
    return ogc_kv4_attention_desc(int(dtype), int(q_heads), int(rows), int(max_rows), int(max_keys), float(scale), _two(q_stride),
                                  _two(o_stride))


def ogc_kv4_attention_validate(cache: ogc_kv4_desc, desc: ogc_kv4_attention_desc) -> int:
    return int(lib().ogc_kv4_attention_validate(cache, desc))


def ogc_kv4_attention_workspace_bytes(cache: ogc_kv4_desc, desc: ogc_kv4_attention_desc) -> int:
    v = ctypes.c_size_t()
    _check(lib().ogc_kv4_attention_workspace_bytes(cache, desc, ctypes.byref(v)), "ogc_kv4_attention_workspace_bytes")
    return v.value


def ogc_kv4_attention_run(cache: ogc_kv4_desc, desc: ogc_kv4_attention_desc, q_ptr: int, cu_ptr: int, lens_ptr: int, table_ptr: int,
                          cache_ptr: int, o_ptr: int, workspace_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_kv4_attention_run(cache, desc, q_ptr, cu_ptr, lens_ptr, table_ptr, cache_ptr, o_ptr, workspace_ptr, stream),
           "ogc_kv4_attention_run")


def prompt_desc(dtype: int, batch: int, q_heads: int, kv_heads: int, head_dim: int, q_rows: int, k_rows: int, max_q: int, max_k: int,
                scale: float, causal: int, q_stride, k_stride, v_stride, o_stride) -> ogc_prompt_desc:
    return ogc_prompt_desc(int(dtype), int(batch), int(q_heads), int(kv_heads), int(head_dim), int(q_rows), int(k_rows), int(max_q),
                           int(max_k), float(scale), int(causal), _two(q_stride), _two(k_stride), _two(v_stride), _two(o_stride))


def ogc_prompt_validate(desc: ogc_prompt_desc) -> int:
    return int(lib().ogc_prompt_validate(desc))


def ogc_prompt_run(desc: ogc_prompt_desc, q_ptr: int, k_ptr: int, v_ptr: int, cu_q_ptr: int, cu_k_ptr: int, o_ptr: int,
                   stream: int = 0) -> None:
    _check(lib().ogc_prompt_run(desc, q_ptr, k_ptr, v_ptr, cu_q_ptr, cu_k_ptr, o_ptr, stream), "ogc_prompt_run")


def ogc_prompt_kernel_name(desc: ogc_prompt_desc) -> str:
    r = lib().ogc_prompt_kernel_name(desc)
    return r.decode() if r else ""


# ---- a decoder's projections in microscaled formats (include/ogc_mx.h); strides in elements
def ogc_mx_bytes(fmt: int, rows: int, channels: int):
    """Bytes of a microscaled matrix: (codes, scales)."""
    codes, scales = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().ogc_mx_bytes(int(fmt), int(rows), int(channels), ctypes.byref(codes), ctypes.byref(scales)), "ogc_mx_bytes")
    return codes.value, scales.value


def norm_desc(dtype: int, rows: int, channels: int, out: int, eps: float, x_stride: int, residual_stride: int = 0, sum_stride: int = 0,
              y_stride: int = 0) -> ogc_norm_desc:
    return ogc_norm_desc(int(dtype), int(rows), int(channels), int(out), float(eps), int(x_stride), int(residual_stride), int(sum_stride),
                         int(y_stride))


def ogc_norm_validate(desc: ogc_norm_desc) -> int:
    return int(lib().ogc_norm_validate(desc))


def ogc_norm_run(desc: ogc_norm_desc, x_ptr: int, residual_ptr: int, weight_ptr: int, sum_ptr: int, y_ptr: int, scales_ptr: int = 0,
                 stream: int = 0) -> None:
    _check(lib().ogc_norm_run(desc, x_ptr, residual_ptr, weight_ptr, sum_ptr, y_ptr, scales_ptr, stream), "ogc_norm_run")


def mx_rows(dtype: int, fmt: int, rows: int, channels: int, gate: int, stride: int) -> ogc_mx_rows:
    return ogc_mx_rows(int(dtype), int(fmt), int(rows), int(channels), int(gate), int(stride))


def ogc_mx_validate(rows: ogc_mx_rows) -> int:
    return int(lib().ogc_mx_validate(rows))


def ogc_mx_write(rows: ogc_mx_rows, x_ptr: int, codes_ptr: int, scales_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_mx_write(rows, x_ptr, codes_ptr, scales_ptr, stream), "ogc_mx_write")


def ogc_mx_read(rows: ogc_mx_rows, codes_ptr: int, scales_ptr: int, y_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_mx_read(rows, codes_ptr, scales_ptr, y_ptr, stream), "ogc_mx_read")


def mx_product_desc(dtype: int, x_format: int, w_format: int, m: int, n: int, k: int, has_bias: int, y_stride: int) -> ogc_mx_product_desc:
    return ogc_mx_product_desc(int(dtype), int(x_format), int(w_format), int(m), int(n), int(k), int(has_bias), int(y_stride))


def ogc_mx_product_validate(desc: ogc_mx_product_desc) -> int:
    return int(lib().ogc_mx_product_validate(desc))


def ogc_mx_product_workspace_bytes(desc: ogc_mx_product_desc) -> int:
    v = ctypes.c_size_t()
    _check(lib().ogc_mx_product_workspace_bytes(desc, ctypes.byref(v)), "ogc_mx_product_workspace_bytes")
    return v.value


def ogc_mx_product_run(desc: ogc_mx_product_desc, x_ptr: int, x_scales_ptr: int, w_ptr: int, w_scales_ptr: int, bias_ptr: int, y_ptr: int,
                       workspace_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_mx_product_run(desc, x_ptr, x_scales_ptr, w_ptr, w_scales_ptr, bias_ptr, y_ptr, workspace_ptr, stream),
           "ogc_mx_product_run")


def ogc_mx_product_kernel_name(desc: ogc_mx_product_desc) -> str:
    r = lib().ogc_mx_product_kernel_name(desc)
    return r.decode() if r else ""


# ---- the choice of a token (include/ogc_sample.h)
def sample_desc(dtype: int, rows: int, vocab: int, stride: int) -> ogc_sample_desc:
    return ogc_sample_desc(int(dtype), int(rows), int(vocab), int(stride))


def ogc_sample_validate(desc: ogc_sample_desc) -> int:
    return int(lib().ogc_sample_validate(desc))


def ogc_sample_workspace_bytes(desc: ogc_sample_desc) -> int:
    v = ctypes.c_size_t()
    _check(lib().ogc_sample_workspace_bytes(desc, ctypes.byref(v)), "ogc_sample_workspace_bytes")
    return v.value


def ogc_sample_run(desc: ogc_sample_desc, logits_ptr: int, temperature_ptr: int, top_k_ptr: int, top_p_ptr: int, min_p_ptr: int,
                   uniform_ptr: int, tokens_ptr: int, log_probabilities_ptr: int, workspace_ptr: int, stream: int = 0) -> None:
    _check(lib().ogc_sample_run(desc, logits_ptr, temperature_ptr, top_k_ptr, top_p_ptr, min_p_ptr, uniform_ptr, tokens_ptr,
                                log_probabilities_ptr, workspace_ptr, stream), "ogc_sample_run")


# ---- convenience wrapper: owns the torch tensors the library needs ---------------------------------
class FusedMLP:
    """plan + packed blob + workspace for one static MLP chain on the current CUDA/HIP device."""

    def __init__(self, dtype: str, m: int, layers: Sequence, ld_x: Optional[int] = None, ld_y: Optional[int] = None,
                 residual: bool = False, mode: int = OGC_MODE_AUTO, x_layout: int = OGC_LAYOUT_PLAIN,
                 y_layout: int = OGC_LAYOUT_PLAIN, overrides: Optional[dict] = None):
        import torch

        self.torch = torch
        self.dtype = dtype
        self.m = m
        self.layer_dicts = []
        for ly in layers:
            d = ly if isinstance(ly, dict) else dict(
                k=ly.k, n=ly.n, has_bias=int(ly.has_bias), act=ly.act, in_scale=ly.in_scale, in_zp=ly.in_zp,
                out_scale=ly.out_scale, out_zp=ly.out_zp, out=OGC_OUT_F32 if ly.out_f32 else OGC_OUT_SAME)
            self.layer_dicts.append(d)
        self.k0 = self.layer_dicts[0]["k"]
        self.n_last = self.layer_dicts[-1]["n"]
        self.ld_x = ld_x or self.k0
        self.ld_y = ld_y or self.n_last
        self.out_f32 = self.layer_dicts[-1].get("out", 0) == OGC_OUT_F32
        if overrides:
            self.plan = ogc_mlp_plan_with_overrides(DTYPES[dtype], m, self.layer_dicts, self.ld_x, self.ld_y, int(residual), mode,
                                                    x_layout, y_layout, overrides)
        else:
            self.plan = ogc_mlp_plan(DTYPES[dtype], m, self.layer_dicts, self.ld_x, self.ld_y, int(residual), mode, x_layout, y_layout)
        self.mode = ogc_mlp_chosen_mode(self.plan)
        self.packed_bytes = ogc_mlp_packed_bytes(self.plan)
        self.workspace_bytes = ogc_mlp_workspace_bytes(self.plan)
        self.packed = None
        self.workspace = None

    def close(self):
        if getattr(self, "plan", None):
            ogc_mlp_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self) -> int:
        return int(self.torch.cuda.current_stream().cuda_stream)

    def prepack(self, w: List, bias: Optional[List] = None, w_scale: Optional[List] = None) -> None:
        """w / bias / w_scale: lists of device tensors (bias and w_scale entries may be None)."""
        torch = self.torch
        dev = w[0].device
        self.packed = torch.empty(max(self.packed_bytes, 256), dtype=torch.uint8, device=dev)
        self.workspace = torch.empty(max(self.workspace_bytes, 256), dtype=torch.uint8, device=dev)
        wp = [t.data_ptr() for t in w]
        bp = None if bias is None else [None if t is None else t.data_ptr() for t in bias]
        sp = None if w_scale is None else [None if t is None else t.data_ptr() for t in w_scale]
        ogc_mlp_prepack_weights(self.plan, wp, bp, sp, self.packed.data_ptr(), self._stream())

    def run(self, x, y) -> None:
        ogc_mlp_run(self.plan, x.data_ptr(), y.data_ptr(), self.packed.data_ptr(),
                    self.workspace.data_ptr() if self.workspace_bytes else 0, self._stream())

    def check(self) -> int:
        """OGC_OK, or OGC_ERR_TIMEOUT if a barrier wait of the cooperative mode gave up since the last check."""
        return ogc_mlp_check(self.plan, self.packed.data_ptr(), self._stream())

    def run_clocked(self, x, y, clocks) -> None:
        ogc_mlp_run_clocked(self.plan, x.data_ptr(), y.data_ptr(), self.packed.data_ptr(),
                            self.workspace.data_ptr() if self.workspace_bytes else 0, clocks.data_ptr(), self._stream())

    def run_profiled(self, x, y):
        return ogc_mlp_run_profiled(self.plan, x.data_ptr(), y.data_ptr(), self.packed.data_ptr(),
                                    self.workspace.data_ptr() if self.workspace_bytes else 0, self._stream())
