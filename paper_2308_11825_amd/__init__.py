"""Python binding of libagcn (the MI355X Accel-GCN aggregation SpMM).

Argument marshalling only: every step of the path runs in the library's HIP
kernels. PyTorch supplies device memory and the current stream. The
low-level functions carry the C names of ``include/agcn.h``; ``Plan`` wraps
them for torch tensors.

The library must have been built (``python -m paper_2308_11825_amd.build``);
there is no fallback of any kind: if ``libagcn.so`` is missing, the functions that
need it raise. The functions of the routed layer's operators are compiled
(``_binding.so``, built with the library): their calls on a few rows take as long
as their marshalling does.
"""
from __future__ import annotations

import ctypes
import os

__all__ = [
    "LIB_PATH", "AgcnError", "load_library", "agcn_default_params", "agcn_plan_create",
    "agcn_spmm_workspace_size", "agcn_spmm", "agcn_spmm_timed", "agcn_plan_info",
    "agcn_plan_export", "agcn_plan_destroy", "agcn_status_string", "agcn_last_error",
    "agcn_release_cached_memory", "agcn_spmm_ex", "agcn_linear", "agcn_gcn_workspace_size",
    "agcn_gcn_layer", "agcn_spmm_noalloc", "AGCN_NOALLOC_MAX_WORKSPACE", "agcn_quantize_rows",
    "agcn_quantize_weight", "agcn_rms_norm", "agcn_quantized_linear", "agcn_grouped_linear",
    "agcn_quantize_rows_int", "agcn_quantize_weight_int", "agcn_int_linear",
    "agcn_grouped_int_linear", "agcn_layer_norm", "agcn_layer_norm_workspace_size",
    "agcn_layer_norm_backward", "agcn_sort_groups_workspace_size", "agcn_sort_groups",
    "agcn_dispatch", "agcn_combine", "agcn_combine_backward", "Plan", "linear", "quantize", "quantize_weight", "rms_norm", "quantized_linear",
    "grouped_linear", "quantize_int", "quantize_weight_int", "int_linear", "grouped_int_linear",
    "layer_norm", "layer_norm_backward", "sort_groups", "dispatch", "combine", "combine_backward",
    "PlanParams", "PlanStats", "EXPORTED_SYMBOLS",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libagcn.so")

EXPORTED_SYMBOLS = [
    "agcn_default_params", "agcn_plan_create", "agcn_spmm_workspace_size", "agcn_spmm",
    "agcn_spmm_timed", "agcn_plan_info", "agcn_plan_export", "agcn_plan_destroy",
    "agcn_status_string", "agcn_last_error", "agcn_release_cached_memory", "agcn_spmm_ex",
    "agcn_linear", "agcn_gcn_workspace_size", "agcn_gcn_layer", "agcn_spmm_noalloc",
    "agcn_quantize_rows", "agcn_quantize_weight", "agcn_rms_norm", "agcn_quantized_linear",
    "agcn_grouped_linear", "agcn_quantize_rows_int", "agcn_quantize_weight_int", "agcn_int_linear",
    "agcn_grouped_int_linear", "agcn_layer_norm", "agcn_layer_norm_workspace_size",
    "agcn_layer_norm_backward", "agcn_sort_groups_workspace_size", "agcn_sort_groups",
    "agcn_dispatch", "agcn_combine", "agcn_combine_backward",
]

AGCN_OK = 0
AGCN_ERR_INVALID_ARGUMENT = 1
AGCN_ERR_INVALID_INPUT = 2
AGCN_ERR_UNSUPPORTED = 3
AGCN_ERR_OUT_OF_MEMORY = 4
AGCN_ERR_HIP = 5

AGCN_PLAN_WARP_LEVEL = 0x1
AGCN_PLAN_COLUMN_LOOP = 0x2

AGCN_NOALLOC_MAX_WORKSPACE = 64 << 20

AGCN_EPILOGUE_NONE = 0
AGCN_EPILOGUE_RELU = 1
AGCN_FLOAT = 0
AGCN_BFLOAT = 1
AGCN_HALF = 2

_EPILOGUES = {None: AGCN_EPILOGUE_NONE, "none": AGCN_EPILOGUE_NONE, "relu": AGCN_EPILOGUE_RELU}


class PlanParams(ctypes.Structure):
    _fields_ = [("max_block_waves", ctypes.c_int32), ("max_wave_nzs", ctypes.c_int32),
                ("hub_chunk_nnz", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class PlanStats(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int32), ("n_cols", ctypes.c_int32), ("nnz", ctypes.c_int64),
                ("n_entries", ctypes.c_int64), ("hub_first_entry", ctypes.c_int64),
                ("n_hub_chunks", ctypes.c_int64), ("n_hub_rows", ctypes.c_int32),
                ("hub_first_row", ctypes.c_int32), ("deg_bound", ctypes.c_int32),
                ("hub_chunk_nnz", ctypes.c_int32), ("max_deg", ctypes.c_int32),
                ("max_block_waves", ctypes.c_int32), ("max_wave_nzs", ctypes.c_int32),
                ("flags", ctypes.c_uint32), ("device_bytes", ctypes.c_size_t),
                ("hub_windows", ctypes.c_int32)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class AgcnError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


_STATUS = {0: "AGCN_OK", 1: "AGCN_ERR_INVALID_ARGUMENT", 2: "AGCN_ERR_INVALID_INPUT",
           3: "AGCN_ERR_UNSUPPORTED", 4: "AGCN_ERR_OUT_OF_MEMORY", 5: "AGCN_ERR_HIP"}

_lib = None
_vp = ctypes.c_void_p


def _hip_runtimes_loaded():
    try:
        with open("/proc/self/maps") as f:
            maps = f.read()
    except OSError:
        return []
    import re
    return sorted(set(re.findall(r"(/\S*libamdhip64\.so[.0-9]*)", maps)))


def load_library(path: str | None = None):
    """Load libagcn.so (raises if it has not been built).

    PyTorch ships its own HIP runtime with the same SONAME as ROCm's. Loading
    torch first makes libagcn bind to that runtime, so torch's streams and
    allocations are valid in the library; two runtimes in one process would
    not share them, so that case raises.
    """
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise ImportError(f"{p} is missing: build it with `python -m paper_2308_11825_amd.build`")
    try:
        import torch  # noqa: F401  (binds the HIP runtime first)
    except ImportError:
        pass
    lib = ctypes.CDLL(p)
    runtimes = _hip_runtimes_loaded()
    if len(runtimes) > 1:
        raise ImportError(f"two HIP runtimes loaded in one process: {runtimes}; import torch "
                          "before loading libagcn")
    lib.agcn_default_params.argtypes = [ctypes.POINTER(PlanParams)]
    lib.agcn_default_params.restype = None
    lib.agcn_plan_create.argtypes = [ctypes.POINTER(_vp), ctypes.c_int32, ctypes.c_int32,
                                     ctypes.c_int64, _vp, _vp, _vp, ctypes.POINTER(PlanParams), _vp]
    lib.agcn_plan_create.restype = ctypes.c_int
    lib.agcn_spmm_workspace_size.argtypes = [_vp, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
    lib.agcn_spmm_workspace_size.restype = ctypes.c_int
    lib.agcn_spmm.argtypes = [_vp, ctypes.c_int32, _vp, ctypes.c_int64, _vp, ctypes.c_int64, _vp,
                              _vp]
    lib.agcn_spmm.restype = ctypes.c_int
    lib.agcn_spmm_timed.argtypes = [_vp, ctypes.c_int32, _vp, ctypes.c_int64, _vp, ctypes.c_int64,
                                    _vp, _vp, _vp, _vp, _vp]
    lib.agcn_spmm_timed.restype = ctypes.c_int
    lib.agcn_spmm_ex.argtypes = [_vp, ctypes.c_int32, _vp, ctypes.c_int64, _vp, ctypes.c_int64,
                                 _vp, _vp, ctypes.c_int32]
    lib.agcn_spmm_ex.restype = ctypes.c_int
    lib.agcn_spmm_noalloc.argtypes = [_vp, ctypes.c_int32, _vp, ctypes.c_int64, _vp,
                                      ctypes.c_int64, _vp, ctypes.c_int32]
    lib.agcn_spmm_noalloc.restype = ctypes.c_int
    lib.agcn_linear.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, _vp,
                                ctypes.c_int64, _vp, ctypes.c_int64, _vp, ctypes.c_int64, _vp]
    lib.agcn_linear.restype = ctypes.c_int
    lib.agcn_gcn_workspace_size.argtypes = [_vp, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
    lib.agcn_gcn_workspace_size.restype = ctypes.c_int
    lib.agcn_gcn_layer.argtypes = [_vp, ctypes.c_int32, ctypes.c_int32, _vp, ctypes.c_int64, _vp,
                                   ctypes.c_int64, _vp, ctypes.c_int64, _vp, _vp, ctypes.c_int32]
    lib.agcn_gcn_layer.restype = ctypes.c_int
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    lib.agcn_quantize_rows.argtypes = [i64, i32, i32, _vp, i64, _vp, i64, _vp, i64, _vp]
    lib.agcn_quantize_rows.restype = ctypes.c_int
    lib.agcn_quantize_weight.argtypes = [i32, i32, i32, i32, _vp, i64, i64, _vp, i64, i64, _vp, i64,
                                         i64, _vp]
    lib.agcn_quantize_weight.restype = ctypes.c_int
    lib.agcn_rms_norm.argtypes = [i64, i32, i32, _vp, i64, _vp, i64, _vp, i64, _vp, i32,
                                  ctypes.c_float, _vp, i64, _vp, i64, _vp]
    lib.agcn_rms_norm.restype = ctypes.c_int
    lib.agcn_quantized_linear.argtypes = [i64, i32, i32, _vp, i64, _vp, i64, _vp, i64, _vp, i64,
                                          i32, _vp, i64, _vp, i32]
    lib.agcn_quantized_linear.restype = ctypes.c_int
    lib.agcn_grouped_linear.argtypes = [i64, i32, i32, i32, _vp, i64, _vp, i64, _vp, i64, i64, _vp,
                                        i64, i64, _vp, i32, _vp, i64, _vp, i32]
    lib.agcn_grouped_linear.restype = ctypes.c_int
    lib.agcn_quantize_rows_int.argtypes = [i64, i32, i32, _vp, i64, _vp, i64, _vp, _vp]
    lib.agcn_quantize_weight_int.argtypes = [i32, i32, i32, i32, _vp, i64, i64, _vp, i64, i64, _vp,
                                             i64, _vp]
    lib.agcn_int_linear.argtypes = [i64, i32, i32, _vp, i64, _vp, _vp, i64, _vp, i32, _vp, i64, _vp,
                                    i32]
    lib.agcn_grouped_int_linear.argtypes = [i64, i32, i32, i32, _vp, i64, _vp, _vp, i64, i64, _vp,
                                            i64, _vp, i32, _vp, i64, _vp, i32]
    lib.agcn_layer_norm.argtypes = [i64, i32, i32, _vp, i64, _vp, i64, _vp, i64, _vp, _vp, i32,
                                    ctypes.c_float, _vp, i64, _vp, i64, _vp]
    lib.agcn_layer_norm_workspace_size.argtypes = [i64, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.agcn_layer_norm_backward.argtypes = [i64, i32, i32, _vp, i64, _vp, i64, _vp, i64, _vp, i64,
                                             _vp, i32, _vp, i64, _vp, _vp, _vp, _vp]
    lib.agcn_sort_groups_workspace_size.argtypes = [i64, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.agcn_sort_groups.argtypes = [i64, i32, i32, _vp, i32, i64, _vp, _vp, i64, _vp, _vp]
    lib.agcn_dispatch.argtypes = [i64, i32, i64, _vp, i64, _vp, i64, _vp, i64, _vp]
    lib.agcn_combine.argtypes = [i64, i32, i32, i32, _vp, i64, _vp, i64, _vp, i64, _vp, i64, _vp]
    lib.agcn_combine_backward.argtypes = [i64, i32, i32, i32, _vp, i64, _vp, i64, _vp, i64, _vp, i64,
                                          _vp, i64, _vp, i64, _vp]
    for name in EXPORTED_SYMBOLS[EXPORTED_SYMBOLS.index("agcn_quantize_rows_int"):]:
        getattr(lib, name).restype = ctypes.c_int
    lib.agcn_plan_info.argtypes = [_vp, ctypes.POINTER(PlanStats)]
    lib.agcn_plan_info.restype = ctypes.c_int
    lib.agcn_plan_export.argtypes = [_vp, _vp, _vp, _vp, _vp, _vp]
    lib.agcn_plan_export.restype = ctypes.c_int
    lib.agcn_plan_destroy.argtypes = [_vp]
    lib.agcn_plan_destroy.restype = None
    lib.agcn_release_cached_memory.argtypes = []
    lib.agcn_release_cached_memory.restype = None
    lib.agcn_status_string.argtypes = [ctypes.c_int]
    lib.agcn_status_string.restype = ctypes.c_char_p
    lib.agcn_last_error.argtypes = []
    lib.agcn_last_error.restype = ctypes.c_char_p
    if path is None:
        _lib = lib
    return lib


def _check(rc):
    if rc != AGCN_OK:
        raise AgcnError(rc, agcn_last_error())


# ---- same-name wrappers of the C ABI (integers are raw device/host addresses) ----

def agcn_default_params() -> PlanParams:
    p = PlanParams()
    load_library().agcn_default_params(ctypes.byref(p))
    return p


def agcn_plan_create(n_rows, n_cols, nnz, d_rowptr, d_colidx, d_vals, params=None, stream=0):
    """Returns the plan handle (int). Raises AgcnError on failure."""
    h = _vp()
    prm = ctypes.byref(params) if params is not None else None
    _check(load_library().agcn_plan_create(ctypes.byref(h), n_rows, n_cols, nnz, d_rowptr, d_colidx,
                                           d_vals, prm, stream))
    return h.value


def agcn_spmm_workspace_size(plan, F) -> int:
    n = ctypes.c_size_t()
    _check(load_library().agcn_spmm_workspace_size(plan, F, ctypes.byref(n)))
    return n.value


def agcn_spmm(plan, F, d_X, ldx, d_Y, ldy, d_ws=None, stream=0):
    _check(load_library().agcn_spmm(plan, F, d_X, ldx, d_Y, ldy, d_ws, stream))


def agcn_spmm_timed(plan, F, d_X, ldx, d_Y, ldy, d_ws, stream, ev_begin, ev_mid, ev_end):
    _check(load_library().agcn_spmm_timed(plan, F, d_X, ldx, d_Y, ldy, d_ws, stream, ev_begin,
                                          ev_mid, ev_end))


def agcn_spmm_ex(plan, F, d_X, ldx, d_Y, ldy, d_ws, stream, epilogue):
    _check(load_library().agcn_spmm_ex(plan, F, d_X, ldx, d_Y, ldy, d_ws, stream, epilogue))


def agcn_spmm_noalloc(plan, F, d_X, ldx, d_Y, ldy, stream, epilogue=AGCN_EPILOGUE_NONE):
    _check(load_library().agcn_spmm_noalloc(plan, F, d_X, ldx, d_Y, ldy, stream, epilogue))


def agcn_linear(n, fin, fout, d_X, ldx, d_W, ldw, d_H, ldh, stream=0):
    _check(load_library().agcn_linear(n, fin, fout, d_X, ldx, d_W, ldw, d_H, ldh, stream))


def agcn_gcn_workspace_size(plan, fout) -> int:
    n = ctypes.c_size_t()
    _check(load_library().agcn_gcn_workspace_size(plan, fout, ctypes.byref(n)))
    return n.value


def agcn_gcn_layer(plan, fin, fout, d_X, ldx, d_W, ldw, d_Y, ldy, d_ws, stream, epilogue):
    _check(load_library().agcn_gcn_layer(plan, fin, fout, d_X, ldx, d_W, ldw, d_Y, ldy, d_ws,
                                         stream, epilogue))


def agcn_quantize_rows(n, f, dtype, d_X, ldx, d_Q, ldq, d_S, lds, stream=0):
    _check(load_library().agcn_quantize_rows(n, f, dtype, d_X, ldx, d_Q, ldq, d_S, lds, stream))


def agcn_quantize_weight(groups, fin, fout, dtype, d_W, ldw, group_w, d_Q, ldq, group_q, d_S, lds,
                         group_s, stream=0):
    _check(load_library().agcn_quantize_weight(groups, fin, fout, dtype, d_W, ldw, group_w, d_Q,
                                               ldq, group_q, d_S, lds, group_s, stream))


def agcn_rms_norm(n, f, dtype, d_X, ldx, d_R, ldr, d_H, ldh, d_g, g_dtype, eps, d_Q, ldq, d_S, lds,
                  stream=0):
    _check(load_library().agcn_rms_norm(n, f, dtype, d_X, ldx, d_R, ldr, d_H, ldh, d_g, g_dtype,
                                        eps, d_Q, ldq, d_S, lds, stream))


def agcn_quantized_linear(n, fin, fout, d_Q, ldq, d_S, lds, d_WQ, ldwq, d_WS, ldws, dtype, d_Y, ldy,
                          stream=0, epilogue=AGCN_EPILOGUE_NONE):
    _check(load_library().agcn_quantized_linear(n, fin, fout, d_Q, ldq, d_S, lds, d_WQ, ldwq, d_WS,
                                                ldws, dtype, d_Y, ldy, stream, epilogue))


def agcn_grouped_linear(n, fin, fout, groups, d_Q, ldq, d_S, lds, d_WQ, ldwq, group_wq, d_WS, ldws,
                        group_ws, d_offsets, dtype, d_Y, ldy, stream=0,
                        epilogue=AGCN_EPILOGUE_NONE):
    _check(load_library().agcn_grouped_linear(n, fin, fout, groups, d_Q, ldq, d_S, lds, d_WQ, ldwq,
                                              group_wq, d_WS, ldws, group_ws, d_offsets, dtype, d_Y,
                                              ldy, stream, epilogue))


def agcn_quantize_rows_int(n, f, dtype, d_X, ldx, d_Q, ldq, d_S, stream=0):
    _check(load_library().agcn_quantize_rows_int(n, f, dtype, d_X, ldx, d_Q, ldq, d_S, stream))


def agcn_quantize_weight_int(groups, fin, fout, dtype, d_W, ldw, group_w, d_Q, ldq, group_q, d_S,
                             group_s, stream=0):
    _check(load_library().agcn_quantize_weight_int(groups, fin, fout, dtype, d_W, ldw, group_w, d_Q,
                                                   ldq, group_q, d_S, group_s, stream))


def agcn_int_linear(n, fin, fout, d_Q, ldq, d_S, d_WQ, ldwq, d_WS, dtype, d_Y, ldy, stream=0,
                    epilogue=AGCN_EPILOGUE_NONE):
    _check(load_library().agcn_int_linear(n, fin, fout, d_Q, ldq, d_S, d_WQ, ldwq, d_WS, dtype, d_Y,
                                          ldy, stream, epilogue))


def agcn_grouped_int_linear(n, fin, fout, groups, d_Q, ldq, d_S, d_WQ, ldwq, group_wq, d_WS, group_ws,
                            d_offsets, dtype, d_Y, ldy, stream=0, epilogue=AGCN_EPILOGUE_NONE):
    _check(load_library().agcn_grouped_int_linear(n, fin, fout, groups, d_Q, ldq, d_S, d_WQ, ldwq,
                                                  group_wq, d_WS, group_ws, d_offsets, dtype, d_Y,
                                                  ldy, stream, epilogue))


def agcn_layer_norm(n, f, dtype, d_X, ldx, d_R, ldr, d_H, ldh, d_g, d_b, p_dtype, eps, d_Y, ldy,
                    d_stats, lds, stream=0):
    _check(load_library().agcn_layer_norm(n, f, dtype, d_X, ldx, d_R, ldr, d_H, ldh, d_g, d_b,
                                          p_dtype, eps, d_Y, ldy, d_stats, lds, stream))


def agcn_layer_norm_workspace_size(n, f, dtype) -> int:
    b = ctypes.c_size_t()
    _check(load_library().agcn_layer_norm_workspace_size(n, f, dtype, ctypes.byref(b)))
    return b.value


def agcn_layer_norm_backward(n, f, dtype, d_dY, lddy, d_H, ldh, d_dH, lddh, d_stats, lds, d_g,
                             p_dtype, d_dX, lddx, d_dg, d_db, d_ws, stream=0):
    _check(load_library().agcn_layer_norm_backward(n, f, dtype, d_dY, lddy, d_H, ldh, d_dH, lddh,
                                                   d_stats, lds, d_g, p_dtype, d_dX, lddx, d_dg,
                                                   d_db, d_ws, stream))


def agcn_sort_groups_workspace_size(n, k, groups) -> int:
    b = ctypes.c_size_t()
    _check(load_library().agcn_sort_groups_workspace_size(n, k, groups, ctypes.byref(b)))
    return b.value


def agcn_sort_groups(n, k, groups, d_ids, id_bytes, ldi, d_offsets, d_place, ldp, d_ws, stream=0):
    _check(load_library().agcn_sort_groups(n, k, groups, d_ids, id_bytes, ldi, d_offsets, d_place,
                                           ldp, d_ws, stream))


def agcn_dispatch(n, k, nbytes, d_X, ldx, d_place, ldp, d_Y, ldy, stream=0):
    _check(load_library().agcn_dispatch(n, k, nbytes, d_X, ldx, d_place, ldp, d_Y, ldy, stream))


def agcn_combine(n, k, f, dtype, d_R, ldr, d_place, ldp, d_W, ldw, d_Y, ldy, stream=0):
    _check(load_library().agcn_combine(n, k, f, dtype, d_R, ldr, d_place, ldp, d_W, ldw, d_Y, ldy,
                                       stream))


def agcn_combine_backward(n, k, f, dtype, d_dY, lddy, d_R, ldr, d_place, ldp, d_W, ldw, d_dR, lddr,
                          d_dW, lddw, stream=0):
    _check(load_library().agcn_combine_backward(n, k, f, dtype, d_dY, lddy, d_R, ldr, d_place, ldp,
                                                d_W, ldw, d_dR, lddr, d_dW, lddw, stream))


def agcn_plan_info(plan) -> PlanStats:
    s = PlanStats()
    _check(load_library().agcn_plan_info(plan, ctypes.byref(s)))
    return s


def agcn_plan_export(plan, h_perm=None, h_rowptr_s=None, h_colidx_s=None, h_vals_s=None,
                     h_meta=None):
    _check(load_library().agcn_plan_export(plan, h_perm, h_rowptr_s, h_colidx_s, h_vals_s, h_meta))


def agcn_plan_destroy(plan):
    load_library().agcn_plan_destroy(plan)


def agcn_release_cached_memory():
    load_library().agcn_release_cached_memory()


def agcn_status_string(status) -> str:
    return load_library().agcn_status_string(status).decode()


def agcn_last_error() -> str:
    return load_library().agcn_last_error().decode()


# ---- torch-facing wrapper ----

def _stream_handle(device):
    """Handle of torch's current stream on `device`: what
    torch.cuda.current_stream(device).cuda_stream is, without the Stream
    object (1.9 us of a call of 11; where torch has the raw query)."""
    if _torch is None:
        _load_torch()
    if _raw_stream is None or device.index is None:
        return _torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(device.index)


def _handle_of(stream, device):
    """Handle of the stream that the caller chose, or of torch's current one. Nothing orders
    a stream of another device with the tensors."""
    if stream is None:
        return _stream_handle(device)
    if stream.device != device:
        raise ValueError(f"stream must be one of {device}, as the tensors are")
    return stream.cuda_stream


def _call(device, fn, *args):
    """fn(*args) with `device` current (the context only where it is not)."""
    if _torch is None:
        _load_torch()
    if _current_device is not None and _current_device() == device.index:
        return fn(*args)
    with _torch.cuda.device(device):
        return fn(*args)


def _written_out(name, t):
    """Refuses a lazily negated view (of the imaginary part of a conjugate): its memory is not its values."""
    if t.is_neg():
        raise TypeError(f"{name} must not be a lazily negated view: resolve_neg() writes it out")


def _unit_col_stride(t):
    return t.shape[1] <= 1 or t.shape[0] == 0 or t.stride(1) == 1


def _row_stride(t):
    """Row stride in elements; any value >= F is valid for 0 or 1 rows."""
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))


class Plan:
    """A degree-sorted, block-partitioned CSR matrix on one GPU.

    ``Plan(rowptr, colidx, vals, n_cols=None, max_block_waves=..., max_wave_nzs=...,
    hub_chunk_nnz=0)`` with int32 / int32 / float32 CUDA tensors; ``plan.spmm(X)``
    returns ``A @ X`` for a float32 CUDA tensor X of shape (n_cols, F).
    """

    def __init__(self, rowptr, colidx, vals, n_cols=None, max_block_waves=None,
                 max_wave_nzs=None, hub_chunk_nnz=None, flags=0, stream=None):
        import torch
        for name, t, dt in (("rowptr", rowptr, torch.int32), ("colidx", colidx, torch.int32),
                            ("vals", vals, torch.float32)):
            if not isinstance(t, torch.Tensor) or t.device.type != "cuda" or t.dtype != dt:
                raise TypeError(f"{name} must be a CUDA tensor of dtype {dt}")
            if t.dim() != 1 or not t.is_contiguous():
                raise ValueError(f"{name} must be 1-D and contiguous")
            _written_out(name, t)
        self.device = rowptr.device
        self.n_rows = rowptr.numel() - 1
        self.n_cols = self.n_rows if n_cols is None else int(n_cols)
        self.nnz = colidx.numel()
        if vals.numel() != self.nnz:
            raise ValueError("colidx and vals differ in length")
        prm = agcn_default_params()
        if max_block_waves is not None:
            prm.max_block_waves = max_block_waves
        if max_wave_nzs is not None:
            prm.max_wave_nzs = max_wave_nzs
        if hub_chunk_nnz is not None:
            prm.hub_chunk_nnz = hub_chunk_nnz
        prm.flags = flags
        self.params = prm
        self._handle = None
        st = _handle_of(stream, self.device)
        self._handle = _call(self.device, agcn_plan_create, self.n_rows, self.n_cols, self.nnz,
                             rowptr.data_ptr(), colidx.data_ptr() if self.nnz else None,
                             vals.data_ptr() if self.nnz else None, prm, st)
        # The plan's last kernel may still read the inputs: on another stream,
        # torch's allocator must not reuse their memory before it.
        if stream is not None:
            for t in (rowptr, colidx, vals):
                t.record_stream(stream)
        self.stats = agcn_plan_info(self._handle)
        self._ws = {}
        self._ws_bytes = {}  # F -> workspace bytes: the plan's, fixed

    @property
    def handle(self):
        if self._handle is None:
            raise RuntimeError("plan destroyed")
        return self._handle

    def workspace_bytes(self, F: int) -> int:
        return agcn_spmm_workspace_size(self.handle, F)

    def workspace(self, F: int, stream=None):
        """A cached device workspace for feature width F on `stream` (None if
        not needed). One per stream, so executes on different streams never
        share hub-row partials."""
        import torch
        nb = self._ws_bytes.get(F)
        if nb is None:
            nb = self._ws_bytes[F] = self.workspace_bytes(F)
        if nb == 0:
            return None
        key = (F, _handle_of(stream, self.device))
        ws = self._ws.get(key)
        if ws is None:
            # allocated on the stream that uses it, so torch's allocator orders
            # any later reuse of the memory after that stream's work
            with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device)):
                ws = torch.empty((nb + 3) // 4, dtype=torch.float32, device=self.device)
            self._ws[key] = ws
        return ws

    def spmm(self, X, out=None, ws=None, stream=None, act=None):
        """A @ X, with act ("relu") applied where Y is written."""
        import torch
        if not isinstance(X, torch.Tensor) or X.device != self.device or X.dtype != torch.float32:
            raise TypeError("X must be a float32 tensor on the plan's device")
        if X.dim() != 2 or X.shape[0] != self.n_cols or not _unit_col_stride(X):
            raise ValueError("X must be (n_cols, F) with unit column stride")
        _written_out("X", X)
        F = X.shape[1]
        if F < 1:
            raise ValueError("F must be >= 1")
        if out is None:
            out = _new(X, stream, (self.n_rows, F), torch.float32)
        if (tuple(out.shape) != (self.n_rows, F) or not _unit_col_stride(out)
                or out.dtype != torch.float32 or out.device != self.device):
            raise ValueError("out must be a float32 (n_rows, F) tensor with unit column stride")
        _written_out("out", out)
        if ws is None:
            ws = self.workspace(F, stream)
        st = _on_stream(self.device, stream, (X, out, ws))
        _call(self.device, agcn_spmm_ex, self.handle, F, X.data_ptr(), _row_stride(X),
              out.data_ptr(), _row_stride(out), ws.data_ptr() if ws is not None else None, st,
              _EPILOGUES[act])
        return out

    def gcn_layer(self, X, W, act="relu", out=None, ws=None, stream=None):
        """One GCNConv forward: act(A @ (X @ W)), X (n_cols, fin), W (fin, fout)."""
        import torch
        for name, t in (("X", X), ("W", W)):
            if (not isinstance(t, torch.Tensor) or t.device != self.device
                    or t.dtype != torch.float32 or t.dim() != 2 or not _unit_col_stride(t)):
                raise TypeError(f"{name} must be a 2-D float32 tensor on the plan's device with "
                                "unit column stride")
            _written_out(name, t)
        fin, fout = W.shape
        if X.shape != (self.n_cols, fin):
            raise ValueError("X must be (n_cols, fin) with fin = W.shape[0]")
        if out is None:
            out = _new(X, stream, (self.n_rows, fout), torch.float32)
        if (tuple(out.shape) != (self.n_rows, fout) or not _unit_col_stride(out)
                or out.dtype != torch.float32 or out.device != self.device):
            raise ValueError("out must be a float32 (n_rows, fout) tensor with unit column stride")
        _written_out("out", out)
        if ws is None:
            nb = agcn_gcn_workspace_size(self.handle, fout)
            ws = _new(X, stream, ((nb + 3) // 4,), torch.float32)
        st = _on_stream(self.device, stream, (X, W, out, ws))
        _call(self.device, agcn_gcn_layer, self.handle, fin, fout, X.data_ptr(), _row_stride(X),
              W.data_ptr(), _row_stride(W), out.data_ptr(), _row_stride(out), ws.data_ptr(), st,
              _EPILOGUES[act])
        return out

    def export(self):
        """Host copies: dict(perm, rowptr_s, colidx_s, vals_s, meta (n_entries x 4))."""
        import numpy as np
        s = self.stats
        perm = np.empty(s.n_rows, np.int32)
        rowptr_s = np.empty(s.n_rows + 1, np.int32)
        colidx_s = np.empty(s.nnz, np.int32)
        vals_s = np.empty(s.nnz, np.float32)
        meta = np.empty((s.n_entries, 4), np.int32)
        import torch
        with torch.cuda.device(self.device):
            agcn_plan_export(self.handle, perm.ctypes.data, rowptr_s.ctypes.data,
                             colidx_s.ctypes.data, vals_s.ctypes.data, meta.ctypes.data)
        return dict(perm=perm, rowptr_s=rowptr_s, colidx_s=colidx_s, vals_s=vals_s, meta=meta)

    def destroy(self):
        if self._handle is not None:
            agcn_plan_destroy(self._handle)
            self._handle = None
        self._ws = {}
        self._ws_bytes = {}

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def linear(X, W, out=None, stream=None):
    """X @ W on the matrix cores: X (n, fin), W (fin, fout), float32 CUDA tensors."""
    import torch
    for name, t in (("X", X), ("W", W)):
        if (not isinstance(t, torch.Tensor) or t.device.type != "cuda" or t.dtype != torch.float32
                or t.dim() != 2 or not _unit_col_stride(t)):
            raise TypeError(f"{name} must be a 2-D float32 CUDA tensor with unit column stride")
        _written_out(name, t)
    n, fin = X.shape
    if W.shape[0] != fin or W.device != X.device:
        raise ValueError("W must be (fin, fout) on X's device")
    fout = W.shape[1]
    if out is None:
        out = _new(X, stream, (n, fout), torch.float32)
    if (tuple(out.shape) != (n, fout) or not _unit_col_stride(out) or out.dtype != torch.float32
            or out.device != X.device):
        raise ValueError("out must be a float32 (n, fout) tensor with unit column stride on X's device")
    _written_out("out", out)
    st = _on_stream(X.device, stream, (X, W, out))
    _call(X.device, agcn_linear, n, fin, fout, X.data_ptr(), _row_stride(X), W.data_ptr(),
          _row_stride(W), out.data_ptr(), _row_stride(out), st)
    return out


# ---- 8-bit operators ----
#
# A matrix in 8 bits is a pair of tensors: the values Q (torch.float8_e4m3fn) and the
# scales S (torch.float8_e8m0fnu, powers of two), one per 128 columns of a row, or
# one per 128 x 128 block of a weight. It stands for Q times its scales.

_MOST_INT32 = 2 ** 31 - 1
_DTYPES = {}  # torch dtype -> AGCN_FLOAT, AGCN_BFLOAT, AGCN_HALF
_torch = None
_Q8 = _S8 = None  # the dtypes of values and of scales
_raw_stream = _current_device = None  # torch's raw queries, where it has them


def _load_torch():
    global _torch, _Q8, _S8, _raw_stream, _current_device
    import torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _current_device = getattr(torch._C, "_cuda_getDevice", None)
    _DTYPES.update({torch.float32: AGCN_FLOAT, torch.bfloat16: AGCN_BFLOAT,
                    torch.float16: AGCN_HALF})
    _Q8, _S8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    _torch = torch


def _matrix(name, t, device, shape, dtype):
    """The row stride of `t`, a matrix (or stacked ones) of this shape and type on `device`
    with unit column stride; refuses anything else. (In one pass over what a right
    tensor has: these checks are the larger part of a small call's time.)"""
    if isinstance(t, _torch.Tensor) and t.dtype is dtype and t.shape == shape and t.device == device:
        stride = t.stride()
        if t.is_neg():
            _written_out(name, t)
        if stride[-1] == 1 and shape[-2] > 1:
            return stride[-2]
        if shape[-1] <= 1 or t.numel() == 0 or stride[-1] == 1:
            # Any value >= a row is valid for 0 or 1 rows.
            return stride[-2] if shape[-2] > 1 else max(shape[-1], stride[-2])
        raise ValueError(f"{name} must have unit column stride, as its contiguous() has")
    if not isinstance(t, _torch.Tensor) or t.device != device:
        raise TypeError(f"{name} must be a tensor on {device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}")
    raise ValueError(f"{name} must have shape {tuple(shape)}")


def _first(name, t, dims, weight=False):
    """The shape and device of the tensor that sets a call's sizes and type."""
    if _torch is None:
        _load_torch()
    if not isinstance(t, _torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dim() != dims:
        raise ValueError(f"{name} must have {dims} dimensions")
    shape = t.shape
    # ctypes cuts what the library counts in 32 bits: all sizes but a matrix's rows.
    if shape[-1] > _MOST_INT32 or (weight and max(shape) > _MOST_INT32):
        raise ValueError(f"{name} must have at most 2^31 - 1 {'rows, columns and groups' if weight else 'columns'}")
    return shape, t.device


def _dtype_code(name, dtype):
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"{name} must have dtype float32, bfloat16 or float16")
    return code


def _on_stream(device, stream, tensors):
    """The stream's handle; on a stream of the caller's choice torch's allocator must
    not reuse the tensors' memory before its work."""
    if stream is None:
        return _stream_handle(device)
    st = _handle_of(stream, device)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return st


def _new(like, stream, shape, dtype):
    """A tensor on like's device, allocated on the stream that writes it."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    if _torch is None:
        _load_torch()
    _handle_of(stream, like.device)
    with _torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _new_rows(like, stream, lead, k, dtype=None):
    """Values (..., k) in 8 bits (e4m3 unless told otherwise) and their row stride: rows
    start on 16 bytes, on 128 (the lines of memory, which a block of 128 columns then is one
    of) where that adds an eighth at most: 230,000 x 602 -> 256 bfloat16 78 us with rows of 640
    bytes, 83 with 608."""
    ld = (k + 127) // 128 * 128
    if ld > k + k // 8:
        ld = (k + 15) // 16 * 16
    q = _new(like, stream, (*lead, ld), _Q8 if dtype is None else dtype)
    return (q[..., :k] if k != ld else q), ld


def quantize(X, out=None, stream=None):
    """The rows of X (n, f) in 8 bits: (Q, S). X: float32, bfloat16 or float16 CUDA
    tensor; out: such a pair to write to."""
    (n, f), device = _first("X", X, 2)
    dtype = X.dtype
    code, ldx, blocks = _dtype_code("X", dtype), _matrix("X", X, device, X.shape, dtype), (f + 127) // 128
    if out is None:
        Q, ldq = _new_rows(X, stream, (n,), f)
        S, lds = _new(X, stream, (n, blocks), _S8), blocks
    else:
        Q, S = out
        ldq = _matrix("out[0]", Q, device, (n, f), _Q8)
        lds = _matrix("out[1]", S, device, (n, blocks), _S8)
    st = _on_stream(device, stream, (X, Q, S))
    _call(device, agcn_quantize_rows, n, f, code, X.data_ptr(), ldx, Q.data_ptr(), ldq,
          S.data_ptr(), lds, st)
    return Q, S


def quantize_weight(W, stream=None):
    """A weight (fin, fout), as ``linear`` takes it, or one per group (groups, fin,
    fout), in 8 bits for ``quantized_linear`` and ``grouped_linear``: (WQ, WS) with WQ
    (..., fout, fin), transposed, and WS (..., ceil(fout / 128), ceil(fin / 128))."""
    shape, device = _first("W", W, 3 if getattr(W, "ndim", 2) == 3 else 2, weight=True)
    *lead, fin, fout = shape
    dtype = W.dtype
    code, ldw = _dtype_code("W", dtype), _matrix("W", W, device, shape, dtype)
    nb, kb = (fout + 127) // 128, (fin + 127) // 128
    Q, ldq = _new_rows(W, stream, (*lead, fout), fin)
    S = _new(W, stream, (*lead, nb, kb), _S8)
    st = _on_stream(device, stream, (W,))
    groups, strides = (lead[0], [t.stride(0) for t in (W, Q, S)]) if lead else (1, (0, 0, 0))
    _call(device, agcn_quantize_weight, groups, fin, fout, code, W.data_ptr(), ldw, strides[0],
          Q.data_ptr(), ldq, strides[1], S.data_ptr(), kb, strides[2], st)
    return Q, S


def rms_norm(X, weight, residual=None, eps=1e-6, hidden=None, out=None, stream=None):
    """y = h / sqrt(mean(h^2) + eps) * weight per row of h = X + residual, in 8 bits:
    (Q, S), and with a residual (Q, S, h).

    X, residual and h are (n, f) of one type (float32, bfloat16 or float16), weight (f,)
    of that type or float32. hidden: where h is written (X or residual itself will
    do); out: a pair (Q, S) to write to."""
    (n, f), device = _first("X", X, 2)
    dtype, shape = X.dtype, X.shape
    code, ldx, blocks = _dtype_code("X", dtype), _matrix("X", X, device, shape, dtype), (f + 127) // 128
    if not isinstance(weight, _torch.Tensor) or weight.device != device:
        raise TypeError("weight must be a tensor on X's device")
    g_code = _dtype_code("weight", weight.dtype)
    if g_code != code and g_code != AGCN_FLOAT:
        raise TypeError("weight must be float32 or of X's type")
    if weight.shape != (f,) or (f > 1 and weight.stride(0) != 1):
        raise ValueError("weight must be (f,) and contiguous")
    if weight.is_neg():
        _written_out("weight", weight)
    r = h = None
    ldr = ldh = 0
    if residual is not None:
        ldr = _matrix("residual", residual, device, shape, dtype)
        r = residual.data_ptr()
        if hidden is None:
            hidden, ldh = _new(X, stream, shape, dtype), f
        else:
            ldh = _matrix("hidden", hidden, device, shape, dtype)
        h = hidden.data_ptr()
    elif hidden is not None:
        raise ValueError("hidden needs a residual: without one h is X")
    if out is None:
        Q, ldq = _new_rows(X, stream, (n,), f)
        S, lds = _new(X, stream, (n, blocks), _S8), blocks
    else:
        Q, S = out
        ldq = _matrix("out[0]", Q, device, shape, _Q8)
        lds = _matrix("out[1]", S, device, (n, blocks), _S8)
    st = _on_stream(device, stream, (X, weight, residual, hidden, Q, S))
    _call(device, agcn_rms_norm, n, f, code, X.data_ptr(), ldx, r, ldr, h, ldh, weight.data_ptr(),
          g_code, eps, Q.data_ptr(), ldq, S.data_ptr(), lds, st)
    return (Q, S) if residual is None else (Q, S, hidden)


def _product(Q, S, WQ, WS, offsets, dtype, act, out, stream):
    shape, device = _first("Q", Q, 2)
    w_shape, _ = _first("WQ", WQ, 2 if offsets is None else 3, weight=True)
    n, fin = shape
    fout = w_shape[-2]
    nb, kb = (fout + 127) // 128, (fin + 127) // 128
    ldq = _matrix("Q", Q, device, shape, _Q8)
    lds = _matrix("S", S, device, (n, kb), _S8)
    lead = w_shape[:-2]
    ldwq = _matrix("WQ", WQ, device, (*lead, fout, fin), _Q8)
    ldws = _matrix("WS", WS, device, (*lead, nb, kb), _S8)
    epilogue = _EPILOGUES.get(act)
    if epilogue is None:
        raise ValueError("act must be None, 'none' or 'relu'")
    if out is None:
        dtype = _torch.float32 if dtype is None else dtype
        code = _dtype_code("the result", dtype)
        out, ldy = _new(Q, stream, (n, fout), dtype), fout
    else:
        code = _dtype_code("out", getattr(out, "dtype", None))
        ldy = _matrix("out", out, device, (n, fout), out.dtype if dtype is None else dtype)
    st = _on_stream(device, stream, (Q, S, WQ, WS, offsets, out))
    if offsets is None:
        _call(device, agcn_quantized_linear, n, fin, fout, Q.data_ptr(), ldq, S.data_ptr(), lds,
              WQ.data_ptr(), ldwq, WS.data_ptr(), ldws, code, out.data_ptr(), ldy, st, epilogue)
        return out
    groups = lead[0]
    if offsets.dtype is not _torch.int32 or offsets.device != device:
        raise TypeError("offsets must be int32 on the inputs' device")
    if offsets.shape != (groups + 1,) or (groups > 0 and offsets.stride(0) != 1):
        raise ValueError("offsets must be (groups + 1,) and contiguous")
    if offsets.is_neg():
        _written_out("offsets", offsets)
    _call(device, agcn_grouped_linear, n, fin, fout, groups, Q.data_ptr(), ldq, S.data_ptr(), lds,
          WQ.data_ptr(), ldwq, WQ.stride(0), WS.data_ptr(), ldws, WS.stride(0), offsets.data_ptr(),
          code, out.data_ptr(), ldy, st, epilogue)
    return out


def quantized_linear(Q, S, WQ, WS, dtype=None, act=None, out=None, stream=None):
    """act(A W^T), (n, fout), of A (n, fin) and W (fout, fin) in 8 bits, as ``quantize``
    or ``rms_norm`` and ``quantize_weight`` give them. dtype: float32 (the default),
    bfloat16 or float16; products are exact and sums in 32 bits, but for bfloat16, whose
    sums the 8-bit matrix instruction takes (1.5e-5 of the 2-norm); act: None or "relu"."""
    return _product(Q, S, WQ, WS, None, dtype, act, out, stream)


def grouped_linear(Q, S, WQ, WS, offsets, dtype=None, act=None, out=None, stream=None):
    """``quantized_linear`` with a weight per group of rows (expert, node type,
    relation): rows offsets[e] to offsets[e + 1] - 1 take WQ[e], WS[e]. offsets: int32 CUDA
    tensor of groups + 1 values that do not decrease, read on the device only; rows
    of no group are 0."""
    if not hasattr(offsets, "data_ptr"):
        raise TypeError("offsets must be an int32 CUDA tensor")
    return _product(Q, S, WQ, WS, offsets, dtype, act, out, stream)


# ---- products of 8-bit integers ----
#
# A matrix in 8-bit integers is a pair of tensors: the values Q (torch.int8) and a float32
# scale S for each row, or for each output of a weight. It stands for Q times its scales.

_native = None  # the compiled binding of these functions and of those below
_NATIVE = ["layer_norm", "layer_norm_workspace_size", "layer_norm_backward",
           "sort_groups_workspace_size", "sort_groups", "dispatch", "combine", "combine_backward",
           "quantize_rows_int", "int_linear", "grouped_int_linear", "last_error"]


def _call_native(name, stream, *args):
    """`name` of the compiled binding. It allocates on the current stream and runs there: the
    caller's, if one is given, and then torch's allocator must not reuse the tensors' memory
    before its work."""
    native = _native or _load_native()
    if stream is None:
        return getattr(native, name)(*args)
    if isinstance(args[0], _torch.Tensor) and args[0].is_cuda:
        _handle_of(stream, args[0].device)
    with _torch.cuda.stream(stream):
        results = getattr(native, name)(*args)
    for t in args:
        for t in t if isinstance(t, tuple) else (t,):
            if isinstance(t, _torch.Tensor):
                t.record_stream(stream)
    return results


def _load_native():
    global _native
    lib = load_library()
    if _torch is None:
        _load_torch()
    try:
        from . import _binding
    except ImportError as e:
        raise ImportError(f"the compiled binding is missing or does not fit this PyTorch ({e}): build it with "
                          "`python -m paper_2308_11825_amd.build`") from e
    _binding.init(AgcnError, _torch.OutOfMemoryError,
                  [ctypes.cast(getattr(lib, "agcn_" + n), _vp).value for n in _NATIVE])
    _native = _binding
    return _native


def quantize_int(X, out=None, stream=None):
    """The rows of X (n, f) in 8-bit integers: (Q, S), Q (n, f) int8 and S (n,) float32, a
    127th of the row's largest value. X: float32, bfloat16 or float16 CUDA tensor; out: such a
    pair to write to."""
    return _call_native("quantize_int", stream, X, out)


def quantize_weight_int(W, stream=None):
    """A weight (fin, fout), as ``linear`` takes it, or one per group (groups, fin, fout), in
    8-bit integers for ``int_linear`` and ``grouped_int_linear``: (WQ, WS) with WQ (..., fout,
    fin), transposed, and WS (..., fout) float32."""
    shape, device = _first("W", W, 3 if getattr(W, "ndim", 2) == 3 else 2, weight=True)
    *lead, fin, fout = shape
    dtype = W.dtype
    code, ldw = _dtype_code("W", dtype), _matrix("W", W, device, shape, dtype)
    Q, ldq = _new_rows(W, stream, (*lead, fout), fin, _torch.int8)
    S = _new(W, stream, (*lead, fout), _torch.float32)
    st = _on_stream(device, stream, (W,))
    groups, strides = (lead[0], [t.stride(0) for t in (W, Q, S)]) if lead else (1, (0, 0, 0))
    _call(device, agcn_quantize_weight_int, groups, fin, fout, code, W.data_ptr(), ldw, strides[0],
          Q.data_ptr(), ldq, strides[1], S.data_ptr(), strides[2], st)
    return Q, S


def _int_product(Q, S, WQ, WS, offsets, dtype, act, out, stream):
    epilogue = _EPILOGUES.get(act)
    if epilogue is None:
        raise ValueError("act must be None, 'none' or 'relu'")
    return _call_native("int_product", stream, Q, S, WQ, WS, offsets, dtype, epilogue, out)


def int_linear(Q, S, WQ, WS, dtype=None, act=None, out=None, stream=None):
    """act(A W^T), (n, fout), of A (n, fin) and W (fout, fin) in 8-bit integers, as
    ``quantize_int`` and ``quantize_weight_int`` give them. dtype: float32 (the default),
    bfloat16 or float16; the integers' sums are exact, fin below 2^17; act: None or "relu"."""
    return _int_product(Q, S, WQ, WS, None, dtype, act, out, stream)


def grouped_int_linear(Q, S, WQ, WS, offsets, dtype=None, act=None, out=None, stream=None):
    """``int_linear`` with a weight per group of rows, as ``grouped_linear``: rows offsets[e]
    to offsets[e + 1] - 1 take WQ[e], WS[e]; rows of no group are 0."""
    if not hasattr(offsets, "data_ptr"):
        raise TypeError("offsets must be an int32 CUDA tensor")
    return _int_product(Q, S, WQ, WS, offsets, dtype, act, out, stream)


# ---- layer norm ----

def layer_norm(X, weight, bias=None, residual=None, eps=1e-5, stats=False, hidden=None, out=None,
               stream=None):
    """y = (h - mean) / sqrt(var + eps) * weight + bias per row of h = X + residual: y; with a
    residual (y, h); with stats=True one more, (n, 2) float32, each row's mean and
    1 / sqrt(var + eps) for ``layer_norm_backward`` (no gradient is recorded).

    X, residual, h and y are (n, f) of one type (float32, bfloat16 or float16), weight and bias
    (f,) both of that type or float32. hidden: where h is written (X or residual itself will
    do); out: where y is."""
    return _call_native("layer_norm", stream, X, weight, bias, residual, eps, stats, hidden, out)


def layer_norm_backward(grad, H, stats, weight, bias=True, grad_hidden=None, out=None, stream=None):
    """Gradients of ``layer_norm`` from grad, that of y: (dX, dweight, dbias). H: the rows h (X
    where there was no residual); stats: as ``layer_norm`` gave them; grad_hidden: the gradient
    of h from elsewhere, added to dX, which is that of X and of the residual; bias=False: dbias
    is None; out: where dX is written. dweight and dbias have weight's type. (An expanded
    gradient, as that of a sum, is refused: its contiguous() copy will do, here and in
    ``combine_backward``.)"""
    return _call_native("layer_norm_backward", stream, grad, H, stats, weight, bias, grad_hidden, out)


# ---- rows sent to groups and back ----

def sort_groups(ids, groups, out=None, stream=None):
    """Sorts ids (n, k), each row's group ids (int32 or int64 CUDA tensor), by group: (offsets,
    place), int32. place (n, k): where each id goes, in the order of the groups and within a
    group of the ids; offsets (groups + 1,): group e has the places offsets[e] to
    offsets[e + 1] - 1, as ``grouped_linear`` takes them. Ids outside [0, groups) get the
    places from offsets[groups] on, written as -1 - place. out: such a pair to write to."""
    return _call_native("sort_groups", stream, ids, groups, out)


def dispatch(X, place, out=None, stream=None):
    """The rows of X (n, f), of any type, in group order: (n * k, f) with row place[t][c] = X[t],
    and rows of ids without a group 0. Rows of one-byte types start on 16 bytes or 128, as
    ``quantize_int`` lays them: a view of wider rows. The gradient of ``dispatch`` is ``combine`` of the
    rows' without weights (none is recorded)."""
    return _call_native("dispatch", stream, X, place, out)


def combine(R, place, weights=None, out=None, stream=None):
    """(n, f) with row t the sum over c of weights[t][c] R[place[t][c]], ids without a group left
    out: R (n * k, f) float32, bfloat16 or float16 rows in group order, place (n, k) as
    ``sort_groups`` gives it, weights (n, k) float32 or None (all 1). Added in 32 bits. No gradient is
    recorded: ``combine_backward`` gives it."""
    return _call_native("combine", stream, R, place, weights, out)


def combine_backward(grad, R, place, weights, out=None, stream=None):
    """Gradients of ``combine`` with weights from grad (n, f), that of its result: (dR, dweights),
    dR (n * k, f) of R's type and dweights (n, k) float32, 0 for ids without a group. out: where dR
    is written. (Without weights dR is ``dispatch`` of grad.)"""
    return _call_native("combine_backward", stream, grad, R, place, weights, out)
