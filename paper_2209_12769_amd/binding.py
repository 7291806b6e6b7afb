"""ctypes binding of libdisco.so -- argument marshalling only.

The module-level functions carry the names of the C ABI (include/disco.h) and
pass raw pointers; every step of the evaluation runs in the HIP kernels.
PyTorch is used for device memory and streams only.  There is no fallback: if
the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import itertools
import operator
import os
import struct
from dataclasses import dataclass
from typing import Dict, Optional, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdisco.so")

DC_OK = 0
DC_ERR_INVALID_ARG = 1
DC_ERR_BAD_GRAPH = 2
DC_ERR_BAD_PARTITION = 3
DC_ERR_CAPACITY = 4
DC_ERR_OOM = 5
DC_ERR_HIP = 6
DC_ERR_UNSUPPORTED = 7
DC_F32 = 0
DC_BF16 = 1
DC_AGG_MEAN = 0
DC_AGG_ATTENTION = 1
DC_KERNELS_SEPARATE_LAYERS = 1
DC_KERNELS_EVERY_FUSED_OP = 2
DC_DRAW_DEPENDENCY, DC_DRAW_OP = 0, 1
DC_KEEP_F32, DC_KEEP_8BIT = 0, 1
DC_DZ_WHOLE, DC_DZ_ROUNDED = 0, 1
DC_MOMENTS_F32, DC_MOMENTS_8BIT = 0, 1
DC_ACT_NONE, DC_ACT_RELU, DC_ACT_GELU, DC_ACT_SILU = 0, 1, 2, 3
ACTIVATIONS = {"none": DC_ACT_NONE, "relu": DC_ACT_RELU, "gelu": DC_ACT_GELU, "silu": DC_ACT_SILU}
STATUS_NAMES = {0: "DC_OK", 1: "DC_ERR_INVALID_ARG", 2: "DC_ERR_BAD_GRAPH", 3: "DC_ERR_BAD_PARTITION",
                4: "DC_ERR_CAPACITY", 5: "DC_ERR_OOM", 6: "DC_ERR_HIP", 7: "DC_ERR_UNSUPPORTED"}


class DcConfig(C.Structure):
    _fields_ = [("F", C.c_int32), ("H", C.c_int32), ("L", C.c_int32), ("dtype", C.c_int32),
                ("max_cand", C.c_int64), ("max_base_nodes", C.c_int64), ("max_base_edges", C.c_int64),
                ("max_nodes", C.c_int64), ("max_edges", C.c_int64),
                ("aggregator", C.c_int32), ("heads", C.c_int32)]


class DcBatch(C.Structure):
    _fields_ = [("n_cand", C.c_int32), ("cap_nodes", C.c_int64), ("cap_edges", C.c_int64),
                ("node_off", C.c_void_p), ("edge_off", C.c_void_p), ("new_id", C.c_void_p),
                ("out_rowptr", C.c_void_p), ("out_col", C.c_void_p), ("in_rowptr", C.c_void_p),
                ("in_col", C.c_void_p), ("Xc", C.c_void_p)]


class DcSearchParams(C.Structure):
    _fields_ = [("alpha", C.c_float), ("beta", C.c_int32), ("max_unchanged", C.c_int32), ("parents", C.c_int32),
                ("max_queue", C.c_int32), ("max_steps", C.c_int64), ("seed", C.c_uint64),
                ("ar_c", C.c_float), ("ar_d", C.c_float), ("op_draw", C.c_int32)]


class DcSearchResult(C.Structure):
    _fields_ = [("cost_in", C.c_float), ("cost_opt", C.c_float), ("steps", C.c_int64), ("evaluated", C.c_int64),
                ("valid", C.c_int64), ("enqueued", C.c_int64), ("improved", C.c_int64), ("queued", C.c_int64),
                ("unchanged", C.c_int64)]


class DcTrainParams(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("floor", C.c_float), ("max_samples", C.c_int64), ("max_rows", C.c_int64)]


class DcKeptRows(C.Structure):
    _fields_ = [("code", C.c_void_p), ("exponent", C.c_void_p), ("ld_code", C.c_int64), ("ld_exponent", C.c_int64)]


class DcDenseArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("rows", C.c_int64), ("n_in", C.c_int32), ("n_out", C.c_int32),
                ("X", C.c_void_p), ("ldx", C.c_int64), ("W", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p),
                ("residual", C.c_void_p), ("ld_residual", C.c_int64), ("Z", C.c_void_p), ("ldz", C.c_int64),
                ("Y", C.c_void_p), ("ldy", C.c_int64)]


class DcDenseBackwardArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("rows", C.c_int64), ("n_in", C.c_int32), ("n_out", C.c_int32),
                ("dY", C.c_void_p), ("lddy", C.c_int64), ("Z", C.c_void_p), ("ldz", C.c_int64), ("X", C.c_void_p),
                ("ldx", C.c_int64), ("kept", C.POINTER(DcKeptRows)), ("W", C.c_void_p), ("ldw", C.c_int64),
                ("dX", C.c_void_p), ("lddx", C.c_int64), ("dW", C.c_void_p), ("lddw", C.c_int64), ("db", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("dz", C.c_int32)]


class DcGraphNormArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("rows", C.c_int64), ("n_graphs", C.c_int32),
                ("channels", C.c_int32), ("groups", C.c_int32), ("eps", C.c_float), ("node_off", C.c_void_p),
                ("X", C.c_void_p), ("ldx", C.c_int64), ("gamma", C.c_void_p), ("beta", C.c_void_p), ("mean", C.c_void_p),
                ("rstd", C.c_void_p), ("Y", C.c_void_p), ("ldy", C.c_int64), ("kept", C.POINTER(DcKeptRows)),
                ("dY", C.c_void_p), ("lddy", C.c_int64), ("dres", C.c_void_p), ("lddres", C.c_int64), ("dX", C.c_void_p),
                ("lddx", C.c_int64), ("dgamma", C.c_void_p), ("dbeta", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t)]


class DcRowNormArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("act", C.c_int32), ("rows", C.c_int64), ("channels", C.c_int32), ("eps", C.c_float),
                ("X", C.c_void_p), ("ldx", C.c_int64), ("gamma", C.c_void_p), ("beta", C.c_void_p), ("mean", C.c_void_p),
                ("rstd", C.c_void_p), ("Y", C.c_void_p), ("ldy", C.c_int64), ("kept", C.POINTER(DcKeptRows)),
                ("dY", C.c_void_p), ("lddy", C.c_int64), ("dres", C.c_void_p), ("lddres", C.c_int64), ("dX", C.c_void_p),
                ("lddx", C.c_int64), ("dgamma", C.c_void_p), ("dbeta", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t)]


class DcEmbedRowsArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("rows", C.c_int64), ("kinds", C.c_int32), ("channels", C.c_int32), ("scale", C.c_float),
                ("id", C.c_void_p), ("table", C.c_void_p), ("ld_table", C.c_int64), ("Y", C.c_void_p), ("ldy", C.c_int64),
                ("dY", C.c_void_p), ("lddy", C.c_int64), ("dtable", C.c_void_p), ("ld_dtable", C.c_int64),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class DcAdamwTensor(C.Structure):
    _fields_ = [("p", C.c_void_p), ("g", C.c_void_p), ("n", C.c_int64), ("at", C.c_int64), ("p_dtype", C.c_int32),
                ("g_dtype", C.c_int32), ("weight_decay", C.c_double)]


class DcAdamwArgs(C.Structure):
    _fields_ = [("moments", C.c_int32), ("n_tensors", C.c_int32), ("tensors", C.c_void_p), ("total", C.c_int64),
                ("m", C.c_void_p), ("v", C.c_void_p), ("m_exponent", C.c_void_p), ("v_exponent", C.c_void_p),
                ("low", C.c_void_p), ("steps", C.c_void_p), ("grad_scale", C.c_void_p), ("lr", C.c_double),
                ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("seed", C.c_uint64)]


# The same structs for the wrapper's calls, packed from values (native sizes and alignment).
_KEPT = struct.Struct("@PPqq")
_DENSE = struct.Struct("@iiqiiPqPqPPqPqPq")
_DENSE_BACK = struct.Struct("@iiqiiPqPqPqPPqPqPqPPNi0q")
_NORM = struct.Struct("@iiqiiifPPqPPPPPqPPqPqPqPPPN")
_ROW_NORM = struct.Struct("@iiqifPqPPPPPqPPqPqPqPPPN")
_EMBED = struct.Struct("@iqiifPPqPqPqPqPN")
_ADAMW = struct.Struct("@iiPqPPPPPPPddddQ")
_ADAMW_TENSOR = np.dtype([("p", np.uint64), ("g", np.uint64), ("n", np.int64), ("at", np.int64), ("p_dtype", np.int32),
                          ("g_dtype", np.int32), ("weight_decay", np.float64)])
assert [s.size for s in (_KEPT, _DENSE, _DENSE_BACK, _NORM, _ROW_NORM, _EMBED, _ADAMW)] == [
    C.sizeof(s) for s in (DcKeptRows, DcDenseArgs, DcDenseBackwardArgs, DcGraphNormArgs, DcRowNormArgs, DcEmbedRowsArgs, DcAdamwArgs)]
assert _ADAMW_TENSOR.itemsize == C.sizeof(DcAdamwTensor)


class DiscoError(RuntimeError):
    def __init__(self, status: int, detail: str = ""):
        self.status = status
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {detail}")


_lib = None


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -m paper_2209_12769_amd.build)")
        # torch first: the process must hold one HIP runtime, the one that owns the tensors whose pointers
        # cross this boundary; loaded afterwards, libdisco.so binds to it instead of bringing a second copy
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        vp, i32, fp = C.c_void_p, C.c_int32, C.POINTER(C.c_float)
        L.dc_create.argtypes = [C.POINTER(vp), C.POINTER(DcConfig)]
        L.dc_destroy.argtypes = [vp]
        L.dc_workspace_bytes.argtypes = [C.POINTER(DcConfig)]
        L.dc_workspace_bytes.restype = C.c_size_t
        L.dc_set_weights.argtypes = [vp, vp, vp, vp, vp]
        L.dc_set_attention_weights.argtypes = [vp, vp, vp, vp, vp, vp]
        L.dc_set_base_graphs.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp]
        L.dc_contract_graphs.argtypes = [vp, i32, vp, vp, vp, C.POINTER(DcBatch), vp]
        L.dc_gnn_forward.argtypes = [vp, C.POINTER(DcBatch), vp, vp]
        L.dc_eval_candidates.argtypes = [vp, i32, vp, vp, vp, vp, vp]
        L.dc_simulate.argtypes = [vp, C.POINTER(DcBatch), vp, vp, C.c_float, C.c_float, vp, vp]
        L.dc_simulate_static.argtypes = [C.POINTER(DcBatch), i32, i32, vp, vp, C.c_float, C.c_float, vp, vp, vp]
        L.dc_simulate_static.restype = i32
        L.dc_simulate_static_error.argtypes = []
        L.dc_simulate_static_error.restype = C.c_char_p
        L.dc_set_profile.argtypes = [vp, vp, vp, vp]
        L.dc_module_times.argtypes = [vp, i32, vp, vp, vp, C.POINTER(DcBatch), vp, vp, vp]
        L.dc_cost_candidates.argtypes = [vp, i32, vp, vp, vp, C.c_float, C.c_float, vp, vp]
        L.dc_last_fused_ops.argtypes = [vp, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.POINTER(C.c_int64), vp]
        L.dc_last_fused_op_repeats.argtypes = [vp, C.POINTER(C.c_int64), vp]
        L.dc_walked_modules.argtypes = [vp, C.POINTER(C.c_int64), vp]
        L.dc_search.argtypes = [vp, i32, C.POINTER(DcSearchParams), vp, C.POINTER(DcSearchResult), vp]
        L.dc_num_params.argtypes = [vp]
        L.dc_num_params.restype = C.c_int64
        L.dc_train_begin.argtypes = [vp, C.POINTER(DcTrainParams), vp]
        L.dc_fused_op_batch.argtypes = [vp, i32, vp, vp, vp, C.POINTER(DcBatch), vp]
        L.dc_loss_gradients.argtypes = [vp, C.POINTER(DcBatch), vp, vp, vp, vp, vp]
        L.dc_train_step.argtypes = [vp, C.POINTER(DcBatch), vp, vp, vp]
        L.dc_get_weights.argtypes = [vp, vp, vp, vp, vp]
        i64, size = C.c_int64, C.c_size_t
        L.dc_set_layer_norms.argtypes = [vp, i32, i32, C.c_float, vp, vp, vp]
        L.dc_get_layer_norms.argtypes = [vp, vp, vp, vp]
        L.dc_train_keep.argtypes = [vp, i32]
        # argument structs as void pointers: a struct by reference, or the bytes of one
        L.dc_keep_rows.argtypes = [vp, i32, i64, i32, vp, i64, vp, vp]
        L.dc_restore_rows.argtypes = [vp, i32, i64, i32, vp, vp, i64, vp]
        L.dc_dense.argtypes = [vp, vp, vp]
        L.dc_dense_backward_bytes.argtypes = [vp, i32, i32, i64, i32, i32]
        L.dc_dense_backward_bytes.restype = size
        L.dc_dense_backward.argtypes = [vp, vp, vp]
        L.dc_graph_norm_bytes.argtypes = [vp, i64, i32, i32, i32, i32]
        L.dc_graph_norm_bytes.restype = size
        L.dc_graph_norm.argtypes = [vp, vp, vp]
        L.dc_graph_norm_backward.argtypes = [vp, vp, vp]
        L.dc_row_norm_bytes.argtypes = [vp, i64, i32]
        L.dc_row_norm_bytes.restype = size
        L.dc_row_norm.argtypes = [vp, vp, vp]
        L.dc_row_norm_backward.argtypes = [vp, vp, vp]
        L.dc_embed_rows_bytes.argtypes = [vp, i64, i32, i32]
        L.dc_embed_rows_bytes.restype = size
        L.dc_embed_rows.argtypes = [vp, vp, vp]
        L.dc_embed_rows_backward.argtypes = [vp, vp, vp]
        L.dc_adamw.argtypes = [vp, vp, vp]
        L.dc_adamw_values.argtypes = [vp, vp, vp, vp, vp, vp]
        L.dc_check.argtypes = [vp, vp]
        L.dc_select_kernels.argtypes = [vp, i32]
        L.dc_last_totals.argtypes = [vp, C.POINTER(C.c_int64), C.POINTER(C.c_int64), vp]
        L.dc_last_error.argtypes = [vp]
        L.dc_last_error.restype = C.c_char_p
        L.dc_profile_begin.argtypes = [vp]
        L.dc_profile_end.argtypes = [vp, C.POINTER(C.c_char_p), fp, C.POINTER(i32), i32]
        for n in ("dc_create", "dc_destroy", "dc_set_weights", "dc_set_attention_weights", "dc_set_base_graphs", "dc_contract_graphs",
                  "dc_gnn_forward", "dc_eval_candidates", "dc_simulate", "dc_check", "dc_last_totals", "dc_profile_begin",
                  "dc_profile_end", "dc_set_profile", "dc_module_times", "dc_cost_candidates", "dc_last_fused_ops",
                  "dc_last_fused_op_repeats", "dc_walked_modules", "dc_search",
                  "dc_train_begin", "dc_select_kernels", "dc_fused_op_batch", "dc_loss_gradients", "dc_train_step", "dc_get_weights",
                  "dc_set_layer_norms", "dc_get_layer_norms", "dc_train_keep", "dc_keep_rows", "dc_restore_rows", "dc_dense", "dc_dense_backward", "dc_graph_norm", "dc_graph_norm_backward",
                  "dc_row_norm", "dc_row_norm_backward", "dc_embed_rows", "dc_embed_rows_backward", "dc_adamw", "dc_adamw_values"):
            getattr(L, n).restype = i32
        _lib = L
    return _lib


# ---- the C ABI, name for name -------------------------------------------------
def dc_workspace_bytes(cfg: DcConfig) -> int:
    return int(lib().dc_workspace_bytes(C.byref(cfg)))


def dc_create(cfg: DcConfig) -> Tuple[int, Optional[int]]:
    h = C.c_void_p()
    st = lib().dc_create(C.byref(h), C.byref(cfg))
    return st, h.value


def dc_destroy(ctx: int) -> int:
    return lib().dc_destroy(ctx)


def dc_set_weights(ctx, W_layers: np.ndarray, b_layers: np.ndarray, head: np.ndarray, stream: int = 0) -> int:
    return lib().dc_set_weights(ctx, W_layers.ctypes.data, b_layers.ctypes.data, head.ctypes.data, stream)


def dc_set_attention_weights(ctx, W_layers: np.ndarray, att: np.ndarray, b_layers: np.ndarray, head: np.ndarray,
                             stream: int = 0) -> int:
    return lib().dc_set_attention_weights(ctx, W_layers.ctypes.data, att.ctypes.data, b_layers.ctypes.data,
                                          head.ctypes.data, stream)


def dc_set_base_graphs(ctx, n_graphs, g_node_off, g_edge_off, rowptr, col, X, stream: int = 0) -> int:
    return lib().dc_set_base_graphs(ctx, n_graphs, g_node_off.ctypes.data, g_edge_off.ctypes.data,
                                    rowptr.ctypes.data, col.ctypes.data if col.size else None, X.ctypes.data, stream)


def dc_contract_graphs(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, batch: DcBatch, stream: int = 0) -> int:
    return lib().dc_contract_graphs(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, C.byref(batch), stream)


def dc_gnn_forward(ctx, batch: DcBatch, pred_ptr, stream: int = 0) -> int:
    return lib().dc_gnn_forward(ctx, C.byref(batch), pred_ptr, stream)


def dc_eval_candidates(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, pred_ptr, stream: int = 0) -> int:
    return lib().dc_eval_candidates(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, pred_ptr, stream)


def dc_simulate(ctx, batch: DcBatch, op_time_ptr, ar_size_ptr, ar_c: float, ar_d: float, cost_ptr,
                stream: int = 0) -> int:
    return lib().dc_simulate(ctx, C.byref(batch), op_time_ptr, ar_size_ptr, ar_c, ar_d, cost_ptr, stream)


def dc_set_profile(ctx, op_time: np.ndarray, ar_size: np.ndarray, stream: int = 0) -> int:
    return lib().dc_set_profile(ctx, op_time.ctypes.data, ar_size.ctypes.data, stream)


def dc_module_times(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, batch: DcBatch, op_time_ptr, ar_size_ptr,
                    stream: int = 0) -> int:
    return lib().dc_module_times(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, C.byref(batch), op_time_ptr,
                                 ar_size_ptr, stream)


def dc_cost_candidates(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, ar_c: float, ar_d: float, cost_ptr,
                       stream: int = 0) -> int:
    return lib().dc_cost_candidates(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, ar_c, ar_d, cost_ptr,
                                    stream)


def dc_last_fused_ops(ctx, stream: int = 0) -> Tuple[int, int, int, int]:
    k, m, e = C.c_int64(), C.c_int64(), C.c_int64()
    st = lib().dc_last_fused_ops(ctx, C.byref(k), C.byref(m), C.byref(e), stream)
    return st, k.value, m.value, e.value


def dc_last_fused_op_repeats(ctx, stream: int = 0) -> Tuple[int, int]:
    n = C.c_int64()
    st = lib().dc_last_fused_op_repeats(ctx, C.byref(n), stream)
    return st, n.value


def dc_walked_modules(ctx, stream: int = 0) -> Tuple[int, int]:
    n = C.c_int64()
    st = lib().dc_walked_modules(ctx, C.byref(n), stream)
    return st, n.value


def dc_search(ctx, graph: int, params: DcSearchParams, labels_opt: Optional[np.ndarray], res: DcSearchResult,
              stream: int = 0) -> int:
    return lib().dc_search(ctx, graph, C.byref(params), None if labels_opt is None else labels_opt.ctypes.data,
                           C.byref(res), stream)


def dc_num_params(ctx) -> int:
    return int(lib().dc_num_params(ctx))


def dc_train_begin(ctx, params: DcTrainParams, stream: int = 0) -> int:
    return lib().dc_train_begin(ctx, C.byref(params), stream)


def dc_fused_op_batch(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, batch: DcBatch, stream: int = 0) -> int:
    return lib().dc_fused_op_batch(ctx, n_cand, cand_graph_ptr, cand_off_ptr, group_id_ptr, C.byref(batch), stream)


def dc_loss_gradients(ctx, batch: DcBatch, target_ptr, loss_ptr, pred_ptr, grad_ptr, stream: int = 0) -> int:
    return lib().dc_loss_gradients(ctx, C.byref(batch), target_ptr, loss_ptr, pred_ptr, grad_ptr, stream)


def dc_train_step(ctx, batch: DcBatch, target_ptr, loss_ptr, stream: int = 0) -> int:
    return lib().dc_train_step(ctx, C.byref(batch), target_ptr, loss_ptr, stream)


def dc_get_weights(ctx, W_layers: np.ndarray, b_layers: np.ndarray, head: np.ndarray, stream: int = 0) -> int:
    return lib().dc_get_weights(ctx, W_layers.ctypes.data, b_layers.ctypes.data, head.ctypes.data, stream)


def dc_set_layer_norms(ctx, groups: int, act: int, eps: float, gamma: Optional[np.ndarray], beta: Optional[np.ndarray],
                       stream: int = 0) -> int:
    return lib().dc_set_layer_norms(ctx, groups, act, eps, None if gamma is None else gamma.ctypes.data,
                                    None if beta is None else beta.ctypes.data, stream)


def dc_get_layer_norms(ctx, gamma: np.ndarray, beta: np.ndarray, stream: int = 0) -> int:
    return lib().dc_get_layer_norms(ctx, gamma.ctypes.data, beta.ctypes.data, stream)


def dc_train_keep(ctx, which: int) -> int:
    return lib().dc_train_keep(ctx, which)


def dc_keep_rows(ctx, dtype: int, rows: int, cols: int, x_ptr, ldx: int, out: DcKeptRows, stream: int = 0) -> int:
    return lib().dc_keep_rows(ctx, dtype, rows, cols, x_ptr, ldx, C.byref(out), stream)


def dc_restore_rows(ctx, dtype: int, rows: int, cols: int, kept: DcKeptRows, x_ptr, ldx: int, stream: int = 0) -> int:
    return lib().dc_restore_rows(ctx, dtype, rows, cols, C.byref(kept), x_ptr, ldx, stream)


def dc_dense(ctx, args: DcDenseArgs, stream: int = 0) -> int:
    return lib().dc_dense(ctx, C.byref(args), stream)


def dc_dense_backward_bytes(ctx, dtype: int, act: int, rows: int, n_in: int, n_out: int) -> int:
    return int(lib().dc_dense_backward_bytes(ctx, dtype, act, rows, n_in, n_out))


def dc_dense_backward(ctx, args: DcDenseBackwardArgs, stream: int = 0) -> int:
    return lib().dc_dense_backward(ctx, C.byref(args), stream)


def dc_graph_norm_bytes(ctx, rows: int, n_graphs: int, channels: int, groups: int, backward: bool) -> int:
    return int(lib().dc_graph_norm_bytes(ctx, rows, n_graphs, channels, groups, int(backward)))


def dc_graph_norm(ctx, args: DcGraphNormArgs, stream: int = 0) -> int:
    return lib().dc_graph_norm(ctx, C.byref(args), stream)


def dc_graph_norm_backward(ctx, args: DcGraphNormArgs, stream: int = 0) -> int:
    return lib().dc_graph_norm_backward(ctx, C.byref(args), stream)


def dc_row_norm_bytes(ctx, rows: int, channels: int) -> int:
    return int(lib().dc_row_norm_bytes(ctx, rows, channels))


def dc_row_norm(ctx, args: DcRowNormArgs, stream: int = 0) -> int:
    return lib().dc_row_norm(ctx, C.byref(args), stream)


def dc_row_norm_backward(ctx, args: DcRowNormArgs, stream: int = 0) -> int:
    return lib().dc_row_norm_backward(ctx, C.byref(args), stream)


def dc_embed_rows_bytes(ctx, rows: int, kinds: int, channels: int) -> int:
    return int(lib().dc_embed_rows_bytes(ctx, rows, kinds, channels))


def dc_embed_rows(ctx, args: DcEmbedRowsArgs, stream: int = 0) -> int:
    return lib().dc_embed_rows(ctx, C.byref(args), stream)


def dc_embed_rows_backward(ctx, args: DcEmbedRowsArgs, stream: int = 0) -> int:
    return lib().dc_embed_rows_backward(ctx, C.byref(args), stream)


def dc_adamw(ctx, args: DcAdamwArgs, stream: int = 0) -> int:
    return lib().dc_adamw(ctx, C.byref(args), stream)


def dc_adamw_values(ctx, args: DcAdamwArgs, w_ptr, m_ptr, v_ptr, stream: int = 0) -> int:
    return lib().dc_adamw_values(ctx, C.byref(args), w_ptr, m_ptr, v_ptr, stream)


def dc_check(ctx, stream: int = 0) -> int:
    return lib().dc_check(ctx, stream)


def dc_simulate_static(batch: DcBatch, max_module_nodes: int, max_module_edges: int, op_time_ptr, ar_size_ptr,
                       ar_c: float, ar_d: float, cost_ptr, dev_status_ptr, stream: int = 0) -> int:
    return lib().dc_simulate_static(C.byref(batch), max_module_nodes, max_module_edges, op_time_ptr, ar_size_ptr,
                                    ar_c, ar_d, cost_ptr, dev_status_ptr, stream)


def dc_simulate_static_error() -> str:
    return lib().dc_simulate_static_error().decode()


def dc_select_kernels(ctx, which: int) -> int:
    return lib().dc_select_kernels(ctx, which)


def dc_last_totals(ctx, stream: int = 0) -> Tuple[int, int, int]:
    n, e = C.c_int64(), C.c_int64()
    st = lib().dc_last_totals(ctx, C.byref(n), C.byref(e), stream)
    return st, n.value, e.value


def dc_last_error(ctx) -> str:
    return lib().dc_last_error(ctx).decode()


def dc_profile_begin(ctx) -> int:
    return lib().dc_profile_begin(ctx)


def dc_profile_end(ctx) -> Dict[str, Tuple[float, int]]:
    cap = 32
    names = (C.c_char_p * cap)()
    ms = (C.c_float * cap)()
    cnt = (C.c_int32 * cap)()
    n = lib().dc_profile_end(ctx, names, ms, cnt, cap)
    return {names[i].decode(): (float(ms[i]), int(cnt[i])) for i in range(min(n, cap))}


# ---- convenience wrapper over torch device memory --------------------------------
@dataclass
class DeviceBatch:
    """Device arrays of one dc_batch (torch tensors own the memory)."""
    c: DcBatch
    node_off: "object"
    edge_off: "object"
    new_id: "object"
    out_rowptr: "object"
    out_col: "object"
    in_rowptr: "object"
    in_col: "object"
    Xc: "object"


class KeptRows:
    """Rows kept in 8 bits (see dc_kept_rows): int8 codes and uint8 exponents, device tensors."""

    def __init__(self, code, exponent, cols: int):
        blocks = -(-cols // 32)
        if code.dim() != 2 or exponent.dim() != 2 or code.shape[1] < 32 * blocks or tuple(exponent.shape) != (code.shape[0], blocks):
            raise ValueError(f"kept rows of {cols} columns need codes [rows, {32 * blocks}] and exponents [rows, {blocks}]")
        self.code, self.exponent, self.cols = code, exponent, cols

    @property
    def c(self) -> DcKeptRows:
        code, exponent = self.code, self.exponent
        apart = self.rows > 1                              # of a single row any distance may be written down
        return DcKeptRows(code.data_ptr(), exponent.data_ptr(), code.stride(0) if apart else code.shape[1],
                          exponent.stride(0) if apart else exponent.shape[1])

    @property
    def rows(self) -> int:
        return int(self.code.shape[0])


class AdamW:
    """AdamW over many tensors in one call (see dc_adamw), made by Evaluator.adamw.

    The state, device tensors of `total` places: m, v (float32, or uint8 codes with m_exponent and v_exponent for each 128
    places), low (int16: the low halves of bfloat16 parameters), steps (int32: steps done, 0).  Tensor k has the places
    at[k] .. at[k] + its elements.  Saved, and copied back into them (copy_), they go on where they were.  lr, betas, eps and seed
    may be changed between steps.  A parameter may be given other memory (data) of its shape and type, contiguous as it was.  A
    bfloat16 parameter that is written anew keeps its low halves, up to half a rounding of it, until they are cleared
    (low[at[k]:at[k] + p.numel()] = 0)."""

    _PARTS = ("m", "v", "m_exponent", "v_exponent", "low", "steps")
    _FIXED = frozenset(_PARTS + ("params", "at", "total", "states"))

    def __setattr__(self, name, value):
        if name in self._FIXED and name in self.__dict__:              # the calls go by where they lie
            raise AttributeError(f"{name} is kept where it is: copy_ into it")
        object.__setattr__(self, name, value)

    def __init__(self, ev: "Evaluator", params, lr: float, betas, eps: float, weight_decay, states: str, seed: int):
        torch = ev.torch
        if states not in ("f32", "8bit"):
            raise ValueError(f"states: 'f32' or '8bit', not {states!r}")
        self.ev, self.params, self.states = ev, list(params), states
        self.lr, self.betas, self.eps, self.seed = lr, tuple(betas), eps, seed
        decay = list(weight_decay) if hasattr(weight_decay, "__len__") else [weight_decay] * len(self.params)
        if len(decay) != len(self.params):
            raise ValueError("weight_decay: need a number, or one for every tensor")
        self._table = np.zeros(len(self.params), _ADAMW_TENSOR)
        self.at, total, half = [], 0, False
        for k, p in enumerate(self.params):
            self._check(k, p)
            n = p.numel()
            self._table[k] = (p.data_ptr(), 0, n, total, ev._types[p.dtype], 0, decay[k])
            self.at.append(total)
            total += -(-n // 128) * 128
            half = half or (p.dtype == torch.bfloat16 and n > 0)
        self.total = total
        self._shapes, self._dtypes = [p.shape for p in self.params], [p.dtype for p in self.params]
        # what the table holds of the tensors' places and the gradients' types, as lists; `_held` keeps that memory theirs, so that a
        # place that is still the same is the same tensor's
        self._ptrs, self._g_dtypes = [p.data_ptr() for p in self.params], None
        self._held = [p.detach() for p in self.params]
        eight = states == "8bit"
        with torch.no_grad():
            self.m, self.v = (torch.zeros(total, dtype=torch.uint8 if eight else torch.float32, device=ev.device) for _ in range(2))
            self.m_exponent, self.v_exponent = (torch.zeros(total // 128, dtype=torch.uint8, device=ev.device) if eight else None for _ in range(2))
            self.low = torch.zeros(total, dtype=torch.int16, device=ev.device) if half else None
            self.steps = torch.zeros(2, dtype=torch.int32, device=ev.device)
        # the state and where it lies; that memory is kept too
        self._state = {name: getattr(self, name) for name in self._PARTS if getattr(self, name) is not None}
        self._state_ptrs = list(map(torch.Tensor.data_ptr, self._state.values()))
        at = dict(zip(self._state, self._state_ptrs))
        self._where = (total, *(at.get(name, 0) for name in self._PARTS))
        self._held_state = [t.detach() for t in self._state.values()]

    def _check(self, k: int, p):
        if p.device != self.ev.device or p.dtype not in self.ev._types or not p.is_contiguous():
            raise ValueError(f"tensor {k}: need contiguous float32 or bfloat16 on {self.ev.device}")

    def _args(self, grad_scale: int) -> bytes:
        T = self.ev.torch.Tensor
        if list(map(T.data_ptr, self._state.values())) != self._state_ptrs:
            moved = [name for name, was in zip(self._state, self._state_ptrs) if self._state[name].data_ptr() != was]
            raise ValueError(f"{', '.join(moved)}: given other memory; copy_ into the state")
        ptrs = list(map(T.data_ptr, self.params))
        # tensors whose owner gave them other memory, or let the same memory stand in another order, type or shape
        if (ptrs != self._ptrs or list(map(T.dtype.__get__, self.params)) != self._dtypes
                or list(map(T.shape.__get__, self.params)) != self._shapes or not all(map(T.is_contiguous, self.params))):
            if len(ptrs) != len(self._shapes):
                raise ValueError(f"params: made of {len(self._shapes)} tensors, not {len(ptrs)}")
            for k, p in enumerate(self.params):
                self._check(k, p)
                if p.shape != self._shapes[k] or p.dtype != self._dtypes[k]:
                    raise ValueError(f"tensor {k}: was {tuple(self._shapes[k])} {self._dtypes[k]}, not {tuple(p.shape)} {p.dtype}")
            self._table["p"] = self._ptrs = ptrs
            self._held = [p.detach() for p in self.params]
        return _ADAMW.pack(DC_MOMENTS_F32 if self.m_exponent is None else DC_MOMENTS_8BIT, len(ptrs), self._table.ctypes.data, *self._where,
                           grad_scale, self.lr, self.betas[0], self.betas[1], self.eps, self.seed)

    def step(self, grads, grad_scale=None):
        """One step with a gradient for every tensor (float32 or bfloat16, contiguous, its shape), None for tensors that stay as
        they are.  grad_scale: a float32 device tensor of one number that the gradients are multiplied by.  `steps` counts for
        all tensors: the corrections of one that had no gradient go on.  Captured in a graph, a step counts on when it is replayed and keeps
        lr, betas, eps and seed of its capture.  A gradient that is not finite stays in the moments for good."""
        ev, T = self.ev, self.ev.torch.Tensor
        if len(grads) != len(self._shapes):
            raise ValueError(f"need {len(self._shapes)} gradients, not {len(grads)}")
        which, have, shapes = slice(None), grads, self._shapes
        if any(map(operator.is_, grads, itertools.repeat(None))):
            which = [k for k, g in enumerate(grads) if g is not None]
            have, shapes = [grads[k] for k in which], [shapes[k] for k in which]
            self._table["g"] = 0
        # A small step is bound by what happens here and in _args: one look at all of them after the other takes a quarter less than
        # all at one (28 parameters: 19.7 us, 4.5 of them for what _args looks at besides addresses).
        dtypes = list(map(T.dtype.__get__, have))
        if (not ev._types.keys() >= set(dtypes) or list(map(T.shape.__get__, have)) != shapes
                or list(map(T.get_device, have)).count(ev.device.index) != len(have)
                or not all(map(T.is_contiguous, have))):
            for k, (g, shape) in enumerate(zip(grads, self._shapes)):
                if g is not None and (g.dtype not in ev._types or g.shape != shape or g.device != ev.device or not g.is_contiguous()):
                    raise ValueError(f"gradient {k}: need contiguous float32 or bfloat16 {tuple(shape)} on {ev.device}")
        self._table["g"][which] = list(map(T.data_ptr, have))
        if dtypes != self._g_dtypes or have is not grads:
            self._table["g_dtype"][which] = [ev._types[t] for t in dtypes]
            self._g_dtypes = dtypes if have is grads else None
        st = lib().dc_adamw(ev.ctx, self._args(0 if grad_scale is None else ev._vector(grad_scale.reshape(-1), "grad_scale", 1)), ev._raw_stream())
        if st:
            ev._ok(st, "dc_adamw")

    def values(self, which: str = "wmv"):
        """The float32 values of the parameters (w) and moments (m, v) that `which` names, in its order, each a tensor of `total`
        places."""
        ev = self.ev
        if not which or set(which) - set("wmv") or len(set(which)) != len(which):
            raise ValueError(f"which: letters of 'wmv', each once, not {which!r}")
        out = {c: ev.torch.empty(self.total, dtype=ev.torch.float32, device=ev.device) for c in which}
        st = lib().dc_adamw_values(ev.ctx, self._args(0), *(out[c].data_ptr() if c in out else 0 for c in "wmv"), ev._raw_stream())
        if st:
            ev._ok(st, "dc_adamw_values")
        return tuple(out[c] for c in which)


class Evaluator:
    """Owns one dc_ctx.  Methods move pointers across the C ABI; nothing is computed in Python."""

    def __init__(self, F: int, H: int, L: int, dtype: str, max_cand: int, max_base_nodes: int, max_base_edges: int,
                 max_nodes: int = 0, max_edges: int = 0, device: str = "cuda:0", agg: str = "mean", heads: int = 1):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        if self.device.index is None:
            self.device = torch.device(self.device.type, torch.cuda.current_device())
        self.cfg = DcConfig(F, H, L, DC_BF16 if dtype == "bf16" else DC_F32, max_cand, max_base_nodes,
                            max_base_edges, max_nodes, max_edges,
                            DC_AGG_ATTENTION if agg == "attention" else DC_AGG_MEAN, heads)
        self.dtype = dtype
        self.agg = agg
        st, h = dc_create(self.cfg)
        if st != DC_OK:
            raise DiscoError(st, "dc_create")
        self.ctx = h

    def close(self):
        if getattr(self, "ctx", None):
            dc_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self) -> int:
        return int(self.torch.cuda.current_stream(self.device).cuda_stream)

    def _ok(self, st: int, what: str):
        if st != DC_OK:
            raise DiscoError(st, f"{what}: {dc_last_error(self.ctx)}")

    def set_weights(self, weights):
        W = np.ascontiguousarray(weights.layers, dtype=np.float32)
        b = np.ascontiguousarray(weights.biases, dtype=np.float32)
        hd = np.ascontiguousarray(weights.head, dtype=np.float32)
        if self.agg == "attention":
            at = np.ascontiguousarray(weights.att, dtype=np.float32)
            self._ok(dc_set_attention_weights(self.ctx, W, at, b, hd, self._stream()), "dc_set_attention_weights")
        else:
            self._ok(dc_set_weights(self.ctx, W, b, hd, self._stream()), "dc_set_weights")

    def set_base_graphs(self, g_node_off, g_edge_off, rowptr, col, X):
        gno = np.ascontiguousarray(g_node_off, dtype=np.int32)
        geo = np.ascontiguousarray(g_edge_off, dtype=np.int32)
        rp = np.ascontiguousarray(rowptr, dtype=np.int32)
        ci = np.ascontiguousarray(col, dtype=np.int32)
        Xf = np.ascontiguousarray(X, dtype=np.float32)
        self._ok(dc_set_base_graphs(self.ctx, len(gno) - 1, gno, geo, rp, ci, Xf, self._stream()), "dc_set_base_graphs")

    def to_device(self, a: np.ndarray):
        return self.torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(self.device)

    def alloc_batch(self, n_cand: int, n_labels: int, cap_nodes: int, cap_edges: int) -> DeviceBatch:
        t = self.torch
        i32 = dict(dtype=t.int32, device=self.device)
        node_off = t.empty(n_cand + 1, **i32)
        edge_off = t.empty(n_cand + 1, **i32)
        new_id = t.empty(max(n_labels, 1), **i32)
        orp = t.empty(cap_nodes + 1, **i32)
        irp = t.empty(cap_nodes + 1, **i32)
        oc = t.empty(max(cap_edges, 1), **i32)
        ic = t.empty(max(cap_edges, 1), **i32)
        Xc = t.empty((max(cap_nodes, 1), self.cfg.F), dtype=t.bfloat16 if self.dtype == "bf16" else t.float32,
                     device=self.device)
        c = DcBatch(n_cand, cap_nodes, cap_edges, node_off.data_ptr(), edge_off.data_ptr(), new_id.data_ptr(),
                    orp.data_ptr(), oc.data_ptr(), irp.data_ptr(), ic.data_ptr(), Xc.data_ptr())
        return DeviceBatch(c, node_off, edge_off, new_id, orp, oc, irp, ic, Xc)

    def contract_graphs(self, cand_graph, cand_off, group_id, batch: DeviceBatch) -> DeviceBatch:
        n_cand = int(cand_graph.numel())
        self._ok(dc_contract_graphs(self.ctx, n_cand, cand_graph.data_ptr(), cand_off.data_ptr(),
                                    group_id.data_ptr(), batch.c, self._stream()), "dc_contract_graphs")
        return batch

    def gnn_forward(self, batch: DeviceBatch, pred=None):
        if pred is None:
            pred = self.torch.empty(max(batch.c.n_cand, 1), dtype=self.torch.float32, device=self.device)
        self._ok(dc_gnn_forward(self.ctx, batch.c, pred.data_ptr(), self._stream()), "dc_gnn_forward")
        return pred[:batch.c.n_cand]

    def simulate(self, batch: DeviceBatch, op_time, ar_size, ar_c: float, ar_d: float, cost=None):
        if cost is None:
            cost = self.torch.empty(max(batch.c.n_cand, 1), dtype=self.torch.float32, device=self.device)
        self._ok(dc_simulate(self.ctx, batch.c, op_time.data_ptr(), ar_size.data_ptr(), ar_c, ar_d,
                             cost.data_ptr(), self._stream()), "dc_simulate")
        return cost[:batch.c.n_cand]

    def eval_candidates(self, cand_graph, cand_off, group_id, pred=None):
        n_cand = int(cand_graph.numel())
        if pred is None:
            pred = self.torch.empty(max(n_cand, 1), dtype=self.torch.float32, device=self.device)
        self._ok(dc_eval_candidates(self.ctx, n_cand, cand_graph.data_ptr(), cand_off.data_ptr(),
                                    group_id.data_ptr(), pred.data_ptr(), self._stream()), "dc_eval_candidates")
        return pred[:n_cand]

    def set_profile(self, op_time: np.ndarray, ar_size: np.ndarray):
        t = np.ascontiguousarray(op_time, dtype=np.float32)
        x = np.ascontiguousarray(ar_size, dtype=np.float32)
        self._ok(dc_set_profile(self.ctx, t, x, self._stream()), "dc_set_profile")

    def module_times(self, cand_graph, cand_off, group_id, batch: DeviceBatch, op_time=None, ar_size=None):
        n_cand = int(cand_graph.numel())
        f32 = dict(dtype=self.torch.float32, device=self.device)
        if op_time is None:
            op_time = self.torch.empty(max(batch.c.cap_nodes, 1), **f32)
        if ar_size is None:
            ar_size = self.torch.empty(max(batch.c.cap_nodes, 1), **f32)
        self._ok(dc_module_times(self.ctx, n_cand, cand_graph.data_ptr(), cand_off.data_ptr(), group_id.data_ptr(),
                                 batch.c, op_time.data_ptr(), ar_size.data_ptr(), self._stream()), "dc_module_times")
        return op_time, ar_size

    def cost_candidates(self, cand_graph, cand_off, group_id, ar_c: float, ar_d: float, cost=None):
        n_cand = int(cand_graph.numel())
        if cost is None:
            cost = self.torch.empty(max(n_cand, 1), dtype=self.torch.float32, device=self.device)
        self._ok(dc_cost_candidates(self.ctx, n_cand, cand_graph.data_ptr(), cand_off.data_ptr(), group_id.data_ptr(),
                                    ar_c, ar_d, cost.data_ptr(), self._stream()), "dc_cost_candidates")
        return cost[:n_cand]

    def search(self, graph: int, n_nodes: int, alpha: float, beta: int, seed: int, ar_c: float, ar_d: float,
               max_unchanged: int = 1000, parents: int = 1, max_steps: int = 1 << 40, max_queue: int = 4096,
               op_draw: int = 0):
        """Alg. 1 on base graph `graph`; returns (labels_opt, DcSearchResult)."""
        p = DcSearchParams(alpha, beta, max_unchanged, parents, max_queue, max_steps, seed, ar_c, ar_d, op_draw)
        r = DcSearchResult()
        labels = np.zeros(n_nodes, np.int32)
        self._ok(dc_search(self.ctx, graph, p, labels, r, self._stream()), "dc_search")
        return labels, r

    def set_layer_norms(self, groups: int, gamma=None, beta=None, act: str = "silu", eps: float = 1e-5):
        """Residual layers with a norm in front (see dc_set_layer_norms); groups = 0: ReLU layers again."""
        g = [None if v is None else np.ascontiguousarray(v, dtype=np.float32) for v in (gamma, beta)]
        for v in g:
            if v is not None and v.size != (self.cfg.L - 1) * self.cfg.H:
                raise ValueError("gamma and beta: need [L - 1, H]")
        self._ok(dc_set_layer_norms(self.ctx, groups, self._act(act), eps, g[0], g[1], self._stream()), "dc_set_layer_norms")

    def get_layer_norms(self):
        gamma = np.empty((self.cfg.L - 1, self.cfg.H), np.float32)
        beta = np.empty_like(gamma)
        self._ok(dc_get_layer_norms(self.ctx, gamma, beta, self._stream()), "dc_get_layer_norms")
        return gamma, beta

    # ---- training of the estimator ----
    def num_params(self) -> int:
        return dc_num_params(self.ctx)

    def train_begin(self, lr: float, max_samples: int, max_rows: int, beta1: float = 0.9, beta2: float = 0.999,
                    eps: float = 1e-8, floor: float = 1e-6, keep: str = "f32"):
        """keep: what a pass keeps of every layer's rows, "f32" or "8bit" (see dc_train_keep)."""
        if keep not in ("f32", "8bit"):
            raise ValueError(f"keep: 'f32' or '8bit', not {keep!r}")
        self._ok(dc_train_keep(self.ctx, DC_KEEP_8BIT if keep == "8bit" else DC_KEEP_F32), "dc_train_keep")
        p = DcTrainParams(lr, beta1, beta2, eps, floor, max_samples, max_rows)
        self._ok(dc_train_begin(self.ctx, p, self._stream()), "dc_train_begin")

    def fused_op_batch(self, cand_graph, cand_off, group_id, batch: DeviceBatch) -> DeviceBatch:
        n_cand = int(cand_graph.numel())
        self._ok(dc_fused_op_batch(self.ctx, n_cand, cand_graph.data_ptr(), cand_off.data_ptr(), group_id.data_ptr(),
                                   batch.c, self._stream()), "dc_fused_op_batch")
        return batch

    def loss_gradients(self, batch: DeviceBatch, target, want_grad: bool = True):
        """(loss [1], pred [n], grad [num_params] or None), device tensors."""
        f32 = dict(dtype=self.torch.float32, device=self.device)
        loss = self.torch.empty(1, **f32)
        pred = self.torch.empty(max(batch.c.n_cand, 1), **f32)
        grad = self.torch.empty(max(self.num_params(), 1), **f32) if want_grad else None
        self._ok(dc_loss_gradients(self.ctx, batch.c, target.data_ptr(), loss.data_ptr(), pred.data_ptr(),
                                   grad.data_ptr() if want_grad else None, self._stream()), "dc_loss_gradients")
        return loss, pred[:batch.c.n_cand], grad

    def train_step(self, batch: DeviceBatch, target, loss=None):
        if loss is None:
            loss = self.torch.empty(1, dtype=self.torch.float32, device=self.device)
        self._ok(dc_train_step(self.ctx, batch.c, target.data_ptr(), loss.data_ptr(), self._stream()), "dc_train_step")
        return loss

    # ---- operators on rows of a batch (device tensors; rows may be apart, columns are neighbours) ----
    # A small call is bound by what happens here: the argument structs are packed in one go, every tensor is looked at once.
    def _raw_stream(self) -> int:
        return self.torch._C._cuda_getCurrentRawStream(self.device.index)

    def _rows(self, x, name: str):
        """(rows, cols, elements from row to row, type) of a matrix on the context's device."""
        if x.device != self.device or x.dim() != 2:
            raise ValueError(f"{name}: need a matrix on {self.device}")
        dtype = self._types.get(x.dtype)
        if dtype is None:
            raise ValueError(f"{name}: need float32 or bfloat16, not {x.dtype}")
        rows, cols = x.shape
        ld, step = x.stride()
        if step != 1 and cols > 1 and rows:
            raise ValueError(f"{name}: the columns of a row must be neighbours")
        return rows, cols, ld if rows > 1 else cols, dtype

    def _like(self, x, name: str, rows: int, cols: int, dtype: int) -> int:
        """Elements from row to row of a matrix that has to be rows x cols of that type."""
        r, c, ld, t = self._rows(x, name)
        if r != rows or c != cols or t != dtype:
            raise ValueError(f"{name}: need {rows} x {cols} {'bfloat16' if dtype else 'float32'}, not {tuple(x.shape)} {x.dtype}")
        return ld

    def _vector(self, x, name: str, n: int, dtype=None) -> int:
        if x.device != self.device or x.dtype != (dtype or self.torch.float32) or tuple(x.shape) != (n,) or not x.is_contiguous():
            raise ValueError(f"{name}: need {n} contiguous {dtype or self.torch.float32} on {self.device}")
        return x.data_ptr()

    def _kept(self, k: KeptRows, rows: int, cols: int) -> bytes:
        """The packed dc_kept_rows."""
        c, e = k.code, k.exponent
        if (c.device != self.device or e.device != self.device or c.dtype != self.torch.int8 or e.dtype != self.torch.uint8
                or k.cols != cols or c.shape[0] != rows):
            raise ValueError(f"kept rows: need {rows} x {cols} on {self.device}")
        lc, le = c.stride(0), e.stride(0)
        if rows <= 1:
            lc, le = c.shape[1], e.shape[1]
        elif c.stride(1) != 1 or (e.shape[1] > 1 and e.stride(1) != 1):
            raise ValueError("kept rows: the columns of a row must be neighbours")
        return _KEPT.pack(c.data_ptr(), e.data_ptr(), lc, le)

    @staticmethod
    def _act(act: str) -> int:
        code = ACTIVATIONS.get(act)
        if code is None:
            raise ValueError(f"unknown activation {act!r}: one of {', '.join(ACTIVATIONS)}")
        return code

    @property
    def _types(self):
        types = self.__dict__.get("_type_codes")
        if types is None:
            types = self.__dict__["_type_codes"] = {self.torch.float32: DC_F32, self.torch.bfloat16: DC_BF16}
        return types

    def keep_rows(self, x) -> KeptRows:
        """x [rows, cols] in 8 bits, one power of two per row and 32 columns."""
        rows, cols, ld, dtype = self._rows(x, "x")
        blocks = -(-cols // 32)
        k = KeptRows.__new__(KeptRows)                   # of shapes that need no check
        k.code = self.torch.empty((rows, 32 * blocks), dtype=self.torch.int8, device=self.device)
        k.exponent = self.torch.empty((rows, blocks), dtype=self.torch.uint8, device=self.device)
        k.cols = cols
        st = lib().dc_keep_rows(self.ctx, dtype, rows, cols, x.data_ptr(), ld,
                                _KEPT.pack(k.code.data_ptr(), k.exponent.data_ptr(), 32 * blocks, blocks), self._raw_stream())
        if st:
            self._ok(st, "dc_keep_rows")
        return k

    def restore_rows(self, kept: KeptRows, dtype=None, out=None):
        rows, cols = kept.code.shape[0], kept.cols
        if out is None:
            out = self.torch.empty((rows, cols), dtype=dtype or self.torch.float32, device=self.device)
        elif dtype is not None and out.dtype != dtype:
            raise ValueError(f"out: need {dtype}, not {out.dtype}")
        r, c, ld, t = self._rows(out, "out")
        if r != rows or c != cols:
            raise ValueError(f"out: need {rows} x {cols}, not {tuple(out.shape)}")
        st = lib().dc_restore_rows(self.ctx, t, rows, cols, self._kept(kept, rows, cols), out.data_ptr(), ld, self._raw_stream())
        if st:
            self._ok(st, "dc_restore_rows")
        return out

    def dense(self, x, w, bias=None, act: str = "none", residual=None, out=None, want_pre: bool = False):
        """act(x w + bias) + residual; with want_pre also x w + bias, which dense_backward takes as `pre`."""
        rows, n_in, ldx, dtype = self._rows(x, "x")
        wr, n_out, ldw, wt = self._rows(w, "w")
        if wr != n_in or wt != dtype:
            raise ValueError(f"w: need {n_in} rows of x's type")
        if out is None:
            out, ldy = self.torch.empty((rows, n_out), dtype=x.dtype, device=self.device), n_out
        else:
            ldy = self._like(out, "out", rows, n_out, dtype)
        pb = self._vector(bias, "bias", n_out) if bias is not None else 0
        pr, ldr = (residual.data_ptr(), self._like(residual, "residual", rows, n_out, dtype)) if residual is not None else (0, 0)
        pre = self.torch.empty((rows, n_out), dtype=x.dtype, device=self.device) if want_pre else None
        a = _DENSE.pack(dtype, self._act(act), rows, n_in, n_out, x.data_ptr(), ldx, w.data_ptr(), ldw, pb, pr, ldr,
                        pre.data_ptr() if want_pre else 0, n_out, out.data_ptr(), ldy)
        st = lib().dc_dense(self.ctx, a, self._raw_stream())
        if st:
            self._ok(st, "dc_dense")
        return (out, pre) if want_pre else out

    def dense_backward(self, dy, x, w, act: str = "none", pre=None, want=("x", "w", "b"), round_dz: bool = False):
        """Gradients (dx, dw, db) of dense at x, w and bias for the gradient dy at its result; None for those not in
        `want`.  x: the rows, or KeptRows of them.  round_dz: in bfloat16 with "gelu" and "silu", the gradient at x w + bias
        rounded to bfloat16 for the products: faster, and less exact (DC_DZ_ROUNDED)."""
        torch = self.torch
        rows, n_out, lddy, dtype = self._rows(dy, "dy")
        n_in, wc, ldw, wt = self._rows(w, "w")
        if wc != n_out or wt != dtype:
            raise ValueError(f"w: need {n_out} columns of dy's type")
        code = self._act(act)
        if code == DC_ACT_NONE:
            pz, ldz = 0, 0
        elif pre is None:
            raise ValueError("pre: the gradient of the activation needs x w + bias")
        else:
            pz, ldz = pre.data_ptr(), self._like(pre, "pre", rows, n_out, dtype)
        px, ldx, kept = 0, 0, None
        if isinstance(x, KeptRows):
            kept = C.create_string_buffer(self._kept(x, rows, n_in), _KEPT.size)
        else:
            px, ldx = x.data_ptr(), self._like(x, "x", rows, n_in, dtype)
        dx = torch.empty((rows, n_in), dtype=dy.dtype, device=self.device) if "x" in want else None
        dw = torch.empty((n_in, n_out), dtype=dy.dtype, device=self.device) if "w" in want else None
        db = torch.empty(n_out, dtype=torch.float32, device=self.device) if "b" in want else None
        size = lib().dc_dense_backward_bytes(self.ctx, dtype, code, rows, n_in, n_out)
        ws = torch.empty(size, dtype=torch.uint8, device=self.device)
        a = _DENSE_BACK.pack(dtype, code, rows, n_in, n_out, dy.data_ptr(), lddy, pz, ldz, px, ldx,
                             0 if kept is None else C.addressof(kept), w.data_ptr(), ldw, 0 if dx is None else dx.data_ptr(), n_in,
                             0 if dw is None else dw.data_ptr(), n_out, 0 if db is None else db.data_ptr(), ws.data_ptr(), size,
                             DC_DZ_ROUNDED if round_dz else DC_DZ_WHOLE)
        st = lib().dc_dense_backward(self.ctx, a, self._raw_stream())
        if st:
            self._ok(st, "dc_dense_backward")
        return dx, dw, db

    def _norm(self, node_off, channels: int, rows: int, groups: int, gamma, beta, backward: int):
        """(graphs, offsets, gamma, beta, workspace, its size)"""
        if node_off.dim() != 1 or node_off.numel() < 1:
            raise ValueError("node_off: need at least one offset")
        n = node_off.numel() - 1
        off = self._vector(node_off, "node_off", n + 1, self.torch.int32)
        pg = 0 if gamma is None else self._vector(gamma, "gamma", channels)
        pb = 0 if beta is None else self._vector(beta, "beta", channels)
        size = lib().dc_graph_norm_bytes(self.ctx, rows, n, channels, groups, backward)
        return n, off, pg, pb, self.torch.empty(size, dtype=self.torch.uint8, device=self.device) if size else None, size

    def graph_norm(self, x, node_off, groups: int, gamma=None, beta=None, eps: float = 1e-5, act: str = "none", out=None):
        """(y, mean, rstd): the norm over the rows of each graph and the channels of each group, with an activation.  Rows
        of no graph are left as they are in `out`."""
        rows, channels, ldx, dtype = self._rows(x, "x")
        n, off, pg, pb, ws, size = self._norm(node_off, channels, rows, groups, gamma, beta, 0)
        if out is None:
            out, ldy = self.torch.empty((rows, channels), dtype=x.dtype, device=self.device), channels
        else:
            ldy = self._like(out, "out", rows, channels, dtype)
        mean, rstd = self.torch.empty((2, n, groups), dtype=self.torch.float32, device=self.device).unbind(0)
        a = _NORM.pack(dtype, self._act(act), rows, n, channels, groups, eps, off, x.data_ptr(), ldx, pg, pb, mean.data_ptr(),
                       rstd.data_ptr(), out.data_ptr(), ldy, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0 if ws is None else ws.data_ptr(), size)
        st = lib().dc_graph_norm(self.ctx, a, self._raw_stream())
        if st:
            self._ok(st, "dc_graph_norm")
        return out, mean, rstd

    def graph_norm_backward(self, dy, x, node_off, groups: int, gamma, beta, mean, rstd, act: str = "none", residual=None,
                            out=None):
        """(dx, dgamma, dbeta) for the gradient dy at the result; `residual` is added to dx.  x: the rows, or KeptRows of
        them; mean, rstd: what graph_norm returned."""
        rows, channels, lddy, dtype = self._rows(dy, "dy")
        n, off, pg, pb, ws, size = self._norm(node_off, channels, rows, groups, gamma, beta, 1)
        for v, name in ((mean, "mean"), (rstd, "rstd")):
            if v.device != self.device or v.dtype != self.torch.float32 or tuple(v.shape) != (n, groups) or not v.is_contiguous():
                raise ValueError(f"{name}: need contiguous float32 [{n}, {groups}] on {self.device}")
        if out is None:
            out, lddx = self.torch.empty((rows, channels), dtype=dy.dtype, device=self.device), channels
        else:
            lddx = self._like(out, "out", rows, channels, dtype)
        px, ldx, kept = 0, 0, None
        if isinstance(x, KeptRows):
            kept = C.create_string_buffer(self._kept(x, rows, channels), _KEPT.size)
        else:
            px, ldx = x.data_ptr(), self._like(x, "x", rows, channels, dtype)
        pr, ldr = (residual.data_ptr(), self._like(residual, "residual", rows, channels, dtype)) if residual is not None else (0, 0)
        dgamma, dbeta = self.torch.empty((2, channels), dtype=self.torch.float32, device=self.device).unbind(0)
        a = _NORM.pack(dtype, self._act(act), rows, n, channels, groups, 0.0, off, px, ldx, pg, pb, mean.data_ptr(), rstd.data_ptr(),
                       0, 0, 0 if kept is None else C.addressof(kept), dy.data_ptr(), lddy, pr, ldr, out.data_ptr(), lddx,
                       dgamma.data_ptr(), dbeta.data_ptr(), 0 if ws is None else ws.data_ptr(), size)
        st = lib().dc_graph_norm_backward(self.ctx, a, self._raw_stream())
        if st:
            self._ok(st, "dc_graph_norm_backward")
        return out, dgamma, dbeta

    def row_norm(self, x, gamma=None, beta=None, eps: float = 1e-5, act: str = "none", out=None):
        """(y, mean, rstd): the norm over the channels of each row, with an activation."""
        rows, channels, ldx, dtype = self._rows(x, "x")
        pg = 0 if gamma is None else self._vector(gamma, "gamma", channels)
        pb = 0 if beta is None else self._vector(beta, "beta", channels)
        if out is None:
            out, ldy = x.new_empty(rows, channels), channels
        else:
            ldy = self._like(out, "out", rows, channels, dtype)
        mean, rstd = x.new_empty(rows, dtype=self.torch.float32), x.new_empty(rows, dtype=self.torch.float32)
        a = _ROW_NORM.pack(dtype, self._act(act), rows, channels, eps, x.data_ptr(), ldx, pg, pb, mean.data_ptr(), rstd.data_ptr(),
                           out.data_ptr(), ldy, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
        st = lib().dc_row_norm(self.ctx, a, self._raw_stream())
        if st:
            self._ok(st, "dc_row_norm")
        return out, mean, rstd

    def row_norm_backward(self, dy, x, gamma, beta, mean, rstd, act: str = "none", residual=None, out=None):
        """(dx, dgamma, dbeta) for the gradient dy at the result; `residual` is added to dx.  x: the rows, or KeptRows of
        them; mean, rstd: what row_norm returned, taken as they are (mean as rounded: see dc_row_norm_args for rows far from zero)."""
        rows, channels, lddy, dtype = self._rows(dy, "dy")
        pg = 0 if gamma is None else self._vector(gamma, "gamma", channels)
        pb = 0 if beta is None else self._vector(beta, "beta", channels)
        pm, ps = self._vector(mean, "mean", rows), self._vector(rstd, "rstd", rows)
        if out is None:
            out, lddx = dy.new_empty(rows, channels), channels
        else:
            lddx = self._like(out, "out", rows, channels, dtype)
        px, ldx, kept = 0, 0, None
        if isinstance(x, KeptRows):
            kept = C.create_string_buffer(self._kept(x, rows, channels), _KEPT.size)
        else:
            px, ldx = x.data_ptr(), self._like(x, "x", rows, channels, dtype)
        pr, ldr = (residual.data_ptr(), self._like(residual, "residual", rows, channels, dtype)) if residual is not None else (0, 0)
        dgamma, dbeta = dy.new_empty(channels, dtype=self.torch.float32), dy.new_empty(channels, dtype=self.torch.float32)
        size = lib().dc_row_norm_bytes(self.ctx, rows, channels)
        ws = dy.new_empty(size, dtype=self.torch.uint8)
        a = _ROW_NORM.pack(dtype, self._act(act), rows, channels, 0.0, px, ldx, pg, pb, pm, ps, 0, 0,
                           0 if kept is None else C.addressof(kept), dy.data_ptr(), lddy, pr, ldr, out.data_ptr(), lddx,
                           dgamma.data_ptr(), dbeta.data_ptr(), ws.data_ptr(), size)
        st = lib().dc_row_norm_backward(self.ctx, a, self._raw_stream())
        if st:
            self._ok(st, "dc_row_norm_backward")
        return out, dgamma, dbeta

    def _ids(self, ids, rows=None) -> int:
        if ids.dim() != 1 or (rows is not None and ids.shape[0] != rows):
            raise ValueError("ids: need one number for each row")
        return self._vector(ids, "ids", ids.shape[0], self.torch.int32)

    def embed_rows(self, ids, table, scale: float = 1.0, out=None):
        """scale * table[ids], rows of zeros where an id is -1; ids: int32.  check() reports ids that are neither."""
        kinds, channels, ldt, dtype = self._rows(table, "table")
        pid, rows = self._ids(ids), ids.shape[0]
        if out is None:
            out, ldy = table.new_empty(rows, channels), channels
        else:
            ldy = self._like(out, "out", rows, channels, dtype)
        a = _EMBED.pack(dtype, rows, kinds, channels, scale, pid, table.data_ptr(), ldt, out.data_ptr(), ldy, 0, 0, 0, 0, 0, 0)
        st = lib().dc_embed_rows(self.ctx, a, self._raw_stream())
        if st:
            self._ok(st, "dc_embed_rows")
        return out

    def embed_rows_backward(self, dy, ids, kinds: int, scale: float = 1.0, out=None):
        """The gradient of embed_rows' table of `kinds` rows for the gradient dy at the result."""
        rows, channels, lddy, dtype = self._rows(dy, "dy")
        if kinds < 1:
            raise ValueError("kinds: need at least one")
        pid = self._ids(ids, rows)
        if out is None:
            out, ldt = dy.new_empty(kinds, channels), channels
        else:
            ldt = self._like(out, "out", kinds, channels, dtype)
        size = lib().dc_embed_rows_bytes(self.ctx, rows, kinds, channels)
        ws = dy.new_empty(size, dtype=self.torch.uint8)
        a = _EMBED.pack(dtype, rows, kinds, channels, scale, pid, 0, 0, 0, 0, dy.data_ptr(), lddy, out.data_ptr(), ldt, ws.data_ptr(), size)
        st = lib().dc_embed_rows_backward(self.ctx, a, self._raw_stream())
        if st:
            self._ok(st, "dc_embed_rows_backward")
        return out

    def adamw(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, states: str = "f32",
              seed: int = 0) -> AdamW:
        """An AdamW optimiser of the tensors `params` (float32 or bfloat16, updated in place), all of them in one call a step.
        weight_decay: a number, or one for every tensor; states: moments in "f32" or "8bit", rounded by draws from `seed`."""
        return AdamW(self, params, lr, betas, eps, weight_decay, states, seed)

    def get_weights(self):
        """(W_layers, b_layers, head) as host fp32 arrays in the layout of dc_set_weights."""
        c = self.cfg
        nW = sum(3 * (c.F if l == 0 else c.H) * c.H for l in range(c.L))
        W = np.empty(nW, np.float32)
        b = np.empty(c.L * c.H, np.float32)
        hd = np.empty(2 * c.H * c.H + 3 * c.H + 1, np.float32)
        self._ok(dc_get_weights(self.ctx, W, b, hd, self._stream()), "dc_get_weights")
        return W, b, hd

    def last_fused_ops(self) -> Tuple[int, int, int]:
        st, k, m, e = dc_last_fused_ops(self.ctx, self._stream())
        self._ok(st, "dc_last_fused_ops")
        return k, m, e

    def last_fused_op_repeats(self) -> int:
        st, n = dc_last_fused_op_repeats(self.ctx, self._stream())
        self._ok(st, "dc_last_fused_op_repeats")
        return n

    def walked_modules(self) -> int:
        st, n = dc_walked_modules(self.ctx, self._stream())
        self._ok(st, "dc_walked_modules")
        return n

    def check(self) -> int:
        return dc_check(self.ctx, self._stream())

    def select_kernels(self, which: int) -> None:
        st = dc_select_kernels(self.ctx, which)
        if st != DC_OK:
            raise DiscoError(st, "dc_select_kernels")

    def last_totals(self) -> Tuple[int, int]:
        st, n, e = dc_last_totals(self.ctx, self._stream())
        self._ok(st, "dc_last_totals")
        return n, e

    def profile_begin(self):
        self._ok(dc_profile_begin(self.ctx), "dc_profile_begin")

    def profile_end(self):
        return dc_profile_end(self.ctx)


def evaluator_for(w, slack: float = 1.0, max_nodes: int = 0, max_edges: int = 0, device: str = "cuda:0") -> Evaluator:
    """Evaluator sized for workload `w` (a workloads.Workload) with its base graphs and weights set."""
    geo = w.g_edge_off()
    nb = int(w.cand_off[-1])
    eb = int(sum(int(geo[b + 1] - geo[b]) for b in w.cand_graph))
    ev = Evaluator(w.model.F, w.model.H, w.model.L, w.model.dtype, max(w.n_cand, 1), max(int(nb * slack), 1),
                   max(int(eb * slack), 1), max_nodes, max_edges, device, getattr(w.model, "agg", "mean"),
                   getattr(w.model, "heads", 1))
    ev.set_base_graphs(w.g_node_off(), geo, w.cat_rowptr(), w.cat_col(), w.cat_X())
    ev.set_weights(w.weights)
    return ev
