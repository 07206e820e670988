"""Thin ctypes binding of libgnn.so (include/gnn.h), with the same names.

Argument marshalling only: every step of the inference runs in the HIP
kernels of libgnn.so.  Device buffers are passed as torch tensors (or raw
integer addresses); torch is used for device memory and streams, nothing
else.  There is no fallback: if the library is missing, importing this
module raises.
"""
from __future__ import annotations

import ctypes
import os
import warnings

import numpy as np
import torch  # imported first so that libgnn.so binds to the HIP runtime torch loaded

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgnn.so")

GNN_OK = 0
GNN_E_INVALID_ARG = -1
GNN_E_NO_DEVICE = -2
GNN_E_OOM = -3
GNN_E_INDEX = -4
GNN_E_HIP = -5
GNN_E_UNSUPPORTED = -6
GNN_FP32 = 0
GNN_BF16 = 1
GNN_F16 = 2
GNN_INT8 = 3
GNN_MLP_MAX_LAYERS = 8
GNN_VALIDATE_INDICES = 1
GNN_LITERAL_GATHER = 2
GNN_FP32_MFMA = 4
GNN_F16_WEIGHTS = 8
GNN_PROFILE_SAMPLE = 2
GNN_SILU = 0
GNN_GELU = 1
GNN_SIGMOID = 2
GNN_RELU = 3

EXPORTS = ("gnn_weight_count", "gnn_create", "gnn_infer", "gnn_infer_logits", "gnn_infer_noalloc",
           "gnn_filter_weight_count", "gnn_filter_create", "gnn_filter_apply",
           "gnn_filter_destroy", "gnn_wcc", "gnn_infer_labels", "gnn_destroy",
           "gnn_release_workspaces", "gnn_last_error",
           "gnn_profile_enable", "gnn_profile_read", "gnn_debug_csr", "gnn_debug_stages",
           "gnn_server_create", "gnn_server_submit", "gnn_server_wait", "gnn_server_wait_info",
           "gnn_server_destroy", "gnn_set_workspace_limit",
           "gnn_embed_weight_count", "gnn_embed_create", "gnn_embed_apply", "gnn_embed_destroy",
           "gnn_frnn", "gnn_debug_shared", "gnn_debug_frnn", "gnn_debug_frnn_bytes",
           "gnn_hbm_probe", "gnn_quantize_rows", "gnn_group_workspace", "gnn_group_rows",
           "gnn_linear_weight_count", "gnn_linear_create", "gnn_linear_workspace",
           "gnn_linear_apply", "gnn_linear_destroy", "gnn_mlp_weight_count", "gnn_mlp_create",
           "gnn_mlp_workspace", "gnn_mlp_apply", "gnn_mlp_destroy", "gnn_last_error_code",
           "gnn_debug_linear", "gnn_layer_norm", "gnn_layer_norm_workspace",
           "gnn_layer_norm_backward", "gnn_gated_workspace", "gnn_gated", "gnn_gated_backward",
           "gnn_clip_workspace", "gnn_clip_grads", "gnn_debug_gated")
STAGES = ("csr", "node_enc", "edge_enc", "edge_update", "aggregate", "node_update",
          "classifier", "total")


class gnn_embed_dims(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("in_features", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("out_dim", ctypes.c_int32),
                ("ln_eps", ctypes.c_float)]


class gnn_dims(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("in_features", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("n_iters", ctypes.c_int32),
                ("n_mp_weight_sets", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("ln_eps", ctypes.c_float), ("flags", ctypes.c_uint32)]


def make_dims(in_features=3, hidden=128, n_iters=8, n_mp_weight_sets=1, dtype=GNN_FP32,
              ln_eps=1e-5, flags=0) -> gnn_dims:
    return gnn_dims(ctypes.sizeof(gnn_dims), in_features, hidden, n_iters, n_mp_weight_sets,
                    dtype, ln_eps, flags)


class gnn_filter_dims(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("in_features", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("ln_eps", ctypes.c_float)]


def make_filter_dims(in_features=3, hidden=64, ln_eps=1e-5) -> gnn_filter_dims:
    return gnn_filter_dims(ctypes.sizeof(gnn_filter_dims), in_features, hidden, ln_eps)


_INT32_MAX = 2 ** 31 - 1


def _int32(what: str, v) -> int:
    """A whole number of 32 bits: ctypes would pass the low bits of a larger one."""
    if -_INT32_MAX - 1 <= v <= _INT32_MAX:
        return v
    raise ValueError(f"{what}: {v} is not a 32-bit number")


class gnn_linear_dims(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("in_features", ctypes.c_int32),
                ("out_features", ctypes.c_int32), ("n_groups", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


def make_linear_dims(in_features, out_features, n_groups=1, dtype=GNN_BF16) -> gnn_linear_dims:
    return gnn_linear_dims(ctypes.sizeof(gnn_linear_dims), _int32("in_features", in_features),
                           _int32("out_features", out_features), _int32("n_groups", n_groups),
                           dtype)


class gnn_mlp_dims(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("n_layers", ctypes.c_int32),
                ("widths", ctypes.c_int32 * (GNN_MLP_MAX_LAYERS + 1)),
                ("n_groups", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("ln_eps", ctypes.c_float)]


def make_mlp_dims(widths, n_groups=1, dtype=GNN_BF16, ln_eps=1e-5) -> gnn_mlp_dims:
    """widths: of the input, the hidden layers and the output."""
    if not 2 <= len(widths) <= GNN_MLP_MAX_LAYERS + 1:
        raise ValueError(f"2..{GNN_MLP_MAX_LAYERS + 1} widths, got {len(widths)}")
    w = (ctypes.c_int32 * (GNN_MLP_MAX_LAYERS + 1))(*[_int32("width", v) for v in widths])
    return gnn_mlp_dims(ctypes.sizeof(gnn_mlp_dims), len(widths) - 1, w,
                        _int32("n_groups", n_groups), dtype, ln_eps)


class gnn_gated_dims(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("in_features", ctypes.c_int32),
                ("hidden", ctypes.c_int32), ("out_features", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("activation", ctypes.c_int32)]


def make_gated_dims(in_features, hidden, out_features, dtype=GNN_BF16,
                    activation=GNN_SILU) -> gnn_gated_dims:
    return gnn_gated_dims(ctypes.sizeof(gnn_gated_dims), _int32("in_features", in_features),
                          _int32("hidden", hidden), _int32("out_features", out_features),
                          dtype, activation)


class gnn_gated_weights(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [
        (name, ctypes.c_void_p) for name in ("gate", "up", "down", "gate_bias", "up_bias",
                                             "down_bias")]


class gnn_grad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("count", ctypes.c_int64),
                ("type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class gnn_profile_stats(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("n_calls", ctypes.c_int32),
                ("launches", ctypes.c_int64 * 8), ("ms", ctypes.c_double * 8)]


class gnn_request_info(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("status", ctypes.c_int32),
                ("latency_ms", ctypes.c_double), ("device_start_ms", ctypes.c_double),
                ("device_end_ms", ctypes.c_double)]


class GnnError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libgnn error {code}: {msg}")
        self.code = code


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() first")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    dp = ctypes.POINTER(gnn_dims)
    L.gnn_weight_count.restype = ctypes.c_size_t
    L.gnn_weight_count.argtypes = [dp]
    L.gnn_create.restype = vp
    L.gnn_create.argtypes = [vp, dp]
    for name in ("gnn_infer", "gnn_infer_logits", "gnn_infer_noalloc"):
        f = getattr(L, name)
        f.restype = ctypes.c_int
        f.argtypes = [vp, vp, vp, i64, i64, vp, vp]
    fdp = ctypes.POINTER(gnn_filter_dims)
    L.gnn_filter_weight_count.restype = ctypes.c_size_t
    L.gnn_filter_weight_count.argtypes = [fdp]
    L.gnn_filter_create.restype = vp
    L.gnn_filter_create.argtypes = [vp, fdp]
    L.gnn_filter_destroy.restype = None
    L.gnn_filter_destroy.argtypes = [vp]
    L.gnn_filter_apply.restype = ctypes.c_int
    L.gnn_filter_apply.argtypes = [vp, vp, vp, i64, i64, ctypes.c_float, vp, vp,
                                   ctypes.POINTER(ctypes.c_int64), vp]
    L.gnn_wcc.restype = ctypes.c_int
    L.gnn_wcc.argtypes = [vp, vp, ctypes.c_float, i64, i64, vp, vp]
    L.gnn_infer_labels.restype = ctypes.c_int
    L.gnn_infer_labels.argtypes = [vp, vp, vp, i64, i64, ctypes.c_float, vp, vp, vp]
    L.gnn_destroy.restype = None
    L.gnn_destroy.argtypes = [vp]
    L.gnn_release_workspaces.restype = ctypes.c_int64
    L.gnn_release_workspaces.argtypes = [vp]
    L.gnn_set_workspace_limit.restype = ctypes.c_int
    L.gnn_set_workspace_limit.argtypes = [vp, i64]
    L.gnn_last_error.restype = ctypes.c_char_p
    L.gnn_last_error.argtypes = []
    L.gnn_last_error_code.restype = ctypes.c_int
    L.gnn_last_error_code.argtypes = []
    L.gnn_profile_enable.restype = ctypes.c_int
    L.gnn_profile_enable.argtypes = [vp, ctypes.c_int]
    L.gnn_profile_read.restype = ctypes.c_int
    L.gnn_profile_read.argtypes = [vp, ctypes.POINTER(gnn_profile_stats)]
    L.gnn_hbm_probe.restype = ctypes.c_int
    L.gnn_hbm_probe.argtypes = [ctypes.c_int, vp, vp, i64, i32, i32, ctypes.POINTER(ctypes.c_float),
                                vp]
    L.gnn_debug_csr.restype = ctypes.c_int
    L.gnn_debug_csr.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, vp]
    L.gnn_debug_stages.restype = ctypes.c_int
    L.gnn_debug_stages.argtypes = [vp, vp, vp, i64, i64, i32, vp, vp, vp, vp, vp]
    edp = ctypes.POINTER(gnn_embed_dims)
    L.gnn_embed_weight_count.restype = ctypes.c_size_t
    L.gnn_embed_weight_count.argtypes = [edp]
    L.gnn_embed_create.restype = vp
    L.gnn_embed_create.argtypes = [vp, edp]
    L.gnn_embed_apply.restype = ctypes.c_int
    L.gnn_embed_apply.argtypes = [vp, vp, i64, vp, vp]
    L.gnn_embed_destroy.restype = None
    L.gnn_embed_destroy.argtypes = [vp]
    L.gnn_debug_shared.restype = ctypes.c_int
    L.gnn_debug_shared.argtypes = [vp, vp]
    L.gnn_debug_frnn.restype = ctypes.c_int
    L.gnn_debug_frnn.argtypes = [vp, i64, i32, ctypes.c_float, vp, i64,
                                 ctypes.POINTER(ctypes.c_int64), i32, i64, vp]
    L.gnn_debug_frnn_bytes.restype = ctypes.c_size_t
    L.gnn_debug_frnn_bytes.argtypes = [i64, i32, i32]
    L.gnn_frnn.restype = ctypes.c_int
    L.gnn_frnn.argtypes = [vp, i64, i32, ctypes.c_float, vp, i64, ctypes.POINTER(ctypes.c_int64),
                           vp]
    L.gnn_quantize_rows.restype = ctypes.c_int
    L.gnn_quantize_rows.argtypes = [vp, i32, i64, i64, i32, vp, i64, vp, vp]
    L.gnn_group_workspace.restype = ctypes.c_size_t
    L.gnn_group_workspace.argtypes = [i64, i32]
    L.gnn_group_rows.restype = ctypes.c_int
    L.gnn_group_rows.argtypes = [vp, i64, i32, vp, vp, vp, i64, vp]
    for name, dims in (("linear", gnn_linear_dims), ("mlp", gnn_mlp_dims)):
        f = getattr(L, f"gnn_{name}_weight_count")
        f.restype, f.argtypes = ctypes.c_size_t, [ctypes.POINTER(dims)]
        f = getattr(L, f"gnn_{name}_create")
        f.restype, f.argtypes = vp, [vp, ctypes.POINTER(dims)]
        f = getattr(L, f"gnn_{name}_workspace")
        f.restype, f.argtypes = ctypes.c_size_t, [vp, i32, i64]
        f = getattr(L, f"gnn_{name}_destroy")
        f.restype, f.argtypes = None, [vp]
    L.gnn_linear_apply.restype = ctypes.c_int
    L.gnn_linear_apply.argtypes = [vp, vp, i32, i64, vp, i64, vp, vp, vp, i32, i64, vp, i64, vp]
    L.gnn_debug_linear.restype = ctypes.c_int
    L.gnn_debug_linear.argtypes = [ctypes.POINTER(gnn_linear_dims), i32, i32, i64, i32, i32, i64,
                                   ctypes.POINTER(ctypes.c_int32)]
    L.gnn_mlp_apply.restype = ctypes.c_int
    L.gnn_mlp_apply.argtypes = [vp, vp, i32, i64, vp, i64, vp, i32, i64, vp, i64, vp]
    L.gnn_layer_norm.restype = ctypes.c_int
    L.gnn_layer_norm.argtypes = [vp, i32, i64, i64, i32, vp, vp, ctypes.c_float, vp, i64, vp, vp,
                                 vp]
    L.gnn_layer_norm_workspace.restype = ctypes.c_size_t
    L.gnn_layer_norm_workspace.argtypes = [i64, i32]
    L.gnn_layer_norm_backward.restype = ctypes.c_int
    L.gnn_layer_norm_backward.argtypes = [vp, i64, vp, i64, i32, i64, i32, vp, vp, vp, vp, i64, vp,
                                          vp, vp, i64, vp]
    gdp, gwp = ctypes.POINTER(gnn_gated_dims), ctypes.POINTER(gnn_gated_weights)
    L.gnn_gated_workspace.restype = ctypes.c_size_t
    L.gnn_gated_workspace.argtypes = [gdp, i64, i32, i32]
    L.gnn_gated.restype = ctypes.c_int
    L.gnn_gated.argtypes = [gdp, gwp, vp, i64, i64, vp, i64, vp, i64, vp]
    L.gnn_gated_backward.restype = ctypes.c_int
    L.gnn_gated_backward.argtypes = [gdp, gwp, vp, i64, vp, i64, i64, vp, i64, gwp, vp, i64, vp]
    L.gnn_debug_gated.restype = ctypes.c_int
    L.gnn_debug_gated.argtypes = [gdp, i32, i64, i32, ctypes.POINTER(ctypes.c_int32)]
    L.gnn_clip_workspace.restype = ctypes.c_size_t
    L.gnn_clip_workspace.argtypes = [vp, i32]
    L.gnn_clip_grads.restype = ctypes.c_int
    L.gnn_clip_grads.argtypes = [vp, i32, ctypes.c_float, vp, vp, i64, vp]
    L.gnn_server_create.restype = vp
    L.gnn_server_create.argtypes = [vp, ctypes.c_int]
    L.gnn_server_submit.restype = i64
    L.gnn_server_submit.argtypes = [vp, vp, vp, i64, i64, vp]
    L.gnn_server_wait.restype = ctypes.c_int
    L.gnn_server_wait.argtypes = [vp, i64, ctypes.POINTER(ctypes.c_double)]
    L.gnn_server_wait_info.restype = ctypes.c_int
    L.gnn_server_wait_info.argtypes = [vp, i64, ctypes.POINTER(gnn_request_info)]
    L.gnn_server_destroy.restype = None
    L.gnn_server_destroy.argtypes = [vp]
    return L


lib = _load()


def _addr(t) -> int | None:
    """Device address of a tensor (checked contiguous), an int, or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, torch.Tensor):
        if not t.is_contiguous():
            raise ValueError("tensor arguments must be contiguous")
        return t.data_ptr()
    raise TypeError(f"expected a tensor, an int address or None, got {type(t)}")


def _stream(stream) -> int | None:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _check(rc: int) -> int:
    if rc != GNN_OK:
        raise GnnError(rc, gnn_last_error())
    return rc


def gnn_last_error() -> str:
    return lib.gnn_last_error().decode()


def gnn_last_error_code() -> int:
    return int(lib.gnn_last_error_code())


def gnn_weight_count(dims: gnn_dims) -> int:
    return int(lib.gnn_weight_count(ctypes.byref(dims)))


def gnn_create(weights: np.ndarray, dims: gnn_dims) -> int:
    """Upload a host fp32 weight blob; returns the handle (an address)."""
    w = np.ascontiguousarray(weights, dtype=np.float32)
    n = gnn_weight_count(dims)
    if n == 0:
        raise GnnError(GNN_E_INVALID_ARG, gnn_last_error())
    if w.size != n:
        raise ValueError(f"weight blob has {w.size} floats, dims need {n}")
    h = lib.gnn_create(w.ctypes.data, ctypes.byref(dims))
    if not h:
        raise GnnError(GNN_E_INVALID_ARG, gnn_last_error())
    return h


def gnn_destroy(handle) -> None:
    lib.gnn_destroy(handle)


def gnn_release_workspaces(handle) -> int:
    """Frees the handle's idle cached workspaces; returns the bytes freed."""
    r = lib.gnn_release_workspaces(handle)
    if r < 0:
        raise GnnError(int(r), gnn_last_error())
    return int(r)


def gnn_set_workspace_limit(handle, n_bytes: int) -> int:
    """Caps the handle's inference workspace bytes (0 = no cap)."""
    return _check(lib.gnn_set_workspace_limit(handle, int(n_bytes)))


def _check_io(node_feat, edge_index, out):
    for t, dt in ((node_feat, torch.float32), (edge_index, torch.int32), (out, torch.float32)):
        if isinstance(t, torch.Tensor):
            if t.dtype != dt:
                raise TypeError(f"expected {dt}, got {t.dtype}")
            if not t.is_cuda:
                raise ValueError("inputs and outputs must be device tensors")


def gnn_infer(handle, node_feat, edge_index, n_nodes: int, n_edges: int, edge_scores,
              stream=None) -> int:
    _check_io(node_feat, edge_index, edge_scores)
    return _check(lib.gnn_infer(handle, _addr(node_feat), _addr(edge_index), n_nodes, n_edges,
                                _addr(edge_scores), _stream(stream)))


def gnn_infer_logits(handle, node_feat, edge_index, n_nodes: int, n_edges: int, edge_logits,
                     stream=None) -> int:
    _check_io(node_feat, edge_index, edge_logits)
    return _check(lib.gnn_infer_logits(handle, _addr(node_feat), _addr(edge_index), n_nodes,
                                       n_edges, _addr(edge_logits), _stream(stream)))


def gnn_infer_noalloc(handle, node_feat, edge_index, n_nodes: int, n_edges: int, edge_scores,
                      stream=None) -> int:
    """gnn_infer in the library's fixed scratch array: allocates nothing."""
    _check_io(node_feat, edge_index, edge_scores)
    return _check(lib.gnn_infer_noalloc(handle, _addr(node_feat), _addr(edge_index), n_nodes,
                                        n_edges, _addr(edge_scores), _stream(stream)))


def gnn_filter_weight_count(dims: gnn_filter_dims) -> int:
    return int(lib.gnn_filter_weight_count(ctypes.byref(dims)))


def gnn_filter_create(weights: np.ndarray, dims: gnn_filter_dims) -> int:
    w = np.ascontiguousarray(weights, dtype=np.float32)
    n = gnn_filter_weight_count(dims)
    if n == 0:
        raise GnnError(GNN_E_INVALID_ARG, gnn_last_error())
    if w.size != n:
        raise ValueError(f"filter blob has {w.size} floats, dims need {n}")
    h = lib.gnn_filter_create(w.ctypes.data, ctypes.byref(dims))
    if not h:
        raise GnnError(GNN_E_INVALID_ARG, gnn_last_error())
    return h


def gnn_filter_destroy(handle) -> None:
    lib.gnn_filter_destroy(handle)


def gnn_filter_apply(handle, node_feat, edge_index, n_nodes: int, n_edges: int,
                     threshold: float, edge_scores, edge_index_out, stream=None) -> int:
    """Returns n_kept; edge_index_out[: 2 * n_kept] holds the kept edges as [2][n_kept]."""
    nk = ctypes.c_int64(0)
    _check(lib.gnn_filter_apply(handle, _addr(node_feat), _addr(edge_index), n_nodes, n_edges,
                                float(threshold), _addr(edge_scores), _addr(edge_index_out),
                                ctypes.byref(nk), _stream(stream)))
    return int(nk.value)


def gnn_wcc(edge_index, edge_scores, threshold: float, n_nodes: int, n_edges: int, labels,
            stream=None) -> int:
    """Component labels (smallest node id per component) of the edges scoring
    above `threshold`; edge_scores may be None (every edge kept)."""
    for t, dt in ((edge_index, torch.int32), (edge_scores, torch.float32), (labels, torch.int32)):
        if isinstance(t, torch.Tensor) and t.dtype != dt:
            raise TypeError(f"expected {dt}, got {t.dtype}")
    return _check(lib.gnn_wcc(_addr(edge_index), _addr(edge_scores), float(threshold), n_nodes,
                              n_edges, _addr(labels), _stream(stream)))


def gnn_infer_labels(handle, node_feat, edge_index, n_nodes: int, n_edges: int,
                     threshold: float, edge_scores, labels, stream=None) -> int:
    return _check(lib.gnn_infer_labels(handle, _addr(node_feat), _addr(edge_index), n_nodes,
                                       n_edges, float(threshold), _addr(edge_scores),
                                       _addr(labels), _stream(stream)))


def gnn_profile_enable(handle, enable=True) -> int:
    """enable: False/0 off, True/1 every stage, GNN_PROFILE_SAMPLE."""
    mode = int(enable) if not isinstance(enable, bool) else (1 if enable else 0)
    return _check(lib.gnn_profile_enable(handle, mode))


def gnn_profile_read(handle) -> dict:
    """{'n_calls': n, stage: {'launches': k, 'ms': total_ms}} per stage."""
    st = gnn_profile_stats()
    st.struct_size = ctypes.sizeof(gnn_profile_stats)
    _check(lib.gnn_profile_read(handle, ctypes.byref(st)))
    out = {"n_calls": st.n_calls}
    for i, name in enumerate(STAGES):
        out[name] = {"launches": int(st.launches[i]), "ms": float(st.ms[i])}
    return out


GNN_PROBE_READ, GNN_PROBE_WRITE, GNN_PROBE_COPY = 0, 1, 2


def gnn_hbm_probe(kind: int, buf, buf2, nbytes: int, grid: int = 0, reps: int = 5,
                  stream=None) -> float:
    """Fastest of `reps` timed launches of the streaming probe, in ms."""
    ms = ctypes.c_float(0.0)
    _check(lib.gnn_hbm_probe(kind, _addr(buf), _addr(buf2), nbytes, grid, reps, ctypes.byref(ms),
                             _stream(stream)))
    return float(ms.value)


def gnn_debug_csr(handle, edge_index, n_nodes: int, n_edges: int, row_ptr_in=None, perm_in=None,
                  row_ptr_out=None, perm_out=None, stream=None) -> int:
    return _check(lib.gnn_debug_csr(handle, _addr(edge_index), n_nodes, n_edges,
                                    _addr(row_ptr_in), _addr(perm_in), _addr(row_ptr_out),
                                    _addr(perm_out), _stream(stream)))


def gnn_debug_stages(handle, node_feat, edge_index, n_nodes: int, n_edges: int, stop_iter: int,
                     h_out=None, e_out=None, agg_in_out=None, agg_out_out=None,
                     stream=None) -> int:
    return _check(lib.gnn_debug_stages(handle, _addr(node_feat), _addr(edge_index), n_nodes,
                                       n_edges, stop_iter, _addr(h_out), _addr(e_out),
                                       _addr(agg_in_out), _addr(agg_out_out), _stream(stream)))


def gnn_debug_shared(handle, stream=None) -> bool:
    """Whether a call on `stream` would find another inference in flight."""
    rc = lib.gnn_debug_shared(handle, _stream(stream))
    if rc < 0:
        raise GnnError(rc, gnn_last_error())
    return bool(rc)


def make_embed_dims(in_features=3, hidden=64, out_dim=8, ln_eps=1e-5) -> gnn_embed_dims:
    return gnn_embed_dims(ctypes.sizeof(gnn_embed_dims), in_features, hidden, out_dim, ln_eps)


def gnn_embed_weight_count(dims: gnn_embed_dims) -> int:
    return int(lib.gnn_embed_weight_count(ctypes.byref(dims)))


def gnn_embed_create(weights: np.ndarray, dims: gnn_embed_dims):
    w = np.ascontiguousarray(weights, np.float32)
    if w.size != gnn_embed_weight_count(dims):
        raise ValueError("embedding weight blob has the wrong size")
    m = lib.gnn_embed_create(w.ctypes.data, ctypes.byref(dims))
    if not m:
        raise GnnError(GNN_E_INVALID_ARG, gnn_last_error())
    return m


def gnn_embed_apply(embedder, node_feat, n_nodes: int, z, stream=None) -> int:
    return _check(lib.gnn_embed_apply(embedder, _addr(node_feat), n_nodes, _addr(z),
                                      _stream(stream)))


def gnn_embed_destroy(embedder) -> None:
    lib.gnn_embed_destroy(embedder)


def gnn_frnn(z, n_nodes: int, dim: int, r2: float, edge_index=None, max_pairs: int = 0,
             stream=None) -> int:
    """Fixed-radius pairs of the rows of z; returns the pair count (and
    fills edge_index [2][count] when given and large enough)."""
    cnt = ctypes.c_int64(0)
    rc = lib.gnn_frnn(_addr(z), n_nodes, dim, float(r2), _addr(edge_index), int(max_pairs),
                      ctypes.byref(cnt), _stream(stream))
    if rc != GNN_OK:
        raise GnnError(rc, gnn_last_error())
    return int(cnt.value)


def gnn_debug_frnn(z, n_nodes: int, dim: int, r2: float, edge_index, max_pairs: int,
                   n_slots: int, scan_direct: int, stream=None) -> int:
    """gnn_frnn with the slots per point and the scan's limit given."""
    cnt = ctypes.c_int64(0)
    _check(lib.gnn_debug_frnn(_addr(z), n_nodes, dim, float(r2), _addr(edge_index), int(max_pairs),
                              ctypes.byref(cnt), n_slots, scan_direct, _stream(stream)))
    return int(cnt.value)


class Embedder:
    """Owns one embedding model: ``Embedder(w, dims)(x) -> z``."""

    def __init__(self, weights: np.ndarray, dims: gnn_embed_dims):
        self.dims = dims
        self.handle = gnn_embed_create(weights, dims)

    def __call__(self, x: torch.Tensor, z=None, stream=None) -> torch.Tensor:
        if z is None:
            z = torch.empty(x.shape[0], self.dims.out_dim, dtype=torch.float32, device=x.device)
        gnn_embed_apply(self.handle, x, x.shape[0], z, stream)
        return z

    def close(self):
        if self.handle:
            gnn_embed_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def radius_graph(z: torch.Tensor, r2: float, stream=None) -> torch.Tensor:
    """[2][n_pairs] int32 edge list of the pairs i < j of rows of z with
    fp32 squared distance < r2 (count first, then fill)."""
    n, d = z.shape
    cap = max(16 * n, 1)  # one call when the pairs fit, a second one otherwise
    out = torch.empty(2 * cap, dtype=torch.int32, device=z.device)
    try:
        cnt = gnn_frnn(z, n, d, r2, out, cap, stream)
    except GnnError as e:
        if e.code != GNN_E_INVALID_ARG:
            raise
        cnt = gnn_frnn(z, n, d, r2, None, 0, stream)
        out = torch.empty(2 * max(cnt, 1), dtype=torch.int32, device=z.device)
        cnt = gnn_frnn(z, n, d, r2, out, cnt, stream)
    return out[:2 * cnt].view(2, cnt)


# ---- linear layers of wide and per-region networks ----

_TYPES = {torch.float32: GNN_FP32, torch.bfloat16: GNN_BF16, torch.float16: GNN_F16,
          torch.int8: GNN_INT8}


def _on(device, stream):
    """Context in which what is allocated, and what runs, belongs to `stream` of
    `device`."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    if stream.device != device:
        raise ValueError(f"stream: expected one of {device}, got one of {stream.device}")
    return torch.cuda.stream(stream)


def _rows(what: str, t: torch.Tensor, width=None, n=None, device=None):
    """Checks a table of rows; (address, element type, stride in elements)."""
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise TypeError(f"{what}: expected a 2-D tensor")
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"{what}: rows of {t.dtype} are not supported")
    if t.device != device:
        raise ValueError(f"{what}: expected a tensor on {device}, got {t.device}")
    rows, cols = t.shape
    stride, step = t.stride()
    if width is not None and cols != width:
        raise ValueError(f"{what}: rows of {cols}, expected {width}")
    if n is not None and rows != n:
        raise ValueError(f"{what}: {rows} rows, expected {n}")
    if cols > _INT32_MAX:  # the call's width has 32 bits
        raise ValueError(f"{what}: rows of {cols}, at most {_INT32_MAX} are supported")
    if step != 1 and cols > 1:
        raise ValueError(f"{what}: the elements of a row must be contiguous")
    if stride < cols:
        if rows > 1:
            raise ValueError(f"{what}: rows overlap")
        stride = cols
    return t.data_ptr(), kind, stride


def _vector(what: str, t, dtype, n: int, device):
    """Address of a contiguous vector of n elements, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.shape != (n,):
        raise TypeError(f"{what}: expected a {dtype} tensor of shape ({n},)")
    if not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what}: expected a contiguous tensor on {device}")
    return t.data_ptr()


def _scratch(nbytes: int, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _device(what: str, t) -> torch.device:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what}: expected a tensor on the GPU")
    return t.device


def gnn_quantize_rows(x, x_type: int, x_stride: int, n_rows: int, width: int, q, q_stride: int,
                      scales, stream=None) -> int:
    """As the C call; addresses or contiguous tensors."""
    _int32("width", width)
    return _check(lib.gnn_quantize_rows(_addr(x), x_type, x_stride, n_rows, width, _addr(q),
                                        q_stride, _addr(scales), _stream(stream)))


# The current stream's handle, without the stream object around it (a call costs
# a third of the time that current_stream() does).
_raw_stream = torch._C._cuda_getCurrentRawStream


def quantize_rows(x: torch.Tensor, out=None, stream=None):
    """(q, scales): the rows of x as int8 with one fp32 scale each; `out`: a pair
    of tensors to fill."""
    dev = _device("x", x)
    if stream is not None or dev.index != torch.cuda.current_device():
        with _on(dev, torch.cuda.current_stream(dev) if stream is None else stream):
            return quantize_rows(x, out)
    xa, xt, xs = _rows("x", x, None, None, dev)
    n, k = x.shape
    q, s = out if out is not None else (torch.empty(n, k, dtype=torch.int8, device=dev),
                                        torch.empty(n, dtype=torch.float32, device=dev))
    qa, qt, qs = _rows("q", q, k, n, dev)
    if qt != GNN_INT8:
        raise TypeError("q: expected int8 rows")
    _check(lib.gnn_quantize_rows(xa, xt, xs, n, k, qa, qs,
                                 _vector("scales", s, torch.float32, n, dev),
                                 _raw_stream(dev.index)))
    return q, s


def gnn_group_workspace(n_rows: int, n_groups: int) -> int:
    return int(lib.gnn_group_workspace(n_rows, _int32("n_groups", n_groups)))


def gnn_group_rows(group_ids, n_rows: int, n_groups: int, offsets, order, workspace=None,
                   workspace_bytes: int = 0, stream=None) -> int:
    """As the C call; addresses or contiguous tensors."""
    _int32("n_groups", n_groups)
    return _check(lib.gnn_group_rows(_addr(group_ids), n_rows, n_groups, _addr(offsets),
                                     _addr(order), _addr(workspace), workspace_bytes,
                                     _stream(stream)))


def group_rows(group_ids: torch.Tensor, n_groups: int, stream=None):
    """(offsets, order) of the rows by their int32 group ids; rows whose id is
    outside [0, n_groups) come last and belong to no group."""
    dev = _device("group_ids", group_ids)
    if stream is not None or dev.index != torch.cuda.current_device():
        with _on(dev, torch.cuda.current_stream(dev) if stream is None else stream):
            return group_rows(group_ids, n_groups)
    n = group_ids.numel()
    ids = _vector("group_ids", group_ids, torch.int32, n, dev)
    nb = gnn_group_workspace(n, n_groups)
    ws = _scratch(nb, dev)
    offsets = torch.empty(max(n_groups, 0) + 1, dtype=torch.int32, device=dev)
    order = torch.empty(n, dtype=torch.int32, device=dev)
    _check(lib.gnn_group_rows(ids, n, n_groups, offsets.data_ptr(), order.data_ptr(),
                              _addr(ws), nb, _raw_stream(dev.index)))
    return offsets, order


def gnn_linear_weight_count(dims: gnn_linear_dims) -> int:
    return int(lib.gnn_linear_weight_count(ctypes.byref(dims)))


def gnn_mlp_weight_count(dims: gnn_mlp_dims) -> int:
    return int(lib.gnn_mlp_weight_count(ctypes.byref(dims)))


def _create_from_blob(count, create, weights, dims, what: str) -> int:
    n = int(count(ctypes.byref(dims)))
    if n == 0:
        raise GnnError(gnn_last_error_code(), gnn_last_error())
    w = np.ascontiguousarray(weights, np.float32)
    if w.size != n:
        raise ValueError(f"{what} blob has {w.size} floats, dims need {n}")
    h = create(w.ctypes.data, ctypes.byref(dims))
    if not h:
        raise GnnError(gnn_last_error_code(), gnn_last_error())
    return h


def gnn_linear_create(weights: np.ndarray, dims: gnn_linear_dims) -> int:
    return _create_from_blob(lib.gnn_linear_weight_count, lib.gnn_linear_create, weights, dims,
                             "linear")


def gnn_linear_destroy(layer) -> None:
    lib.gnn_linear_destroy(layer)


def gnn_linear_workspace(layer, x_type: int, n_rows: int) -> int:
    return int(lib.gnn_linear_workspace(layer, x_type, n_rows))


def gnn_linear_apply(layer, x, x_type: int, x_stride: int, x_scales, n_rows: int, offsets, order,
                     y, y_type: int, y_stride: int, workspace=None, workspace_bytes: int = 0,
                     stream=None) -> int:
    """As the C call; addresses or contiguous tensors."""
    return _check(lib.gnn_linear_apply(layer, _addr(x), x_type, x_stride, _addr(x_scales), n_rows,
                                       _addr(offsets), _addr(order), _addr(y), y_type, y_stride,
                                       _addr(workspace), workspace_bytes, _stream(stream)))


def gnn_debug_linear(dims: gnn_linear_dims, n_cu: int, x_type: int, n_rows: int, grouped=False,
                     y_type: int = GNN_FP32, y_stride: int = 0) -> tuple:
    """The C call's kernel[0 .. 5]; y_stride 0: the output's width."""
    k = (ctypes.c_int32 * 6)()
    _check(lib.gnn_debug_linear(ctypes.byref(dims), n_cu, x_type, n_rows, int(grouped), y_type,
                                y_stride or dims.out_features, k))
    return tuple(k)


def gnn_mlp_create(weights: np.ndarray, dims: gnn_mlp_dims) -> int:
    return _create_from_blob(lib.gnn_mlp_weight_count, lib.gnn_mlp_create, weights, dims, "MLP")


def gnn_mlp_destroy(mlp) -> None:
    lib.gnn_mlp_destroy(mlp)


def gnn_mlp_workspace(mlp, x_type: int, n_rows: int) -> int:
    return int(lib.gnn_mlp_workspace(mlp, x_type, n_rows))


def gnn_mlp_apply(mlp, x, x_type: int, x_stride: int, group_ids, n_rows: int, y, y_type: int,
                  y_stride: int, workspace=None, workspace_bytes: int = 0, stream=None) -> int:
    """As the C call; addresses or contiguous tensors."""
    return _check(lib.gnn_mlp_apply(mlp, _addr(x), x_type, x_stride, _addr(group_ids), n_rows,
                                    _addr(y), y_type, y_stride, _addr(workspace), workspace_bytes,
                                    _stream(stream)))


class _RowsHandle:
    """A handle that turns rows of one width into rows of another."""

    _free = None
    handle = None

    def _out(self, n: int, width: int, x, out, out_dtype, grouped: bool):
        if out is None:
            if out_dtype is None:
                out_dtype = x.dtype if x.dtype.is_floating_point else torch.float32
            # rows of no group are not written: zeros in a new output
            new = torch.zeros if grouped else torch.empty
            out = new(n, width, dtype=out_dtype, device=self.device)
        elif out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out: expected {out_dtype}, got {out.dtype}")
        return out, _rows("out", out, width, n, self.device)

    def close(self):
        if self.handle:
            type(self)._free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Linear(_RowsHandle):
    """Owns one layer: ``Linear(w, dims)(x) -> y``, with ``offsets`` and ``order``
    as ``group_rows`` gives them where the layer has several groups.  x: rows of
    any float type, or int8 rows with their ``scales`` (GNN_INT8 layers).  Rows of
    no group are left as they were in ``out``, zeros in a new output."""

    _free = staticmethod(gnn_linear_destroy)

    def __init__(self, weights: np.ndarray, dims: gnn_linear_dims):
        self.dims = dims
        self.widths = (int(dims.in_features), int(dims.out_features), int(dims.n_groups))
        self.handle = gnn_linear_create(weights, dims)
        self.device = torch.device("cuda", torch.cuda.current_device())

    def __call__(self, x: torch.Tensor, scales=None, offsets=None, order=None, out=None,
                 out_dtype=None, stream=None) -> torch.Tensor:
        (k, n_out, groups), dev = self.widths, self.device
        if stream is not None:
            with _on(dev, stream):
                return self(x, scales, offsets, order, out, out_dtype)
        xa, xt, xs = _rows("x", x, k, None, dev)
        n = x.shape[0]
        sc = _vector("scales", scales, torch.float32, n, dev)
        off = _vector("offsets", offsets, torch.int32, groups + 1, dev)
        ordr = _vector("order", order, torch.int32, n, dev)
        out, (ya, yt, ys) = self._out(n, n_out, x, out, out_dtype,
                                      off is not None or ordr is not None)
        nb = lib.gnn_linear_workspace(self.handle, xt, n)
        ws = _scratch(nb, dev)
        _check(lib.gnn_linear_apply(self.handle, xa, xt, xs, sc, n, off, ordr, ya, yt, ys,
                                    _addr(ws), nb, _raw_stream(dev.index)))
        return out


class Mlp(_RowsHandle):
    """Owns one network of linear layers: ``Mlp(w, dims)(x, group_ids) -> y``.
    Rows of no group are left as they were in ``out``, zeros in a new output."""

    _free = staticmethod(gnn_mlp_destroy)

    def __init__(self, weights: np.ndarray, dims: gnn_mlp_dims):
        self.dims = dims
        # the network's own: the caller may use dims for the next one
        self.widths = tuple(dims.widths[:dims.n_layers + 1])
        self.handle = gnn_mlp_create(weights, dims)
        self.device = torch.device("cuda", torch.cuda.current_device())

    def __call__(self, x: torch.Tensor, group_ids=None, out=None, out_dtype=None,
                 stream=None) -> torch.Tensor:
        dev = self.device
        if stream is not None:
            with _on(dev, stream):
                return self(x, group_ids, out, out_dtype)
        xa, xt, xs = _rows("x", x, self.widths[0], None, dev)
        n = x.shape[0]
        ids = _vector("group_ids", group_ids, torch.int32, n, dev)
        out, (ya, yt, ys) = self._out(n, self.widths[-1], x, out, out_dtype, ids is not None)
        nb = lib.gnn_mlp_workspace(self.handle, xt, n)
        ws = _scratch(nb, dev)
        _check(lib.gnn_mlp_apply(self.handle, xa, xt, xs, ids, n, ya, yt, ys, _addr(ws), nb,
                                 _raw_stream(dev.index)))
        return out


# ---- training operators ----
# None of them records an autograd graph: gradients are what the *_backward calls return.


def _no_graph(name: str, *tensors):
    """Says so where a result stands in a graph that autograd would go back through:
    beside a residual connection, say, nothing else would tell."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        warnings.warn(f"{name} records no autograd graph, though an argument requires grad: use "
                      f"{name}_backward, and torch.no_grad() or detach() here", stacklevel=3)


_ACTIVATIONS = {"silu": GNN_SILU, "gelu": GNN_GELU, "sigmoid": GNN_SIGMOID, "relu": GNN_RELU}


def _elsewhere(what: str, t, stream):
    """(device of t, context to run the call in): None where the call may run as
    it is, on the current stream of the current device."""
    dev = _device(what, t)
    if stream is None and dev.index == torch.cuda.current_device():
        return dev, None
    return dev, _on(dev, torch.cuda.current_stream(dev) if stream is None else stream)


def _like(what: str, x: torch.Tensor, width: int, out, device):
    """A table of x's type and number of rows, new if none is given; (table, address,
    stride)."""
    if out is None:
        out = torch.empty(x.shape[0], width, dtype=x.dtype, device=device)
        return out, out.data_ptr(), width
    a, t, s = _rows(what, out, width, x.shape[0], device)
    if out.dtype != x.dtype:
        raise TypeError(f"{what}: expected {x.dtype}, got {out.dtype}")
    return out, a, s


def _float_rows(what: str, t, width=None, n=None, device=None):
    a, kind, s = _rows(what, t, width, n, device)
    if kind == GNN_INT8:
        raise TypeError(f"{what}: expected rows of a float type")
    return a, kind, s


def layer_norm(x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, eps: float = 1e-5,
               out=None, save: bool = False, stream=None):
    """The layer norm of x's rows, of x's type; with ``save`` (y, mean, rstd), which
    ``layer_norm_backward`` takes.  gamma, beta: fp32.  ``out`` may be x.  No autograd graph
    is recorded."""
    dev, where = _elsewhere("x", x, stream)
    if where is not None:
        with where:
            return layer_norm(x, gamma, beta, eps, out, save)
    xa, xt, xs = _float_rows("x", x, None, None, dev)
    n, k = x.shape
    ga = _vector("gamma", gamma, torch.float32, k, dev)
    ba = _vector("beta", beta, torch.float32, k, dev)
    _no_graph("layer_norm", x, gamma, beta)
    out, ya, ys = _like("out", x, k, out, dev)
    mean = rstd = None
    if save:
        mean, rstd = torch.empty(2, n, dtype=torch.float32, device=dev).unbind(0)
    _check(lib.gnn_layer_norm(xa, xt, xs, n, k, ga, ba, eps, ya, ys, _addr(mean), _addr(rstd),
                              _raw_stream(dev.index)))
    return (out, mean, rstd) if save else out


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, gamma: torch.Tensor,
                        mean: torch.Tensor, rstd: torch.Tensor, out=None, stream=None):
    """(dx, dgamma, dbeta) from dy and what ``layer_norm`` saved; ``out``: the dx to
    fill, which may be dy."""
    dev, where = _elsewhere("x", x, stream)
    if where is not None:
        with where:
            return layer_norm_backward(dy, x, gamma, mean, rstd, out)
    xa, xt, xs = _float_rows("x", x, None, None, dev)
    n, k = x.shape
    da, dt, ds = _float_rows("dy", dy, k, n, dev)
    if dt != xt:
        raise TypeError(f"dy: expected {x.dtype}, got {dy.dtype}")
    ga = _vector("gamma", gamma, torch.float32, k, dev)
    ma = _vector("mean", mean, torch.float32, n, dev)
    ra = _vector("rstd", rstd, torch.float32, n, dev)
    out, oa, os_ = _like("out", x, k, out, dev)
    dgamma, dbeta = torch.empty(2, k, dtype=torch.float32, device=dev).unbind(0)
    nb = lib.gnn_layer_norm_workspace(n, k)
    ws = _scratch(nb, dev)
    _check(lib.gnn_layer_norm_backward(da, ds, xa, xs, xt, n, k, ga, ma, ra, oa, os_,
                                       dgamma.data_ptr(), dbeta.data_ptr(), _addr(ws), nb,
                                       _raw_stream(dev.index)))
    return out, dgamma, dbeta


def _gated_args(x, w_gate, w_up, w_down, biases, activation, dev):
    """(dims, weights, address and stride of x, the three biases, whether everything is
    aligned)."""
    xa, xt, xs = _rows("x", x, None, None, dev)
    if xt not in (GNN_BF16, GNN_F16):
        raise TypeError(f"x: rows of {x.dtype} are not supported, bfloat16 and float16 are")
    act = _ACTIVATIONS.get(activation)
    if act is None:
        raise ValueError(f"activation: {activation!r} is none of {', '.join(_ACTIVATIONS)}")
    k = x.shape[1]
    for what, w in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        if not isinstance(w, torch.Tensor) or w.dim() != 2 or w.dtype != x.dtype:
            raise TypeError(f"{what}: expected a 2-D tensor of {x.dtype}")
        if not w.is_contiguous() or w.device != dev:
            raise ValueError(f"{what}: expected a contiguous tensor on {dev}")
    hidden, n_out = w_gate.shape[0], w_down.shape[0]
    for what, w, shape in (("w_gate", w_gate, (hidden, k)), ("w_up", w_up, (hidden, k)),
                           ("w_down", w_down, (n_out, hidden))):
        if tuple(w.shape) != shape:
            raise ValueError(f"{what}: expected shape {shape}, got {tuple(w.shape)}")
    b = (None, None, None) if biases is None else tuple(biases)
    if len(b) != 3:
        raise ValueError("biases: expected three, of gate, up and down (some may be None)")
    ba = [_vector(what, v, x.dtype, n, dev) for what, v, n in
          zip(("gate bias", "up bias", "down bias"), b, (hidden, hidden, n_out))]
    dims = make_gated_dims(k, hidden, n_out, xt, act)
    ptrs = (w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr())
    weights = gnn_gated_weights(ctypes.sizeof(gnn_gated_weights), *ptrs, *ba)
    return dims, weights, xa, xs, b, _lies_aligned(xa, xs) and all(p % 16 == 0 for p in ptrs)


def _lies_aligned(address: int, stride: int) -> bool:
    return address % 16 == 0 and stride % 8 == 0 and stride <= 1 << 21


def gated(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
          biases=None, activation: str = "silu", out=None, stream=None) -> torch.Tensor:
    """A gated feed-forward block: act(x w_gate^T + b) * (x w_up^T + b) through w_down.
    Rows, weights and biases (of gate, up and down) bfloat16 or float16; activation
    "silu", "gelu", "sigmoid" or "relu".  No autograd graph is recorded
    (``gated_backward``)."""
    dev, where = _elsewhere("x", x, stream)
    if where is not None:
        with where:
            return gated(x, w_gate, w_up, w_down, biases, activation, out)
    dims, weights, xa, xs, biases, aligned = _gated_args(x, w_gate, w_up, w_down, biases,
                                                         activation, dev)
    _no_graph("gated", x, w_gate, w_up, w_down, *biases)
    n = x.shape[0]
    out, ya, ys = _like("out", x, dims.out_features, out, dev)
    nb = lib.gnn_gated_workspace(dims, n, 0, aligned)
    ws = _scratch(nb, dev)
    _check(lib.gnn_gated(dims, weights, xa, xs, n, ya, ys, _addr(ws), nb, _raw_stream(dev.index)))
    return out


def gated_backward(dy: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
                   w_down: torch.Tensor, biases=None, activation: str = "silu", out=None,
                   stream=None):
    """(dx, dw_gate, dw_up, dw_down, db_gate, db_up, db_down) of ``gated`` from dy;
    None for biases that are None.  ``out``: the dx to fill."""
    dev, where = _elsewhere("x", x, stream)
    if where is not None:
        with where:
            return gated_backward(dy, x, w_gate, w_up, w_down, biases, activation, out)
    dims, weights, xa, xs, biases, aligned = _gated_args(x, w_gate, w_up, w_down, biases,
                                                         activation, dev)
    n = x.shape[0]
    da, dt, ds = _rows("dy", dy, dims.out_features, n, dev)
    if dt != dims.dtype:
        raise TypeError(f"dy: expected {x.dtype}, got {dy.dtype}")
    out, oa, os_ = _like("out", x, dims.in_features, out, dev)
    grads = [torch.empty_like(w) for w in (w_gate, w_up, w_down)]
    grads += [None if b is None else torch.empty_like(b) for b in biases]
    into = gnn_gated_weights(ctypes.sizeof(gnn_gated_weights), *map(_addr, grads))
    nb = lib.gnn_gated_workspace(dims, n, 1, aligned and _lies_aligned(da, ds))
    ws = _scratch(nb, dev)
    _check(lib.gnn_gated_backward(dims, weights, da, ds, xa, xs, n, oa, os_, into, _addr(ws), nb,
                                  _raw_stream(dev.index)))
    return (out, *grads)


def gnn_debug_gated(dims: gnn_gated_dims, n_cu: int, n_rows: int, backward=False) -> tuple:
    """The C call's kernel[0 .. 6]."""
    k = (ctypes.c_int32 * 7)()
    _check(lib.gnn_debug_gated(dims, n_cu, n_rows, int(backward), k))
    return tuple(k)


_FLOATS = frozenset((torch.float32, torch.bfloat16, torch.float16))
_GRAD = np.dtype([("grad", np.uint64), ("out", np.uint64), ("count", np.int64),
                  ("type", np.int32), ("reserved", np.int32)])


def clip_grads(grads, max_norm: float, out=None, stream=None) -> torch.Tensor:
    """The global norm of the gradients (a 0-dim fp32 tensor on their device), which
    are scaled by min(1, max_norm / (norm + 1e-6)): in place, or into ``out``, a
    tensor of the same size and type for each.  Contiguous fp32, bfloat16 and
    float16 tensors, side by side in any mixture."""
    grads = list(grads)
    out = grads if out is None else list(out)
    if not grads:
        raise ValueError("grads: expected one tensor at least")
    dev, where = _elsewhere("grads", grads[0], stream)
    if where is not None:
        with where:
            return clip_grads(grads, max_norm, out)
    if len(out) != len(grads):
        raise ValueError(f"out: {len(out)} tensors, expected {len(grads)}")
    # a step has hundreds of tensors: whole lists at a time
    listed = (("grads", grads),) if out is grads else (("out", out), ("grads", grads))
    for what, ts in listed:
        if not all([isinstance(t, torch.Tensor) for t in ts]):
            raise TypeError(f"{what}: expected tensors")
        kinds = [t.dtype for t in ts]
        if not _FLOATS.issuperset(kinds):
            raise TypeError(f"{what}: expected float32, bfloat16 and float16 tensors")
        if {t.get_device() for t in ts} != {dev.index} or not all([t.is_contiguous() for t in ts]):
            raise ValueError(f"{what}: expected contiguous tensors on {dev}")
    table = np.zeros(len(grads), _GRAD)
    table["grad"] = [t.data_ptr() for t in grads]
    table["count"] = counts = [t.numel() for t in grads]
    table["type"] = [_TYPES[k] for k in kinds]
    if out is grads:
        table["out"] = table["grad"]
    else:
        if [t.numel() for t in out] != counts or [t.dtype for t in out] != kinds:
            raise ValueError("out: expected tensors of the gradients' sizes and types")
        table["out"] = [t.data_ptr() for t in out]
    norm = torch.empty((), dtype=torch.float32, device=dev)
    nb = lib.gnn_clip_workspace(table.ctypes.data, len(grads))
    ws = _scratch(nb, dev)
    _check(lib.gnn_clip_grads(table.ctypes.data, len(grads), max_norm, norm.data_ptr(), _addr(ws),
                              nb, _raw_stream(dev.index)))
    return norm


def gnn_server_create(handle, n_instances: int):
    s = lib.gnn_server_create(handle, int(n_instances))
    if not s:
        raise GnnError(GNN_E_INVALID_ARG, gnn_last_error())
    return s


def gnn_server_submit(server, node_feat, edge_index, n_nodes: int, n_edges: int,
                      edge_scores) -> int:
    """Queue one event; returns the request id."""
    _check_io(node_feat, edge_index, edge_scores)
    rid = lib.gnn_server_submit(server, _addr(node_feat), _addr(edge_index), n_nodes, n_edges,
                                _addr(edge_scores))
    if rid < 0:
        raise GnnError(int(rid), gnn_last_error())
    return int(rid)


def gnn_server_wait(server, request_id: int) -> float:
    """Wait for one request; returns its latency (ms, queueing included)."""
    lat = ctypes.c_double(0.0)
    _check(lib.gnn_server_wait(server, int(request_id), ctypes.byref(lat)))
    return lat.value


def gnn_server_wait_info(server, request_id: int) -> dict:
    """Wait for one request; returns its status, latency and device interval (ms)."""
    info = gnn_request_info(ctypes.sizeof(gnn_request_info), 0, 0.0, -1.0, -1.0)
    _check(lib.gnn_server_wait_info(server, int(request_id), ctypes.byref(info)))
    return {"status": info.status, "latency_ms": info.latency_ms,
            "device_start_ms": info.device_start_ms, "device_end_ms": info.device_end_ms}


def gnn_server_destroy(server) -> None:
    lib.gnn_server_destroy(server)


class Server:
    """A request queue served by ``n_instances`` streams of one model."""

    def __init__(self, model: "Model", n_instances: int):
        self.model = model
        self.server = gnn_server_create(model.handle, n_instances)

    def submit(self, x: torch.Tensor, edge_index: torch.Tensor, out: torch.Tensor) -> int:
        return gnn_server_submit(self.server, x, edge_index, x.shape[0], edge_index.shape[1], out)

    def wait(self, request_id: int) -> float:
        return gnn_server_wait(self.server, request_id)

    def wait_info(self, request_id: int) -> dict:
        return gnn_server_wait_info(self.server, request_id)

    def close(self):
        if self.server:
            gnn_server_destroy(self.server)
            self.server = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Model:
    """Owns one handle: ``Model(weights, dims)(x, edge_index) -> scores``."""

    def __init__(self, weights: np.ndarray, dims: gnn_dims):
        self.dims = dims
        self.handle = gnn_create(weights, dims)

    def __call__(self, x: torch.Tensor, edge_index: torch.Tensor, out=None, logits=False,
                 stream=None) -> torch.Tensor:
        E = edge_index.shape[1]
        if out is None:
            out = torch.empty(E, dtype=torch.float32, device=x.device)
        f = gnn_infer_logits if logits else gnn_infer
        f(self.handle, x, edge_index, x.shape[0], E, out, stream)
        return out

    def close(self):
        if self.handle:
            gnn_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
