"""Thin Python binding of libtfg (the C ABI in include/tfg.h).

Argument marshalling only: it checks tensor devices, dtypes and shapes,
allocates output and workspace tensors with PyTorch (device memory), passes
raw pointers and the current CUDA stream, and turns error codes into
exceptions.  Every step of the computation runs in the CUDA kernels of
libtfg.so; there is no CPU fallback.  If the library has not been built, the
first call raises.

Function names follow the ABI (``tfg_build_csr`` ...).  All tensors must be
CUDA tensors on the same device; calls are asynchronous on the current stream.
"""
from __future__ import annotations

import array
import ctypes
import math
import operator
import os
import threading
from typing import NamedTuple, Optional

import torch

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtfg.so")

TFG_OK = 0
TFG_ERR_INVALID_ARG = -1
TFG_ERR_TOO_LARGE = -2
TFG_ERR_WORKSPACE = -3
TFG_ERR_CUDA = -4
TFG_ERR_INDEX_RANGE = -5
TFG_ERR_UNSORTED = -6
TFG_ERR_TIMEOUT = -7
TFG_F32, TFG_BF16 = 0, 1
REDUCERS = {"sum": 0, "mean": 1, "max": 2}
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
NO_PADDING = -(1 << 63)       # padding_id of a list without padding

_lock = threading.Lock()
_lib: Optional[ctypes.CDLL] = None


class TfgError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libtfg error {code}: {message}")
        self.code = code


def lib() -> ctypes.CDLL:
    """Load libtfg.so (once).  Raises if it has not been built."""
    global _lib
    with _lock:
        if _lib is None:
            _lib = _load(LIB_PATH)
        return _lib


def use_library(path: str) -> ctypes.CDLL:
    """Switch every call of this module to another build of the library (for
    example the bounds-checked debug build, ``build.build_library(defines=
    ("TFG_CHECK_BOUNDS=1",), lib_path=...)``); returns the loaded library."""
    global _lib
    with _lock:
        _lib = _load(path)
        return _lib


def _load(path: str) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} is missing: build it first (python -m paper_2101_11552_gb300.build "
            "or __graft_entry__.build()); there is no CPU fallback")
    L = ctypes.CDLL(path)
    P, I64, I, F, SZ = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float,
                        ctypes.c_size_t)
    sigs = {
        "tfg_version": [],
        "tfg_check_bounds_enabled": [],
        "tfg_build_csr_workspace_size": [I64, I64, ctypes.POINTER(SZ)],
        "tfg_build_csr": [P, I64, I64, P, P, P, P, P, SZ, P, P],
        "tfg_build_csr_by_source": [P, I64, I64, P, P, P, P, P, SZ, P, P],
        "tfg_build_csr32": [P, I64, I64, P, P, P, P, P, SZ, P, P],
        "tfg_build_csr32_by_source": [P, I64, I64, P, P, P, P, P, SZ, P, P],
        "tfg_aggregate_backward_workspace_size": [I, I64, ctypes.POINTER(SZ)],
        "tfg_aggregate_backward": [I, P, P, P, P, P, P, I64, I64, I64, P, P, SZ, P],
        "tfg_gcn_aggregate_backward": [P, P, P, P, I64, I64, I, F, P, P],
        "tfg_aggregate_max_argmax": [P, P, P, P, P, I, I64, I64, P, P, P],
        "tfg_aggregate_max_backward_workspace_size": [I64, I64, I64, ctypes.POINTER(SZ)],
        "tfg_aggregate_max_backward": [P, P, P, P, P, P, I64, I64, I64, P, P, SZ, P],
        "tfg_gcn_norm": [P, P, P, P, I64, I64, I, F, P, P, P],
        "tfg_aggregate_sum": [P, P, P, P, I, I64, I64, P, P],
        "tfg_aggregate_mean": [P, P, P, P, I, I64, I64, P, P],
        "tfg_aggregate_max": [P, P, P, P, I, I64, I64, P, P],
        "tfg_gcn_aggregate_sum": [P, P, P, P, P, I, I64, I64, I, F, P, P],
        "tfg_propagate_workspace_size": [I64, I64, I64, ctypes.POINTER(SZ)],
        "tfg_appnp_propagate": [P, P, P, P, P, I, I64, I64, I64, F, I, F, P, P, SZ, P],
        "tfg_sgc_propagate": [P, P, P, P, P, I, I64, I64, I64, I, F, P, P, SZ, P],
        "tfg_edge_softmax_workspace_size": [I64, I, ctypes.POINTER(SZ)],
        "tfg_edge_softmax_aggregate": [P, P, P, I, I64, I64, I, I, P, P, F, P, P, P, SZ, P],
        "tfg_dot_edge_softmax_aggregate": [P, P, P, P, P, I, I64, I64, I, I, F, P, P, P],
        "tfg_edge_softmax_aggregate_noalloc": [P, P, P, I, I64, I64, I, I, P, P, F, P, P, P],
        "tfg_segment_pool": [P, I, P, I64, I64, I64, I, P, P, P],
        "tfg_segment_pool_meanmax": [P, I, P, I64, I64, I64, P, P, P],
        "tfg_batch_graphs_workspace_size": [I64, ctypes.POINTER(SZ)],
        "tfg_batch_graphs": [I64, P, P, P, I64, I64, P, P, P, P, SZ, P, P],
        "tfg_gather_xor": [P, I64, P, I64, I64, P, P],
        "tfg_embedding_lookup": [P, I64, P, I, I64, I64, F, I64, P, I, P, P],
        "tfg_embedding_lookup32": [P, I64, P, I, I64, I64, F, I64, P, I, P, P],
        "tfg_group_ids_workspace_size": [I64, I64, ctypes.POINTER(SZ)],
        "tfg_group_ids": [P, I64, I64, I64, P, P, P, P, SZ, P, P],
        "tfg_group_ids32": [P, I64, I64, I64, P, P, P, P, SZ, P, P],
        "tfg_embedding_backward_workspace_size": [I64, ctypes.POINTER(SZ)],
        "tfg_embedding_backward": [P, P, P, P, I, I64, I64, I64, F, P, P, SZ, P],
        "tfg_group_norm_workspace_size": [I64, I64, I64, I64, ctypes.POINTER(SZ)],
        "tfg_group_norm": [P, I, P, I64, I64, I64, I64, P, P, F, I, P, I, P, P, P, SZ, P, P],
        "tfg_group_norm_backward_workspace_size": [I64, I64, I64, I64, ctypes.POINTER(SZ)],
        "tfg_group_norm_backward": [P, I, P, I64, I64, I64, I64, P, P, P, P, I, P, I, P, P, P, P, SZ, P],
        "tfg_global_norm_workspace_size": [I64, ctypes.POINTER(SZ)],
        "tfg_global_norm": [I64, P, P, P, P, P, SZ, P],
        "tfg_clip_by_global_norm": [I64, P, P, P, F, P, P, P, SZ, P],
        "tfg_edge_softmax_backward_workspace_size": [I64, I, I, ctypes.POINTER(SZ)],
        "tfg_edge_softmax_aggregate_backward": [P, P, P, P, P, I, I64, I64, I, I, P, P, F,
                                                P, P, P, P, P, P, SZ, P],
        "tfg_dot_edge_softmax_backward_workspace_size": [I64, I, I, ctypes.POINTER(SZ)],
        "tfg_dot_edge_softmax_aggregate_backward": [P, P, P, P, P, P, P, I, I64, I64, I, I,
                                                    F, P, P, P, P, P, P, SZ, P],
    }
    for name, args in sigs.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    L.tfg_last_error.argtypes = []
    L.tfg_last_error.restype = ctypes.c_char_p
    return L


def tfg_version() -> int:
    return lib().tfg_version()


def tfg_last_error() -> str:
    return lib().tfg_last_error().decode()


def _check(rc: int):
    if rc != TFG_OK:
        raise TfgError(rc, tfg_last_error())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device: torch.device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _need_cuda(name: str, t: torch.Tensor, dtype=None, device=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")


def _x_dtype(x: torch.Tensor) -> int:
    if x.dtype == torch.float32:
        return TFG_F32
    if x.dtype == torch.bfloat16:
        return TFG_BF16
    raise ValueError(f"features must be float32 or bfloat16, got {x.dtype}")


class CSR(NamedTuple):
    rowptr: torch.Tensor     # int32 [N + 1]
    col: torch.Tensor        # int32 [E]
    perm: torch.Tensor       # int32 [E]
    in_degree: torch.Tensor  # int32 [N]
    status: torch.Tensor     # int32 [1] (device)


def check_status(status: torch.Tensor):
    """Synchronise on the status word and raise if a kernel flagged bad input."""
    code = int(status.item())
    if code != 0:
        raise TfgError(code, "device-side validation failed "
                             f"({'index out of range' if code == TFG_ERR_INDEX_RANGE else 'unsorted batch'})")


def tfg_build_csr_workspace_size(num_nodes: int, num_edges: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().tfg_build_csr_workspace_size(num_nodes, num_edges, ctypes.byref(n)))
    return n.value


def tfg_build_csr(edge_index: torch.Tensor, num_nodes: int,
                  workspace: Optional[torch.Tensor] = None) -> CSR:
    """Group the edges of ``edge_index`` (int64 or int32 [2, E]) by target node."""
    _need_cuda("edge_index", edge_index, None)
    if edge_index.dtype not in (torch.int64, torch.int32):
        raise TypeError("edge_index must be int64 or int32")
    if edge_index.dim() != 2 or edge_index.shape[0] != 2:
        raise ValueError("edge_index must have shape [2, E]")
    dev = edge_index.device
    e = edge_index.shape[1]
    rowptr = torch.empty(num_nodes + 1, dtype=torch.int32, device=dev)
    col = torch.empty(e, dtype=torch.int32, device=dev)
    perm = torch.empty(e, dtype=torch.int32, device=dev)
    deg = torch.empty(num_nodes, dtype=torch.int32, device=dev)
    status = torch.empty(1, dtype=torch.int32, device=dev)
    need = tfg_build_csr_workspace_size(num_nodes, e)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    fn = lib().tfg_build_csr32 if edge_index.dtype == torch.int32 else lib().tfg_build_csr
    _check(fn(_ptr(edge_index), e, num_nodes, _ptr(rowptr), _ptr(col), _ptr(perm), _ptr(deg),
              _ptr(workspace), workspace.numel(), _ptr(status), _stream(dev)))
    return CSR(rowptr, col, perm, deg, status)


def tfg_build_csr_by_source(edge_index: torch.Tensor, num_nodes: int,
                            workspace: Optional[torch.Tensor] = None) -> CSR:
    """Group the edges by SOURCE (the transposed graph's CSR).  Returns the CSR
    tuple with rowptr over sources, col = targets, perm = original edge ids,
    in_degree = out-degrees."""
    _need_cuda("edge_index", edge_index, None)
    if edge_index.dtype not in (torch.int64, torch.int32):
        raise TypeError("edge_index must be int64 or int32")
    if edge_index.dim() != 2 or edge_index.shape[0] != 2:
        raise ValueError("edge_index must have shape [2, E]")
    dev = edge_index.device
    e = edge_index.shape[1]
    rowptr = torch.empty(num_nodes + 1, dtype=torch.int32, device=dev)
    col = torch.empty(e, dtype=torch.int32, device=dev)
    perm = torch.empty(e, dtype=torch.int32, device=dev)
    deg = torch.empty(num_nodes, dtype=torch.int32, device=dev)
    status = torch.empty(1, dtype=torch.int32, device=dev)
    need = tfg_build_csr_workspace_size(num_nodes, e)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    fn = (lib().tfg_build_csr32_by_source if edge_index.dtype == torch.int32
          else lib().tfg_build_csr_by_source)
    _check(fn(_ptr(edge_index), e, num_nodes, _ptr(rowptr), _ptr(col), _ptr(perm), _ptr(deg),
              _ptr(workspace), workspace.numel(), _ptr(status), _stream(dev)))
    return CSR(rowptr, col, perm, deg, status)


def tfg_aggregate_backward(reduce: str, csr_src: CSR, grad_out, edge_weight=None, in_degree=None,
                           out=None):
    """grad_x of tfg_aggregate_sum / _mean: the sum over the transposed graph
    (csr_src from tfg_build_csr_by_source; edge_weight in original order; the
    forward CSR's in_degree for the mean)."""
    _need_cuda("grad_out", grad_out, torch.float32)
    dev = grad_out.device
    n, f = grad_out.shape
    e = csr_src.col.numel()
    code = REDUCERS[reduce]
    nb = ctypes.c_size_t(0)
    _check(lib().tfg_aggregate_backward_workspace_size(code, e, ctypes.byref(nb)))
    ws = torch.empty(max(nb.value, 1), dtype=torch.uint8, device=dev)
    if out is None:
        out = torch.empty(n, f, dtype=torch.float32, device=dev)
    _check(lib().tfg_aggregate_backward(code, _ptr(csr_src.rowptr), _ptr(csr_src.col), _ptr(csr_src.perm),
                                        _ptr(edge_weight), _ptr(in_degree), _ptr(grad_out), n, e, f,
                                        _ptr(out), _ptr(ws), ws.numel(), _stream(dev)))
    return out


def tfg_gcn_aggregate_backward(csr_src: CSR, dinv, grad_out, add_self_loops: int = 0,
                               self_loop_fill: float = 1.0, out=None):
    """grad_x of tfg_gcn_aggregate_sum (on-the-fly weights), with the forward's dinv."""
    _need_cuda("grad_out", grad_out, torch.float32)
    dev = grad_out.device
    n, f = grad_out.shape
    if out is None:
        out = torch.empty(n, f, dtype=torch.float32, device=dev)
    _check(lib().tfg_gcn_aggregate_backward(_ptr(csr_src.rowptr), _ptr(csr_src.col), _ptr(dinv),
                                            _ptr(grad_out), n, f, int(add_self_loops),
                                            float(self_loop_fill), _ptr(out), _stream(dev)))
    return out


def tfg_aggregate_max_argmax(csr: CSR, x, w_csr=None):
    """(out, argmax): the max aggregation and, per (t, f), the original id of
    the first edge attaining it (-1 for a row without edges)."""
    _need_cuda("x", x)
    dev = x.device
    n, f = x.shape
    out = torch.empty(n, f, dtype=torch.float32, device=dev)
    arg = torch.empty(n, f, dtype=torch.int32, device=dev)
    _check(lib().tfg_aggregate_max_argmax(_ptr(csr.rowptr), _ptr(csr.col), _ptr(csr.perm), _ptr(w_csr),
                                          _ptr(x), _x_dtype(x), n, f, _ptr(out), _ptr(arg), _stream(dev)))
    return out, arg


def tfg_aggregate_max_backward_workspace_size(num_nodes: int, num_edges: int,
                                              num_features: int) -> int:
    nb = ctypes.c_size_t(0)
    _check(lib().tfg_aggregate_max_backward_workspace_size(num_nodes, num_edges, num_features,
                                                           ctypes.byref(nb)))
    return nb.value


def tfg_aggregate_max_backward(csr_src: CSR, argmax, grad_out, edge_weight=None, out=None,
                               marks: bool = True):
    """grad_x of the max: w_e grad_out[t, f] to the source of the edge argmax[t, f]
    (edge_weight in original edge order, or None).  marks=False runs without the
    win-mark workspace (every out-edge's rows read; the same result)."""
    _need_cuda("grad_out", grad_out, torch.float32)
    dev = grad_out.device
    n, f = grad_out.shape
    e = csr_src.col.numel()
    ws = None
    nb = tfg_aggregate_max_backward_workspace_size(n, e, f) if marks else 0
    if nb > 0:
        ws = torch.empty(nb, dtype=torch.uint8, device=dev)
    if out is None:
        out = torch.empty(n, f, dtype=torch.float32, device=dev)
    _check(lib().tfg_aggregate_max_backward(_ptr(csr_src.rowptr), _ptr(csr_src.col), _ptr(csr_src.perm),
                                            _ptr(argmax), _ptr(edge_weight), _ptr(grad_out), n, e, f,
                                            _ptr(out), _ptr(ws), ws.numel() if ws is not None else 0,
                                            _stream(dev)))
    return out


def tfg_gcn_norm(rowptr: torch.Tensor, col: torch.Tensor, perm: torch.Tensor, num_nodes: int,
                 edge_weight: Optional[torch.Tensor] = None, add_self_loops: int = 0,
                 self_loop_fill: float = 1.0, want_w_csr: bool = True):
    """Return (dinv [N], w_csr [E] or None) of the GCN normalisation of A + I."""
    _need_cuda("rowptr", rowptr, torch.int32)
    dev = rowptr.device
    e = col.numel()
    if edge_weight is not None:
        _need_cuda("edge_weight", edge_weight, torch.float32, dev)
    dinv = torch.empty(num_nodes, dtype=torch.float32, device=dev)
    w_csr = torch.empty(e, dtype=torch.float32, device=dev) if want_w_csr else None
    _check(lib().tfg_gcn_norm(_ptr(rowptr), _ptr(col), _ptr(perm), _ptr(edge_weight), num_nodes, e,
                              int(add_self_loops), float(self_loop_fill), _ptr(dinv), _ptr(w_csr),
                              _stream(dev)))
    return dinv, w_csr


def _aggregate(fn_name: str, rowptr, col, x, w_csr, out):
    _need_cuda("rowptr", rowptr, torch.int32)
    dev = rowptr.device
    _need_cuda("col", col, torch.int32, dev)
    _need_cuda("x", x, None, dev)
    n, f = x.shape
    if rowptr.numel() != n + 1:
        raise ValueError("rowptr must have N + 1 entries")
    if w_csr is not None:
        _need_cuda("w_csr", w_csr, torch.float32, dev)
    if out is None:
        out = torch.empty(n, f, dtype=torch.float32, device=dev)
    _need_cuda("out", out, torch.float32, dev)
    _check(getattr(lib(), fn_name)(_ptr(rowptr), _ptr(col), _ptr(w_csr), _ptr(x), _x_dtype(x), n, f,
                                   _ptr(out), _stream(dev)))
    return out


def tfg_aggregate_sum(rowptr, col, x, w_csr=None, out=None):
    return _aggregate("tfg_aggregate_sum", rowptr, col, x, w_csr, out)


def tfg_aggregate_mean(rowptr, col, x, w_csr=None, out=None):
    return _aggregate("tfg_aggregate_mean", rowptr, col, x, w_csr, out)


def tfg_aggregate_max(rowptr, col, x, w_csr=None, out=None):
    return _aggregate("tfg_aggregate_max", rowptr, col, x, w_csr, out)


def tfg_gcn_aggregate_sum(rowptr, col, dinv, x, w_csr=None, add_self_loops: int = 0,
                          self_loop_fill: float = 1.0, out=None):
    _need_cuda("rowptr", rowptr, torch.int32)
    dev = rowptr.device
    _need_cuda("col", col, torch.int32, dev)
    _need_cuda("dinv", dinv, torch.float32, dev)
    _need_cuda("x", x, None, dev)
    n, f = x.shape
    if rowptr.numel() != n + 1:
        raise ValueError("rowptr must have N + 1 entries")
    if w_csr is not None:
        _need_cuda("w_csr", w_csr, torch.float32, dev)
    if out is None:
        out = torch.empty(n, f, dtype=torch.float32, device=dev)
    _need_cuda("out", out, torch.float32, dev)
    _check(lib().tfg_gcn_aggregate_sum(_ptr(rowptr), _ptr(col), _ptr(dinv), _ptr(w_csr), _ptr(x),
                                       _x_dtype(x), n, f, int(add_self_loops),
                                       float(self_loop_fill), _ptr(out), _stream(dev)))
    return out


def tfg_propagate_workspace_size(num_nodes: int, num_features: int, num_hops: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().tfg_propagate_workspace_size(num_nodes, num_features, num_hops, ctypes.byref(n)))
    return n.value


def tfg_appnp_propagate(rowptr, col, dinv, x0, num_hops: int, alpha: float, w_csr=None,
                        add_self_loops: int = 0, self_loop_fill: float = 1.0, out=None,
                        workspace=None):
    """h_{k+1} = (1 - alpha) Ahat h_k + alpha x0, h_0 = x0; returns h_K (fp32)."""
    return _propagate("tfg_appnp_propagate", rowptr, col, dinv, x0, num_hops, alpha, w_csr,
                      add_self_loops, self_loop_fill, out, workspace)


def tfg_sgc_propagate(rowptr, col, dinv, x0, num_hops: int, w_csr=None, add_self_loops: int = 0,
                      self_loop_fill: float = 1.0, out=None, workspace=None):
    """Ahat^K x0 (fp32)."""
    return _propagate("tfg_sgc_propagate", rowptr, col, dinv, x0, num_hops, None, w_csr,
                      add_self_loops, self_loop_fill, out, workspace)


def _propagate(name, rowptr, col, dinv, x0, num_hops, alpha, w_csr, add_self_loops,
               self_loop_fill, out, workspace):
    _need_cuda("rowptr", rowptr, torch.int32)
    dev = rowptr.device
    _need_cuda("col", col, torch.int32, dev)
    _need_cuda("dinv", dinv, torch.float32, dev)
    _need_cuda("x0", x0, None, dev)
    n, f = x0.shape
    if rowptr.numel() != n + 1:
        raise ValueError("rowptr must have N + 1 entries")
    if w_csr is not None:
        _need_cuda("w_csr", w_csr, torch.float32, dev)
    if out is None:
        out = torch.empty(n, f, dtype=torch.float32, device=dev)
    _need_cuda("out", out, torch.float32, dev)
    nb = tfg_propagate_workspace_size(n, f, num_hops)
    if workspace is None or workspace.numel() < nb:
        workspace = torch.empty(max(nb, 1), dtype=torch.uint8, device=dev)
    head = [_ptr(rowptr), _ptr(col), _ptr(dinv), _ptr(w_csr), _ptr(x0), _x_dtype(x0), n, f,
            int(num_hops)]
    tail = [int(add_self_loops), float(self_loop_fill), _ptr(out), _ptr(workspace),
            workspace.numel(), _stream(dev)]
    fn = getattr(lib(), name)
    _check(fn(*head, *([] if alpha is None else [float(alpha)]), *tail))
    return out


def tfg_edge_softmax_workspace_size(num_nodes: int, heads: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().tfg_edge_softmax_workspace_size(num_nodes, heads, ctypes.byref(n)))
    return n.value


def tfg_edge_softmax_aggregate(rowptr, col, x, heads: int, channels: int, a_src, a_dst,
                               negative_slope: float = 0.2, want_alpha: bool = False,
                               out=None, workspace=None):
    """Return (out [N, H*C], alpha [E, H] in CSR order or None)."""
    _need_cuda("rowptr", rowptr, torch.int32)
    dev = rowptr.device
    _need_cuda("col", col, torch.int32, dev)
    _need_cuda("x", x, None, dev)
    _need_cuda("a_src", a_src, torch.float32, dev)
    _need_cuda("a_dst", a_dst, torch.float32, dev)
    n, f = x.shape
    if f != heads * channels:
        raise ValueError("x must have heads * channels columns")
    e = col.numel()
    if out is None:
        out = torch.empty(n, f, dtype=torch.float32, device=dev)
    alpha = torch.empty(e, heads, dtype=torch.float32, device=dev) if want_alpha else None
    need = tfg_edge_softmax_workspace_size(n, heads)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    _check(lib().tfg_edge_softmax_aggregate(_ptr(rowptr), _ptr(col), _ptr(x), _x_dtype(x), n, e,
                                            heads, channels,
                                            _ptr(a_src), _ptr(a_dst), float(negative_slope),
                                            _ptr(out), _ptr(alpha), _ptr(workspace),
                                            workspace.numel(), _stream(dev)))
    return out, alpha


def tfg_dot_edge_softmax_aggregate(rowptr, col, q, k, v, heads: int, channels: int,
                                   scale: Optional[float] = None, want_alpha: bool = False,
                                   out=None, alpha=None):
    """Transformer-style attention over in-edges; scale defaults to 1/sqrt(channels).
    Returns (out [N, H*C] fp32, alpha [E, H] or None)."""
    _need_cuda("rowptr", rowptr, torch.int32)
    dev = rowptr.device
    _need_cuda("col", col, torch.int32, dev)
    _need_cuda("q", q, None, dev)
    _need_cuda("k", k, q.dtype, dev)
    _need_cuda("v", v, q.dtype, dev)
    n, f = q.shape
    if k.shape != q.shape or v.shape != q.shape:
        raise ValueError("q, k and v must have the same shape")
    if f != heads * channels:
        raise ValueError("feature width must equal heads * channels")
    e = col.numel()
    if scale is None:
        scale = 1.0 / math.sqrt(channels)
    if out is None:
        out = torch.empty(n, f, dtype=torch.float32, device=dev)
    if want_alpha and alpha is None:
        alpha = torch.empty(e, heads, dtype=torch.float32, device=dev)
    _check(lib().tfg_dot_edge_softmax_aggregate(
        _ptr(rowptr), _ptr(col), _ptr(q), _ptr(k), _ptr(v), _x_dtype(q), n, e, heads, channels,
        float(scale), _ptr(out), _ptr(alpha), _stream(dev)))
    return out, alpha


def tfg_edge_softmax_aggregate_noalloc(rowptr, col, x, heads: int, channels: int, a_src, a_dst,
                                       negative_slope: float = 0.2, out=None, alpha=None):
    """Edge-softmax aggregation through the entry point that allocates nothing.

    The library keeps the node scores in its own fixed device array, so the
    C call takes no workspace; ``out`` (and ``alpha`` if wanted) may be passed
    in preallocated so that nothing at all is allocated.  Returns
    (out, alpha)."""
    _need_cuda("rowptr", rowptr, torch.int32)
    dev = rowptr.device
    _need_cuda("col", col, torch.int32, dev)
    _need_cuda("x", x, None, dev)
    _need_cuda("a_src", a_src, torch.float32, dev)
    _need_cuda("a_dst", a_dst, torch.float32, dev)
    n, f = x.shape
    if f != heads * channels:
        raise ValueError("x must have heads * channels columns")
    if out is None:
        out = torch.empty(n, f, dtype=torch.float32, device=dev)
    _check(lib().tfg_edge_softmax_aggregate_noalloc(
        _ptr(rowptr), _ptr(col), _ptr(x), _x_dtype(x), n, col.numel(), heads, channels,
        _ptr(a_src), _ptr(a_dst), float(negative_slope), _ptr(out), _ptr(alpha), _stream(dev)))
    return out, alpha


def tfg_segment_pool(x, batch, num_graphs: int, reduce: str = "sum", out=None):
    """Return (out [G, F], status) -- status is the device status word."""
    _need_cuda("x", x)
    dev = x.device
    _need_cuda("batch", batch, torch.int64, dev)
    n, f = x.shape
    if out is None:
        out = torch.empty(num_graphs, f, dtype=torch.float32, device=dev)
    status = torch.empty(1, dtype=torch.int32, device=dev)
    _check(lib().tfg_segment_pool(_ptr(x), _x_dtype(x), _ptr(batch), n, num_graphs, f,
                                  REDUCERS[reduce], _ptr(out), _ptr(status), _stream(dev)))
    return out, status


def tfg_segment_pool_meanmax(x, batch, num_graphs: int, out=None):
    """Return (out [G, 2F] = [mean | max], status)."""
    _need_cuda("x", x)
    dev = x.device
    _need_cuda("batch", batch, torch.int64, dev)
    n, f = x.shape
    if out is None:
        out = torch.empty(num_graphs, 2 * f, dtype=torch.float32, device=dev)
    status = torch.empty(1, dtype=torch.int32, device=dev)
    _check(lib().tfg_segment_pool_meanmax(_ptr(x), _x_dtype(x), _ptr(batch), n, num_graphs, f,
                                          _ptr(out), _ptr(status), _stream(dev)))
    return out, status


def tfg_batch_graphs_workspace_size(num_graphs: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().tfg_batch_graphs_workspace_size(num_graphs, ctypes.byref(n)))
    return n.value


class BatchGraph(NamedTuple):
    edge_index: torch.Tensor    # int64 [2, E]
    batch: torch.Tensor         # int64 [N]
    node_offsets: torch.Tensor  # int64 [G + 1]
    status: torch.Tensor        # int32 [1] (device)


def tfg_batch_graphs(node_counts: torch.Tensor, edge_counts: torch.Tensor,
                     edge_index: torch.Tensor, total_nodes: int) -> BatchGraph:
    """Combine graphs into one BatchGraph on the device (reindexing trick)."""
    _need_cuda("node_counts", node_counts, torch.int64)
    dev = node_counts.device
    _need_cuda("edge_counts", edge_counts, torch.int64, dev)
    _need_cuda("edge_index", edge_index, torch.int64, dev)
    g = node_counts.numel()
    e = edge_index.shape[1]
    out_ei = torch.empty(2, e, dtype=torch.int64, device=dev)
    batch = torch.empty(total_nodes, dtype=torch.int64, device=dev)
    offs = torch.empty(g + 1, dtype=torch.int64, device=dev)
    status = torch.empty(1, dtype=torch.int32, device=dev)
    ws = torch.empty(tfg_batch_graphs_workspace_size(g), dtype=torch.uint8, device=dev)
    _check(lib().tfg_batch_graphs(g, _ptr(node_counts), _ptr(edge_counts), _ptr(edge_index), e,
                                  total_nodes, _ptr(out_ei), _ptr(batch), _ptr(offs), _ptr(ws),
                                  ws.numel(), _ptr(status), _stream(dev)))
    return BatchGraph(out_ei, batch, offs, status)


def tfg_gather_xor(col: torch.Tensor, x: torch.Tensor, out=None) -> torch.Tensor:
    """Gather-only floor: every row x[col[k]] read once and XOR-folded.
    Returns uint32 words as an int32 tensor [row_bytes / 4]."""
    _need_cuda("col", col, torch.int32)
    _need_cuda("x", x)
    dev = x.device
    row_bytes = x[0].numel() * x.element_size() if x.shape[0] else 16
    if out is None:
        out = torch.empty(row_bytes // 4, dtype=torch.int32, device=dev)
    _check(lib().tfg_gather_xor(_ptr(col), col.numel(), _ptr(x), x.shape[0], row_bytes, _ptr(out),
                                _stream(dev)))
    return out


def tfg_edge_softmax_backward_workspace_size(num_nodes: int, heads: int, channels: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().tfg_edge_softmax_backward_workspace_size(num_nodes, heads, channels,
                                                          ctypes.byref(n)))
    return n.value


def tfg_edge_softmax_aggregate_backward(rowptr, col, rowptr_src, col_src, x, heads: int,
                                        channels: int, a_src, a_dst, negative_slope: float,
                                        out, grad_out):
    """Gradients of tfg_edge_softmax_aggregate with respect to x, a_src and
    a_dst.  Returns (grad_x [N, H*C], grad_a_src [H*C], grad_a_dst [H*C])."""
    _need_cuda("x", x)
    dev = x.device
    for name, t, dt in (("rowptr", rowptr, torch.int32), ("col", col, torch.int32),
                        ("rowptr_src", rowptr_src, torch.int32), ("col_src", col_src, torch.int32),
                        ("a_src", a_src, torch.float32), ("a_dst", a_dst, torch.float32),
                        ("out", out, torch.float32), ("grad_out", grad_out, torch.float32)):
        _need_cuda(name, t, dt, dev)
    n = x.shape[0]
    f = heads * channels
    grad_x = torch.empty(n, f, dtype=torch.float32, device=dev)
    ga_src = torch.empty(f, dtype=torch.float32, device=dev)
    ga_dst = torch.empty(f, dtype=torch.float32, device=dev)
    ws = torch.empty(max(tfg_edge_softmax_backward_workspace_size(n, heads, channels), 1),
                     dtype=torch.uint8, device=dev)
    _check(lib().tfg_edge_softmax_aggregate_backward(
        _ptr(rowptr), _ptr(col), _ptr(rowptr_src), _ptr(col_src), _ptr(x), _x_dtype(x), n,
        col.numel(), heads, channels, _ptr(a_src), _ptr(a_dst), negative_slope, _ptr(out),
        _ptr(grad_out), _ptr(grad_x), _ptr(ga_src), _ptr(ga_dst), _ptr(ws), ws.numel(),
        _stream(dev)))
    return grad_x, ga_src, ga_dst


def tfg_dot_edge_softmax_backward_workspace_size(num_nodes: int, heads: int, channels: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().tfg_dot_edge_softmax_backward_workspace_size(num_nodes, heads, channels,
                                                              ctypes.byref(n)))
    return n.value


def tfg_dot_edge_softmax_aggregate_backward(rowptr, col, rowptr_src, col_src, q, k, v,
                                            heads: int, channels: int, scale: float, out,
                                            grad_out):
    """Gradients of tfg_dot_edge_softmax_aggregate with respect to q, k and v.
    Returns (grad_q, grad_k, grad_v), each [N, H*C] fp32."""
    _need_cuda("q", q)
    dev = q.device
    _need_cuda("k", k, q.dtype, dev)
    _need_cuda("v", v, q.dtype, dev)
    for name, t, dt in (("rowptr", rowptr, torch.int32), ("col", col, torch.int32),
                        ("rowptr_src", rowptr_src, torch.int32), ("col_src", col_src, torch.int32),
                        ("out", out, torch.float32), ("grad_out", grad_out, torch.float32)):
        _need_cuda(name, t, dt, dev)
    n = q.shape[0]
    f = heads * channels
    grads = [torch.empty(n, f, dtype=torch.float32, device=dev) for _ in range(3)]
    ws = torch.empty(max(tfg_dot_edge_softmax_backward_workspace_size(n, heads, channels), 1),
                     dtype=torch.uint8, device=dev)
    _check(lib().tfg_dot_edge_softmax_aggregate_backward(
        _ptr(rowptr), _ptr(col), _ptr(rowptr_src), _ptr(col_src), _ptr(q), _ptr(k), _ptr(v),
        _x_dtype(q), n, col.numel(), heads, channels, float(scale), _ptr(out), _ptr(grad_out),
        _ptr(grads[0]), _ptr(grads[1]), _ptr(grads[2]), _ptr(ws), ws.numel(), _stream(dev)))
    return tuple(grads)


# The calls below are often as short as a few microseconds on the device, so their host side
# is kept short too: pointers go to ctypes as integers, a tensor's device is compared by
# its index, and the current stream is taken as the raw handle.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_DTYPES = {torch.float32: TFG_F32, torch.bfloat16: TFG_BF16}
_IDS = {torch.int64: False, torch.int32: True}


def _run(index: int, name: str, *args):
    """Call the C entry point ``name`` on the current stream of device ``index``."""
    fn = getattr(_lib or lib(), name)
    if index == torch.cuda.current_device():
        rc = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            rc = fn(*args, _raw_stream(index))
    if rc != TFG_OK:
        raise TfgError(rc, tfg_last_error())


def _at(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _index(name: str, t: torch.Tensor) -> int:
    """The CUDA device index of a contiguous tensor."""
    try:
        index = t.get_device()
        if index >= 0 and t.is_contiguous():
            return index
    except AttributeError:                        # no tensor at all
        index = -1
    raise ValueError(f"{name} must be contiguous" if index >= 0 else f"{name} must be a CUDA tensor")


def _same(name: str, t: torch.Tensor, index: int, dtype=None):
    if _index(name, t) != index:
        raise ValueError(f"{name} is on {t.device}, expected cuda:{index}")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")


def _dtype_code(name: str, dtype: torch.dtype) -> int:
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"{name} must be float32 or bfloat16, got {dtype}")
    return code


def _workspace(workspace, need: int, like: torch.Tensor):
    """The caller's workspace, checked for its kind, or a new one on like's device (None for
    0 bytes)."""
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=like.device) if need else None
    _same("workspace", workspace, like.get_device(), torch.uint8)
    return workspace


def _span(workspace):
    return (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())


def _need_out(name: str, out, shape, dtype, like: torch.Tensor):
    """An output tensor: the caller's, which must be what would be allocated, or a new one."""
    if out is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    _same(name, out, like.get_device(), dtype)
    if out.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(out.shape)}")
    return out


def _need_ids(ids):
    """(device index, whether the ids are int32)."""
    index = _index("ids", ids)
    id32 = _IDS.get(ids.dtype)
    if id32 is None:
        raise TypeError("ids must be int64 or int32")
    return index, id32


def _padding(padding_id: Optional[int]) -> int:
    if padding_id is None:
        return NO_PADDING
    if not NO_PADDING <= padding_id < 1 << 63:    # ctypes would pass its lowest 64 bits
        raise ValueError(f"padding_id must be an int64, got {padding_id}")
    return padding_id


def _size(name: str, *args) -> int:
    """A workspace query."""
    n = ctypes.c_size_t()
    rc = getattr(_lib or lib(), name)(*args, ctypes.byref(n))
    if rc != TFG_OK:
        raise TfgError(rc, tfg_last_error())
    return n.value


def tfg_embedding_lookup(table, ids, scale: float = 1.0, padding_id: Optional[int] = None,
                         out_dtype: Optional[torch.dtype] = None, out=None):
    """scale * table[ids] for ids (int64 or int32) of any shape, zeros where an id is
    ``padding_id``; the result has the shape of ids with a last dimension of F, in
    ``out_dtype`` (the table's by default).  Returns (out, status)."""
    index, id32 = _need_ids(ids)
    _same("table", table, index)
    if table.dim() != 2:
        raise ValueError("table must have shape [V, F]")
    v, f = table.shape
    if out_dtype is None:
        out_dtype = table.dtype if out is None else out.dtype
    codes = _dtype_code("table", table.dtype), _dtype_code("out", out_dtype)
    out = _need_out("out", out, (*ids.shape, f), out_dtype, table)
    status = torch.empty(1, dtype=torch.int32, device=table.device)
    _run(index, "tfg_embedding_lookup32" if id32 else "tfg_embedding_lookup", ids.data_ptr(), ids.numel(),
         table.data_ptr(), codes[0], v, f, scale, _padding(padding_id), out.data_ptr(),
         codes[1], status.data_ptr())
    return out, status


class IdGroups(NamedTuple):
    rowptr: torch.Tensor      # int32 [V + 1]: places of id v are rowptr[v] .. rowptr[v + 1] - 1
    sorted_ids: torch.Tensor  # int32 [n]: the id of each place, V behind the last group
    perm: torch.Tensor        # int32 [n]: the position that each place holds
    status: torch.Tensor      # int32 [1] (device)


def tfg_group_ids_workspace_size(num_rows: int, num_ids: int) -> int:
    return _size("tfg_group_ids_workspace_size", num_rows, num_ids)


def tfg_group_ids(ids, num_rows: int, padding_id: Optional[int] = None, workspace=None) -> IdGroups:
    """Order the positions of ``ids`` (any shape, taken flat) by id, equal ids by position."""
    index, id32 = _need_ids(ids)
    n, dev = ids.numel(), ids.device
    workspace = _workspace(workspace, tfg_group_ids_workspace_size(num_rows, n), ids)
    rowptr, sorted_ids, perm, status = (torch.empty(k, dtype=torch.int32, device=dev) for k in (num_rows + 1, n, n, 1))
    _run(index, "tfg_group_ids32" if id32 else "tfg_group_ids", ids.data_ptr(), n, num_rows,
         _padding(padding_id), rowptr.data_ptr(), sorted_ids.data_ptr(), perm.data_ptr(),
         *_span(workspace), status.data_ptr())
    return IdGroups(rowptr, sorted_ids, perm, status)


def tfg_embedding_backward_workspace_size(num_features: int) -> int:
    return _size("tfg_embedding_backward_workspace_size", num_features)


def tfg_embedding_backward(groups: IdGroups, grad_out, scale: float = 1.0, out=None, workspace=None):
    """grad_table [V, F] fp32 of tfg_embedding_lookup, for the groups of its ids
    (tfg_group_ids with the same padding_id)."""
    index = _index("grad_out", grad_out)
    rowptr, sorted_ids, perm = groups[:3]
    for name, t in (("rowptr", rowptr), ("sorted_ids", sorted_ids), ("perm", perm)):
        _same(name, t, index, torch.int32)
    n, v, f = perm.numel(), rowptr.numel() - 1, grad_out.shape[-1]
    if sorted_ids.numel() != n or grad_out.numel() != n * f:
        raise ValueError("grad_out must hold a row for every id of the groups")
    code = _dtype_code("grad_out", grad_out.dtype)
    out = _need_out("out", out, (v, f), torch.float32, grad_out)
    workspace = _workspace(workspace, tfg_embedding_backward_workspace_size(f), grad_out)
    _run(index, "tfg_embedding_backward", rowptr.data_ptr(), sorted_ids.data_ptr(), perm.data_ptr(), grad_out.data_ptr(),
         code, n, v, f, scale, out.data_ptr(), *_span(workspace))
    return out


class GroupNorm(NamedTuple):
    out: torch.Tensor
    mean: Optional[torch.Tensor]   # fp32 [G, K], for the backward
    rstd: Optional[torch.Tensor]   # fp32 [G, K]
    status: torch.Tensor           # int32 [1] (device)


def tfg_group_norm_workspace_size(num_nodes: int, num_graphs: int, num_features: int, num_groups: int) -> int:
    return _size("tfg_group_norm_workspace_size", num_nodes, num_graphs, num_features, num_groups)


def _norm_inputs(x, node_offsets, gamma, beta, activation):
    index = _index("x", x)
    if x.dim() != 2:
        raise ValueError("x must have shape [N, F]")
    n, f = x.shape
    _same("node_offsets", node_offsets, index, torch.int64)
    if node_offsets.dim() != 1 or node_offsets.numel() < 1:
        raise ValueError("node_offsets must have shape [G + 1]")
    for name, w in (("gamma", gamma), ("beta", beta)):
        if w is not None:
            _same(name, w, index, torch.float32)
            if w.numel() != f:
                raise ValueError(f"{name} must have {f} values")
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, got {activation!r}")
    return index, n, f, node_offsets.numel() - 1, _dtype_code("x", x.dtype)


def tfg_group_norm(x, node_offsets, num_groups: int, gamma=None, beta=None, eps: float = 1e-5, activation: str = "none",
                   out_dtype: Optional[torch.dtype] = None, want_stats: bool = True, out=None,
                   workspace=None) -> GroupNorm:
    """Group norm over the graphs of a batch and an activation ("none", "relu", "silu",
    "gelu").  Graph g holds the rows node_offsets[g] .. node_offsets[g + 1] - 1 of x
    [N, F]; rows outside all graphs are left as they are in ``out`` (unset in a new one: give
    a padded batch whose rows are all read later an ``out`` of zeros)."""
    index, n, f, g, code = _norm_inputs(x, node_offsets, gamma, beta, activation)
    if out_dtype is None:
        out_dtype = x.dtype if out is None else out.dtype
    out_code = _dtype_code("out", out_dtype)
    need = tfg_group_norm_workspace_size(n, g, f, num_groups)
    out = _need_out("out", out, (n, f), out_dtype, x)
    workspace = _workspace(workspace, need, x)
    mean = rstd = None
    if want_stats:
        mean, rstd = (torch.empty(g, num_groups, dtype=torch.float32, device=x.device) for _ in range(2))
    status = torch.empty(1, dtype=torch.int32, device=x.device)
    _run(index, "tfg_group_norm", x.data_ptr(), code, node_offsets.data_ptr(), n, g, f, num_groups, _at(gamma), _at(beta),
         eps, ACTIVATIONS[activation], out.data_ptr(), out_code, _at(mean), _at(rstd), *_span(workspace), status.data_ptr())
    return GroupNorm(out, mean, rstd, status)


def tfg_group_norm_backward_workspace_size(num_nodes: int, num_graphs: int, num_features: int, num_groups: int) -> int:
    return _size("tfg_group_norm_backward_workspace_size", num_nodes, num_graphs, num_features, num_groups)


def tfg_group_norm_backward(x, node_offsets, num_groups: int, gamma, beta, mean, rstd, grad_out, activation: str = "none",
                            want_weight_grads: bool = True, grad_x=None, workspace=None):
    """Gradients of tfg_group_norm with the forward's arguments and statistics.  Returns
    (grad_x [N, F] in grad_out's type, grad_gamma [F], grad_beta [F]); the last two None
    without ``want_weight_grads``.  Rows outside all graphs are left as they are in
    ``grad_x`` (unset in a new one)."""
    index, n, f, g, code = _norm_inputs(x, node_offsets, gamma, beta, activation)
    _same("grad_out", grad_out, index)
    if grad_out.shape != (n, f):
        raise ValueError("grad_out must have the shape of x")
    grad_code = _dtype_code("grad_out", grad_out.dtype)
    for name, s in (("mean", mean), ("rstd", rstd)):
        _same(name, s, index, torch.float32)
        if s.numel() != g * num_groups:
            raise ValueError(f"{name} must have shape [G, num_groups]")
    need = tfg_group_norm_backward_workspace_size(n, g, f, num_groups)
    grad_x = _need_out("grad_x", grad_x, (n, f), grad_out.dtype, x)
    grad_gamma = grad_beta = None
    if want_weight_grads:
        grad_gamma, grad_beta = (torch.empty(f, dtype=torch.float32, device=x.device) for _ in range(2))
    workspace = _workspace(workspace, need, x)
    _run(index, "tfg_group_norm_backward", x.data_ptr(), code, node_offsets.data_ptr(), n, g, f, num_groups, _at(gamma),
         _at(beta), mean.data_ptr(), rstd.data_ptr(), ACTIVATIONS[activation], grad_out.data_ptr(), grad_code,
         grad_x.data_ptr(), _at(grad_gamma), _at(grad_beta), *_span(workspace))
    return grad_x, grad_gamma, grad_beta


def tfg_global_norm_workspace_size(num_tensors: int) -> int:
    return _size("tfg_global_norm_workspace_size", num_tensors)


_DTYPE_OF = operator.attrgetter("dtype")


def _tensor_list(name: str, tensors, index: int):
    """(pointers, sizes, types) of a list of contiguous tensors on one device, the first two
    as the host arrays that the C calls read.  A model has hundreds of gradients: the checks
    are passes of built-in functions over the list, and only a list that fails one is looked
    at tensor by tensor."""
    try:
        types = list(map(_DTYPE_OF, tensors))
        if (index >= 0 and set(map(torch.Tensor.get_device, tensors)) <= {index}
                and all(map(torch.Tensor.is_contiguous, tensors)) and set(types) <= _DTYPES.keys()):
            return (array.array("Q", map(torch.Tensor.data_ptr, tensors)),
                    array.array("q", map(torch.Tensor.numel, tensors)), types)
    except (TypeError, AttributeError):           # no tensor at all
        pass
    for t in tensors:                             # say which, and why
        _same(name, t, max(index, 0))
        _dtype_code(name, t.dtype)
    raise ValueError(f"{name} must be contiguous float32 or bfloat16 CUDA tensors of one device")


def _codes(types) -> array.array:
    if len(set(types)) == 1:
        return array.array("i", [_DTYPES[types[0]]]) * len(types)
    return array.array("i", [_DTYPES[t] for t in types])


def _host(a: array.array) -> int:
    return a.buffer_info()[0]


def _list_device(tensors) -> torch.device:
    return tensors[0].device if tensors else torch.device("cuda", torch.cuda.current_device())


def tfg_global_norm(tensors, workspace=None) -> torch.Tensor:
    """sqrt of the sum of all squares over a list of tensors (fp32 or bf16), fp32 [1]."""
    tensors = list(tensors)
    dev = _list_device(tensors)
    ptrs, sizes, types = _tensor_list("tensors", tensors, -1 if dev.index is None else dev.index)
    codes = _codes(types)
    norm = torch.empty(1, dtype=torch.float32, device=dev)
    workspace = _workspace(workspace, tfg_global_norm_workspace_size(len(tensors)), norm)
    _run(dev.index, "tfg_global_norm", len(tensors), _host(ptrs), _host(sizes), _host(codes), norm.data_ptr(),
         *_span(workspace))
    return norm


def tfg_clip_by_global_norm(tensors, clip_norm: float, outs=None, workspace=None):
    """tensors * clip_norm / max(global norm, clip_norm): new tensors, or ``outs`` (which may
    be the tensors themselves, in place).  Returns (outs, norm [1] before clipping)."""
    tensors = list(tensors)
    dev = _list_device(tensors)
    index = -1 if dev.index is None else dev.index
    ptrs, sizes, types = _tensor_list("tensors", tensors, index)
    codes = _codes(types)
    outs = list(map(torch.empty_like, tensors)) if outs is None else list(outs)
    out_ptrs, out_sizes, out_types = _tensor_list("outs", outs, index)
    if out_sizes != sizes or out_types != types:
        raise ValueError("outs must have the sizes and types of tensors")
    norm = torch.empty(1, dtype=torch.float32, device=dev)
    workspace = _workspace(workspace, tfg_global_norm_workspace_size(len(tensors)), norm)
    _run(index, "tfg_clip_by_global_norm", len(tensors), _host(ptrs), _host(sizes), _host(codes), clip_norm,
         _host(out_ptrs), norm.data_ptr(), *_span(workspace))
    return outs, norm
