"""ctypes binding of librgnn.so (declared in include/rgnn.h).

Argument marshalling only: every computation runs inside the HIP library.
Tensors are torch tensors on the GPU (PyTorch provides device memory and the
stream); index arrays for graph creation are host numpy arrays.  If the built
library is missing, importing this module raises -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librgnn.so")

OK, EINVAL, ERANGE, ENOMEM, EDEVICE, EUNSUPPORTED = 0, -1, -2, -3, -4, -5
PLAN_AUTO, PLAN_TRANSFORM_FIRST, PLAN_AGGREGATE_FIRST = 0, 1, 2
PLAN_TRANSFORM_FIRST_UNREORDERED = 3
PLAN_TRANSFORM_FIRST_ATTMSG = 4
LAYER_RGCN, LAYER_RGAT, LAYER_HGT, LAYER_RGAT_BACKWARD, LAYER_SEGMENT_GEMM = 0, 1, 2, 3, 4
LAYER_RGCN_BACKWARD, LAYER_HGT_BACKWARD = 5, 6
SOFTMAX_PER_DST, SOFTMAX_PER_DST_REL = 0, 1
FLAG_RELU, FLAG_RESIDUAL, FLAG_A_LINEAR = 1, 2, 4
GRAPH_HOST_ONLY, GRAPH_NO_COMPACT = 1, 2
F32, BF16, F16, F8_E4M3, I8 = 0, 1, 2, 3, 4

INDEX_KINDS = {
    "dst_rowptr": 0, "in_src": 1, "in_rel": 2, "in_eid": 3, "seg_ptr": 4, "seg_rel": 5,
    "dst_segptr": 6, "uniq_src": 7, "uniq_rel_ptr": 8, "edge2uniq": 9, "ntype_perm": 10,
    "ntype_ptr": 11, "out_ptr": 12, "out_pos": 13,
}

EXPORTED = [
    "rgnn_graph_create_coo", "rgnn_graph_create_csr", "rgnn_graph_destroy", "rgnn_graph_info",
    "rgnn_graph_export", "rgnn_workspace_size", "rgnn_select_plan", "rgcn_forward",
    "rgat_forward", "rgat_forward_noalloc", "hgt_forward", "rgat_backward", "rgcn_backward", "hgt_backward",
    "rgnn_segment_gemm",
    "rgnn_segment_gemm_workspace_size", "rgnn_typed_linear", "rgnn_typed_linear_wgrad",
    "rgnn_typed_linear_wgrad_workspace_size", "rgnn_typed_linear_select_tile",
    "rgnn_typed_linear_wgrad_select_tile", "rgnn_fp8_quantize_rows", "rgnn_fp8_quantize_weights",
    "rgnn_typed_linear_fp8", "rgnn_int8_quantize_rows", "rgnn_int8_quantize_weights", "rgnn_typed_linear_int8",
    "rgnn_dropout", "rgnn_rms_norm", "rgnn_rms_norm_backward", "rgnn_rms_norm_backward_workspace_size", "rgnn_adamw_step", "rgnn_profile_enable", "rgnn_profile_count",
    "rgnn_profile_read", "rgnn_profile_reset", "rgnn_last_error", "rgnn_version",
]


class RgnnError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"librgnn status {status}: {msg}")
        self.status = status


class GraphInfo(ctypes.Structure):
    _fields_ = [("num_nodes", ctypes.c_int64), ("num_edges", ctypes.c_int64),
                ("num_rels", ctypes.c_int32), ("num_ntypes", ctypes.c_int32),
                ("num_src_pairs", ctypes.c_int64), ("num_dst_segments", ctypes.c_int64),
                ("max_in_degree", ctypes.c_int64), ("num_empty_dst", ctypes.c_int64),
                ("num_vsegs", ctypes.c_int64), ("num_items", ctypes.c_int64),
                ("num_split_dst", ctypes.c_int64), ("chunk_edges", ctypes.c_int32),
                ("device", ctypes.c_int32)]


class Tile(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "cols", "stages", "any")]


# The arguments of dropout, rms_norm and rms_norm_backward as the header lays them out, packed at once: a call
# with one pointer costs the host a microsecond less than one with twenty arguments.
_DROPOUT_PACK = struct.Struct("3Q4QQqd3i4x").pack
_NORM_PACK = struct.Struct("7Q5QdQqd5i4x").pack
_NORM_BACKWARD_PACK = struct.Struct("9Q6QQQqd6i").pack
_NO_DROPOUT = (0, 0, 0.0)


class AdamwTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("copy", ctypes.c_void_p), ("n", ctypes.c_int64), ("param_dtype", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32), ("copy_dtype", ctypes.c_int32),
                ("state_bits", ctypes.c_int32)]


_ADAMW_PACK = struct.Struct("7Qq4i")    # an AdamwTensor at once


class AdamwHyper(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                          "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    i32, i64, vp, f32, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t
    P = ctypes.POINTER
    sig = {
        "rgnn_graph_create_coo": [i64, i32, i32, i64, vp, vp, vp, vp, i32, vp, P(vp)],
        "rgnn_graph_create_csr": [i64, i32, i32, vp, vp, vp, vp, i32, vp, P(vp)],
        "rgnn_graph_destroy": [vp],
        "rgnn_graph_info": [vp, P(GraphInfo)],
        "rgnn_graph_export": [vp, i32, vp, sz],
        "rgnn_workspace_size": [vp, i32, i32, i32, i32, i32, P(sz)],
        "rgnn_select_plan": [vp, i32, i32, i32, i32, P(i32), P(ctypes.c_double), P(ctypes.c_double)],
        "rgcn_forward": [vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, sz, vp],
        "rgat_forward": [vp, vp, vp, vp, vp, i32, i32, i32, f32, i32, i32, vp, vp, vp, sz, vp],
        "rgat_forward_noalloc": [vp, vp, vp, vp, vp, i32, i32, i32, f32, i32, i32, vp, vp, vp],
        "hgt_forward": [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, i32, vp, vp, vp, sz, vp],
        "rgat_backward": [vp, vp, vp, vp, vp, i32, i32, i32, f32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp],
        "rgcn_backward": [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp],
        "hgt_backward": [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, i32, vp, vp, vp, vp, vp, vp, vp,
                         vp, vp, vp, vp, sz, vp],
        "rgnn_segment_gemm": [vp, i64, vp, vp, i32, vp, i32, i32, vp, i64, vp, vp, sz, vp],
        "rgnn_segment_gemm_workspace_size": [i64, i32, P(sz)],
        "rgnn_typed_linear": [i32, vp, i64, i64, vp, vp, i32, i64, vp, i32, i32, i32, i32, vp, i64, i64, vp, vp],
        "rgnn_typed_linear_wgrad": [i32, vp, i64, i64, vp, vp, i64, i64, vp, vp, i32, i64, i32, i32, i32, vp, vp,
                                    sz, vp],
        "rgnn_typed_linear_wgrad_workspace_size": [i32, i64, i32, i32, i32, P(sz)],
        "rgnn_typed_linear_select_tile": [i32, vp, i64, i64, vp, i32, i64, vp, i32, i32, i32, P(Tile)],
        "rgnn_typed_linear_wgrad_select_tile": [i32, vp, i64, i64, vp, vp, i64, i64, vp, i32, i64, i32, i32, P(Tile)],
        "rgnn_fp8_quantize_rows": [i32, vp, i64, i64, i32, vp, vp, vp],
        "rgnn_fp8_quantize_weights": [i32, vp, i32, i32, i32, vp, vp, vp],
        "rgnn_typed_linear_fp8": [vp, vp, i64, vp, vp, i32, i64, vp, vp, i32, i32, i32, vp, i64, i64, vp, vp],
        "rgnn_int8_quantize_rows": [i32, vp, i64, i64, i32, vp, vp, vp],
        "rgnn_int8_quantize_weights": [i32, vp, i32, i32, i32, vp, vp, vp],
        "rgnn_typed_linear_int8": [vp, vp, i64, vp, vp, i32, i64, vp, vp, i32, i32, i32, vp, i64, i64, vp, vp],
        "rgnn_dropout": [ctypes.c_char_p, vp],
        "rgnn_rms_norm": [ctypes.c_char_p, vp],
        "rgnn_rms_norm_backward": [ctypes.c_char_p, vp],
        "rgnn_rms_norm_backward_workspace_size": [i64, i32, P(sz)],
        "rgnn_adamw_step": [P(AdamwTensor), i32, P(AdamwHyper), i64, vp, vp, vp],
        "rgnn_profile_enable": [i32],
        "rgnn_profile_count": [P(i32)],
        "rgnn_profile_read": [i32, ctypes.c_char_p, sz, P(i64), P(ctypes.c_double)],
        "rgnn_profile_reset": [],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = ctypes.c_int
    lib.rgnn_last_error.restype = ctypes.c_char_p
    lib.rgnn_last_error.argtypes = []
    lib.rgnn_version.restype = ctypes.c_char_p
    lib.rgnn_version.argtypes = []
    return lib


_lib = _load()


def lib():
    return _lib


def _check(st: int):
    if st != OK:
        raise RgnnError(st, _lib.rgnn_last_error().decode())


def _ptr(t):
    """Device pointer of a torch tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to librgnn must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _host(a, dtype):
    return None if a is None else np.ascontiguousarray(a, dtype=dtype)


def _np_ptr(a):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def _stream(stream):
    if stream is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


class Graph:
    """A graph index built by rgnn_graph_create_{coo,csr}."""

    def __init__(self, handle):
        self._h = handle

    @classmethod
    def from_coo(cls, N, T, R, src, dst, rel, ntype=None, host_only=False, stream=None,
                 compact=True):
        src, dst, rel = _host(src, np.int32), _host(dst, np.int32), _host(rel, np.int32)
        ntype = _host(ntype, np.int32)
        h = ctypes.c_void_p()
        flags = (GRAPH_HOST_ONLY if host_only else 0) | (0 if compact else GRAPH_NO_COMPACT)
        st = _lib.rgnn_graph_create_coo(int(N), int(T), int(R), len(src), _np_ptr(src),
                                        _np_ptr(dst), _np_ptr(rel), _np_ptr(ntype), flags,
                                        None if host_only else _stream(stream), ctypes.byref(h))
        _check(st)
        return cls(h)

    @classmethod
    def from_csr(cls, N, T, R, rowptr, col_src, rel, ntype=None, host_only=False, stream=None):
        rowptr = _host(rowptr, np.int64)
        col_src, rel, ntype = _host(col_src, np.int32), _host(rel, np.int32), _host(ntype, np.int32)
        h = ctypes.c_void_p()
        st = _lib.rgnn_graph_create_csr(int(N), int(T), int(R), _np_ptr(rowptr), _np_ptr(col_src),
                                        _np_ptr(rel), _np_ptr(ntype),
                                        GRAPH_HOST_ONLY if host_only else 0,
                                        None if host_only else _stream(stream), ctypes.byref(h))
        _check(st)
        return cls(h)

    @classmethod
    def from_dict(cls, g, host_only=False, compact=True):
        return cls.from_coo(g["N"], g["T"], g["R"], g["src"], g["dst"], g["rel"], g["ntype"],
                            host_only=host_only, compact=compact)

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("graph destroyed")
        return self._h

    def info(self) -> dict:
        inf = GraphInfo()
        _check(_lib.rgnn_graph_info(self.handle, ctypes.byref(inf)))
        return {f: getattr(inf, f) for f, _ in GraphInfo._fields_}

    def export(self, kind: str) -> np.ndarray:
        inf = self.info()
        n = {"dst_rowptr": inf["num_nodes"] + 1, "dst_segptr": inf["num_nodes"] + 1,
             "in_src": inf["num_edges"], "in_rel": inf["num_edges"], "in_eid": inf["num_edges"],
             "edge2uniq": inf["num_edges"], "seg_ptr": inf["num_dst_segments"] + 1,
             "seg_rel": inf["num_dst_segments"], "uniq_src": inf["num_src_pairs"],
             "uniq_rel_ptr": inf["num_rels"] + 1, "ntype_perm": inf["num_nodes"],
             "ntype_ptr": inf["num_ntypes"] + 1, "out_ptr": inf["num_nodes"] + 1,
             "out_pos": inf["num_edges"]}[kind]
        out = np.empty(max(n, 1), np.int32)
        _check(_lib.rgnn_graph_export(self.handle, INDEX_KINDS[kind], _np_ptr(out), out.nbytes))
        return out[:n]

    def close(self):
        if self._h is not None:
            _check(_lib.rgnn_graph_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def workspace_size(g: Graph, layer: int, d_in: int, d_out: int, heads: int = 1,
                   plan: int = PLAN_AUTO) -> int:
    n = ctypes.c_size_t()
    _check(_lib.rgnn_workspace_size(g.handle, layer, d_in, d_out, heads, plan, ctypes.byref(n)))
    return n.value


def select_plan(g: Graph, layer: int, d_in: int, d_out: int, heads: int = 1):
    p = ctypes.c_int32()
    tf, af = ctypes.c_double(), ctypes.c_double()
    _check(_lib.rgnn_select_plan(g.handle, layer, d_in, d_out, heads, ctypes.byref(p),
                                 ctypes.byref(tf), ctypes.byref(af)))
    return p.value, tf.value, af.value


def rgcn_forward(g, h, W, W0, out, ws, d_in, d_out, flags=0, plan=PLAN_AUTO, stream=None):
    _check(_lib.rgcn_forward(g.handle, _ptr(h), _ptr(W), _ptr(W0), d_in, d_out, flags, plan,
                             _ptr(out), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                             _stream(stream)))


def rgat_forward(g, h, W, w_src, w_dst, out, saved, ws, d_in, d_out, heads=1, neg_slope=0.2,
                 softmax_scope=SOFTMAX_PER_DST, plan=PLAN_AUTO, stream=None):
    _check(_lib.rgat_forward(g.handle, _ptr(h), _ptr(W), _ptr(w_src), _ptr(w_dst), d_in, d_out,
                             heads, float(neg_slope), softmax_scope, plan, _ptr(out), _ptr(saved),
                             _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                             _stream(stream)))


def rgat_forward_noalloc(g, h, W, w_src, w_dst, out, saved, d_in, d_out, heads=1, neg_slope=0.2,
                         softmax_scope=SOFTMAX_PER_DST, plan=PLAN_AUTO, stream=None):
    """rgat_forward with the workspace in the library's static device scratch."""
    _check(_lib.rgat_forward_noalloc(g.handle, _ptr(h), _ptr(W), _ptr(w_src), _ptr(w_dst), d_in, d_out,
                                     heads, float(neg_slope), softmax_scope, plan, _ptr(out), _ptr(saved),
                                     _stream(stream)))


def hgt_forward(g, h, Wk, Wq, Wv, Wa, Watt, Wmsg, mu, out, ws, d, heads, att_scale,
                flags=FLAG_RESIDUAL | FLAG_A_LINEAR, stream=None, saved=None):
    """saved: None or a [N, heads, 2] tensor for the softmax statistics."""
    _check(_lib.hgt_forward(g.handle, _ptr(h), _ptr(Wk), _ptr(Wq), _ptr(Wv), _ptr(Wa), _ptr(Watt),
                            _ptr(Wmsg), _ptr(mu), d, heads, float(att_scale), flags, _ptr(out),
                            _ptr(saved), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                            _stream(stream)))


def hgt_backward(g, h, Wk, Wq, Wv, Wa, Watt, Wmsg, mu, grad_out, grads, ws, d, heads, att_scale,
                 flags=FLAG_RESIDUAL | FLAG_A_LINEAR, stream=None, saved=None):
    """grads: dict of output tensors dh, dWk, dWq, dWv, dWa (or None), dWatt, dWmsg, dmu.
    saved: the forward's statistics (hgt_forward's saved), or None to recompute them."""
    _check(_lib.hgt_backward(g.handle, _ptr(h), _ptr(Wk), _ptr(Wq), _ptr(Wv), _ptr(Wa), _ptr(Watt),
                             _ptr(Wmsg), _ptr(mu), d, heads, float(att_scale), flags, _ptr(grad_out),
                             _ptr(saved), _ptr(grads["dh"]), _ptr(grads["dWk"]), _ptr(grads["dWq"]), _ptr(grads["dWv"]),
                             _ptr(grads.get("dWa")), _ptr(grads["dWatt"]), _ptr(grads["dWmsg"]),
                             _ptr(grads["dmu"]), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                             _stream(stream)))


def rgcn_backward(g, h, W, W0, out, grad_out, grad_h, grad_W, grad_W0, ws, d_in, d_out, flags=0,
                  stream=None):
    _check(_lib.rgcn_backward(g.handle, _ptr(h), _ptr(W), _ptr(W0), d_in, d_out, flags, _ptr(out),
                              _ptr(grad_out), _ptr(grad_h), _ptr(grad_W), _ptr(grad_W0), _ptr(ws),
                              0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)))


def rgat_backward(g, h, W, w_src, w_dst, saved, grad_out, grad_h, grad_W, grad_w_src,
                  grad_w_dst, ws, d_in, d_out, heads=1, neg_slope=0.2,
                  softmax_scope=SOFTMAX_PER_DST, stream=None):
    _check(_lib.rgat_backward(g.handle, _ptr(h), _ptr(W), _ptr(w_src), _ptr(w_dst), d_in, d_out,
                              heads, float(neg_slope), softmax_scope, _ptr(saved), _ptr(grad_out),
                              _ptr(grad_h),
                              _ptr(grad_W), _ptr(grad_w_src), _ptr(grad_w_dst), _ptr(ws),
                              0 if ws is None else ws.numel() * ws.element_size(),
                              _stream(stream)))


def segment_gemm_workspace_size(M: int, num_types: int) -> int:
    n = ctypes.c_size_t()
    _check(_lib.rgnn_segment_gemm_workspace_size(M, num_types, ctypes.byref(n)))
    return n.value


def segment_gemm(X, gather, type_ptr, W, Y, scatter, ws, K, Nc, stream=None):
    tp = _host(type_ptr, np.int64)
    _check(_lib.rgnn_segment_gemm(_ptr(X), X.shape[1], _ptr(gather), _np_ptr(tp), len(tp) - 1,
                                  _ptr(W), K, Nc, _ptr(Y), Y.shape[1], _ptr(scatter), _ptr(ws),
                                  0 if ws is None else ws.numel() * ws.element_size(),
                                  _stream(stream)))


# ---------------------------------------------------------------- typed linear, AdamW
#
# These calls check their tensors here: type, shape, device and strides, since a wrong
# one would read out of range.  Matrices may have any row stride (their columns lie
# side by side); everything else is contiguous.

_DTYPES: dict = {}


def _dtype_codes() -> dict:
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    return _DTYPES


def _dtype(t) -> int:
    d = _dtype_codes().get(t.dtype)
    if d is None:
        raise ValueError(f"tensors must be fp32, bf16 or fp16, not {t.dtype}")
    return d


def _need(ok, why: str):
    if not ok:
        raise ValueError(why)


def _same_device(first, *others) -> int:
    """The device of the tensors, which is the current one."""
    import torch
    d = first.get_device()
    if d < 0:
        raise ValueError("tensors must be on a GPU")
    if d != torch.cuda.current_device():
        raise ValueError(f"tensors are on device {d}, the current one is {torch.cuda.current_device()}")
    for t in others:
        if t is not None and t.get_device() != d:
            raise ValueError("tensors must be on one device")
    return d


def _stream_on(stream, device: int):
    """The stream's handle; None: the device's current stream, without making an object of it."""
    if stream is not None:
        if getattr(stream, "device_index", device) != device:
            raise ValueError(f"the stream is on device {stream.device_index}, the tensors on {device}")
        return _stream(stream)
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device) if raw is not None else _stream(None)


def _matrix(t, name: str, cols: int):
    """(pointer, rows, leading dimension) of a matrix with `cols` columns."""
    if t.dim() != 2 or t.shape[1] != cols:
        raise ValueError(f"{name} must have {cols} columns")
    rows, ld = t.shape[0], t.stride(0)
    if rows <= 1:
        ld = max(ld, cols)
    if ld < cols or (cols > 1 and t.stride(1) != 1):
        raise ValueError(f"{name}'s columns must lie side by side, its rows apart")
    return t.data_ptr(), rows, ld


def _index(t):
    """Pointer of an index array, None for none."""
    if t is None:
        return None
    import torch
    if t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous():
        raise ValueError("gather and scatter must be contiguous int32 [M]")
    return t.data_ptr()


def _positions(type_ptr, types: int, first, second, rows: int) -> int:
    """Checks the offsets and the index arrays' lengths; the number of positions."""
    import torch
    if type_ptr.dtype != torch.int64 or type_ptr.dim() != 1 or type_ptr.shape[0] != types + 1 or \
            not type_ptr.is_contiguous():
        raise ValueError("type_ptr must be contiguous int64 [types + 1]")
    if first is not None and second is not None and first.shape[0] != second.shape[0]:
        raise ValueError("gather and scatter must have one length")
    return first.shape[0] if first is not None else second.shape[0] if second is not None else rows


def typed_linear(X, type_ptr, W, Y, gather=None, scatter=None, trans_w=False, stream=None):
    """Y[scatter[i]] = X[gather[i]] W[t(i)] over the positions of device offsets
    type_ptr [types + 1] (trans_w: W [types, N, K] used transposed).  X, W, Y fp32, bf16
    or fp16; Y of that type or fp32."""
    d = _same_device(X, type_ptr, W, Y, gather, scatter)
    if W.dim() != 3 or not W.is_contiguous() or W.dtype != X.dtype:
        raise ValueError("W must be contiguous [types, ., .] of X's type")
    T, K, N = W.shape
    if trans_w:
        K, N = N, K
    xp, xr, ldx = _matrix(X, "X", K)
    yp, yr, ldy = _matrix(Y, "Y", N)
    gp, sp = _index(gather), _index(scatter)
    M = _positions(type_ptr, T, gather, scatter, xr)
    _check(_lib.rgnn_typed_linear(_dtype(X), xp, xr, ldx, gp, type_ptr.data_ptr(), T, M, W.data_ptr(), K, N,
                                  1 if trans_w else 0, _dtype(Y), yp, yr, ldy, sp, _stream_on(stream, d)))


def typed_linear_wgrad_workspace_size(dtype, M: int, num_types: int, K: int, N: int) -> int:
    """dtype: torch.float32, torch.bfloat16 or torch.float16."""
    import torch
    n = ctypes.c_size_t()
    _check(_lib.rgnn_typed_linear_wgrad_workspace_size(_dtype(torch.empty(0, dtype=dtype)), M, num_types, K, N,
                                                       ctypes.byref(n)))
    return n.value


def typed_linear_wgrad(X, dY, type_ptr, dW, ws, gather=None, dy_gather=None, stream=None):
    """dW[t] = sum over the positions i of type t of X[gather[i]]^T dY[dy_gather[i]]."""
    d = _same_device(X, dY, type_ptr, dW, ws, gather, dy_gather)
    if dY.dtype != X.dtype:
        raise ValueError("dY must be of X's type")
    if dW.dim() != 3 or not dW.is_contiguous():
        raise ValueError("dW must be contiguous [types, K, N]")
    T, K, N = dW.shape
    xp, xr, ldx = _matrix(X, "X", K)
    dp, dr, ldd = _matrix(dY, "dY", N)
    gp, sp = _index(gather), _index(dy_gather)
    M = _positions(type_ptr, T, gather, dy_gather, xr)
    _check(_lib.rgnn_typed_linear_wgrad(_dtype(X), xp, xr, ldx, gp, dp, dr, ldd, sp, type_ptr.data_ptr(), T, M, K, N,
                                        _dtype(dW), dW.data_ptr(), _ptr(ws),
                                        0 if ws is None else ws.numel() * ws.element_size(), _stream_on(stream, d)))


def _tile(t: Tile):
    return t.rows, t.cols, t.stages, bool(t.any)


def typed_linear_select_tile(X, W, gather=None, scatter=None, trans_w=False):
    """(rows, columns, stages, any address) of the tile that typed_linear takes for these tensors, or, for
    float8_e4m3fn X and W, typed_linear_fp8, for int8 typed_linear_int8."""
    import torch
    eight = {torch.float8_e4m3fn: F8_E4M3, torch.int8: I8}.get(X.dtype)
    T, K, N = W.shape
    if trans_w or eight is not None:
        K, N = N, K
    xp, xr, ldx = _matrix(X, "X", K)
    gp, _ = _index(gather), _index(scatter)
    M = gather.shape[0] if gather is not None else scatter.shape[0] if scatter is not None else xr
    t = Tile()
    _check(_lib.rgnn_typed_linear_select_tile(_dtype(X) if eight is None else eight, xp, xr, ldx, gp, T, M, W.data_ptr(),
                                              K, N, 1 if trans_w or eight is not None else 0, ctypes.byref(t)))
    return _tile(t)


def typed_linear_wgrad_select_tile(X, dY, types: int, gather=None, dy_gather=None):
    """(rows of k, columns of n, stages, any address) of the tile that typed_linear_wgrad takes."""
    K, N = X.shape[1], dY.shape[1]
    xp, xr, ldx = _matrix(X, "X", K)
    dp, dr, ldd = _matrix(dY, "dY", N)
    gp, sp = _index(gather), _index(dy_gather)
    M = gather.shape[0] if gather is not None else dy_gather.shape[0] if dy_gather is not None else xr
    t = Tile()
    _check(_lib.rgnn_typed_linear_wgrad_select_tile(_dtype(X), xp, xr, ldx, gp, dp, dr, ldd, sp, types, M, K, N,
                                                    ctypes.byref(t)))
    return _tile(t)


def fp8_widths(K: int):
    """(columns of the codes, bytes of the scales) of K elements."""
    return -(-K // 128) * 128, -(-K // 512) * 4


def _on_stream(stream, device, make):
    """make() with the allocator on `stream`."""
    import torch
    if stream is None or device.type != "cuda":
        return make()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.stream(stream):
        return make()


def _fp8_out(codes, scales, lead, blocks, K, device, stream):
    """The outputs, those that are not given in memory of the stream that writes them."""
    import torch
    if stream is not None and (codes is None or scales is None):
        return _on_stream(stream, device, lambda: _fp8_out(codes, scales, lead, blocks, K, device, None))
    Kp, Ks = fp8_widths(K)
    if codes is None:
        codes = torch.empty(*lead, Kp, dtype=torch.float8_e4m3fn, device=device)
    if scales is None:
        scales = torch.empty(*blocks, Ks, dtype=torch.uint8, device=device)
    _fp8_check(codes, scales, lead, blocks, K)
    return codes, scales


def _fp8_check(codes, scales, lead, blocks, K):
    import torch
    Kp, Ks = fp8_widths(K)
    if codes.dtype != torch.float8_e4m3fn or codes.shape != (*lead, Kp) or not codes.is_contiguous():
        raise ValueError(f"codes must be contiguous float8_e4m3fn {(*lead, Kp)}")
    if scales.dtype != torch.uint8 or scales.shape != (*blocks, Ks) or not scales.is_contiguous():
        raise ValueError(f"scales must be contiguous uint8 {(*blocks, Ks)}")


def fp8_quantize_rows(X, codes=None, scales=None, stream=None):
    """X [rows, K] -> (codes float8_e4m3fn [rows, Kp], scales uint8 [rows, Ks]), a
    power-of-two scale for each 128 columns of a row.  Outputs that are not given are
    made in the memory of `stream`: to use them on another one, wait for it there."""
    if X.dim() != 2:
        raise ValueError("X must be a matrix")
    K = X.shape[1]
    xp, rows, ldx = _matrix(X, "X", K)
    codes, scales = _fp8_out(codes, scales, (rows,), (rows,), K, X.device, stream)
    d = _same_device(X, codes, scales)
    _check(_lib.rgnn_fp8_quantize_rows(_dtype(X), xp, rows, ldx, K, codes.data_ptr(), scales.data_ptr(),
                                       _stream_on(stream, d)))
    return codes, scales


def fp8_quantize_weights(W, codes=None, scales=None, stream=None):
    """W [types, K, N] -> (codes float8_e4m3fn [types, N, Kp], scales uint8
    [types, ceil(N / 128), Ks]), a power-of-two scale for each 128 x 128 block."""
    if W.dim() != 3 or not W.is_contiguous():
        raise ValueError("W must be contiguous [types, K, N]")
    T, K, N = W.shape
    codes, scales = _fp8_out(codes, scales, (T, N), (T, -(-N // 128)), K, W.device, stream)
    d = _same_device(W, codes, scales)
    _check(_lib.rgnn_fp8_quantize_weights(_dtype(W), W.data_ptr(), T, K, N, codes.data_ptr(), scales.data_ptr(),
                                          _stream_on(stream, d)))
    return codes, scales


def typed_linear_fp8(X, x_scales, type_ptr, W, w_scales, Y, gather=None, scatter=None, stream=None):
    """typed_linear on the codes and scales of fp8_quantize_rows and
    fp8_quantize_weights; Y fp32, bf16 or fp16."""
    d = _same_device(X, x_scales, type_ptr, W, w_scales, Y, gather, scatter)
    if W.dim() != 3 or X.dim() != 2:
        raise ValueError("X must be [rows, Kp], W [types, N, Kp]")
    T, N, K = W.shape
    rows = X.shape[0]
    _fp8_check(X, x_scales, (rows,), (rows,), K)
    _fp8_check(W, w_scales, (T, N), (T, -(-N // 128)), K)
    yp, yr, ldy = _matrix(Y, "Y", N)
    gp, sp = _index(gather), _index(scatter)
    M = _positions(type_ptr, T, gather, scatter, rows)
    _check(_lib.rgnn_typed_linear_fp8(X.data_ptr(), x_scales.data_ptr(), rows, gp, type_ptr.data_ptr(), T, M,
                                      W.data_ptr(), w_scales.data_ptr(), K, N, _dtype(Y), yp, yr, ldy, sp,
                                      _stream_on(stream, d)))


class _Torch:
    """What these calls take from torch, looked up once."""

    def __init__(self):
        import torch
        self.current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        self.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.empty, self.float32, self.e4m3 = torch.empty, torch.float32, torch.float8_e4m3fn
        self.int8, self.uint8, self.int32, self.int64 = torch.int8, torch.uint8, torch.int32, torch.int64

        class Floats(dict):
            def __missing__(self, dtype):
                raise ValueError(f"tensors must be fp32, bf16 or fp16, not {dtype}")
        self.floats = Floats(_dtype_codes())


_torch_cache: list = []


def _torch() -> _Torch:
    if not _torch_cache:
        _torch_cache.append(_Torch())
    return _torch_cache[0]


def _device_of(X, t: _Torch) -> int:
    """The device of a call, which is that of X and the current one."""
    d = X.get_device()
    if d < 0:
        raise ValueError("tensors must be on a GPU")
    if d != t.current():
        raise ValueError(f"tensors are on device {d}, the current one is {t.current()}")
    return d


def _stream_of(stream, device: int, t: _Torch):
    """The stream's handle; None: the device's current stream."""
    return t.raw_stream(device) if stream is None and t.raw_stream is not None else _stream_on(stream, device)


def _rows(t, name: str, shape, device: int):
    """(pointer, leading dimension) of a matrix of that shape and device."""
    if t.shape != shape or t.get_device() != device:
        raise ValueError(f"{name} must be {tuple(shape)}, on device {device}")
    if t.is_contiguous():
        return t.data_ptr(), shape[1]
    p, _, ld = _matrix(t, name, shape[1])
    return p, ld


def _flat(t, name: str, shape, device: int, dtype=None) -> int:
    """Pointer of a contiguous tensor of that shape, type and device."""
    if t.shape != shape or t.get_device() != device or not t.is_contiguous() or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} must be contiguous {tuple(shape)}" + (f" of {dtype}" if dtype is not None else "") +
                         f", on device {device}")
    return t.data_ptr()


def _int8_out(codes, scales, lead, K, device, stream):
    """The outputs, those that are not given in memory of the stream that writes them."""
    if codes is not None and scales is not None:
        return codes, scales
    if stream is not None:
        return _on_stream(stream, device, lambda: _int8_out(codes, scales, lead, K, device, None))
    t = _torch()
    if codes is None:
        codes = t.empty(*lead, -(-K // 128) * 128, dtype=t.int8, device=device)
    if scales is None:
        scales = t.empty(*lead, dtype=t.float32, device=device)
    return codes, scales


def int8_quantize_rows(X, codes=None, scales=None, stream=None):
    """X [rows, K] -> (codes int8 [rows, Kp], scales float32 [rows]), a scale for each row.  Outputs that
    are not given are made in the memory of `stream`: to use them on another one, wait for it there."""
    t = _torch()
    d = _device_of(X, t)
    if X.dim() != 2:
        raise ValueError("X must be a matrix")
    rows, K = shape = X.shape
    xp, ldx = _rows(X, "X", shape, d)
    made = codes is None, scales is None
    codes, scales = _int8_out(codes, scales, (rows,), K, X.device, stream)
    cp = codes.data_ptr() if made[0] else _flat(codes, "codes", (rows, -(-K // 128) * 128), d, t.int8)
    sp = scales.data_ptr() if made[1] else _flat(scales, "scales", (rows,), d, t.float32)
    _check(_lib.rgnn_int8_quantize_rows(t.floats[X.dtype], xp, rows, ldx, K, cp, sp, _stream_of(stream, d, t)))
    return codes, scales


def int8_quantize_weights(W, codes=None, scales=None, stream=None):
    """W [types, K, N] -> (codes int8 [types, N, Kp], scales float32 [types, N]), a scale for each output."""
    t = _torch()
    d = _device_of(W, t)
    if W.dim() != 3 or not W.is_contiguous():
        raise ValueError("W must be contiguous [types, K, N]")
    T, K, N = W.shape
    codes, scales = _int8_out(codes, scales, (T, N), K, W.device, stream)
    _check(_lib.rgnn_int8_quantize_weights(t.floats[W.dtype], W.data_ptr(), T, K, N,
                                           _flat(codes, "codes", (T, N, -(-K // 128) * 128), d, t.int8),
                                           _flat(scales, "scales", (T, N), d, t.float32), _stream_of(stream, d, t)))
    return codes, scales


def typed_linear_int8(X, x_scales, type_ptr, W, w_scales, Y, gather=None, scatter=None, stream=None):
    """typed_linear on the codes and scales of int8_quantize_rows (or rms_norm) and
    int8_quantize_weights; Y fp32, bf16 or fp16."""
    t = _torch()
    d = _device_of(X, t)
    if W.dim() != 3 or X.dim() != 2 or Y.dim() != 2:
        raise ValueError("X must be [rows, Kp], W [types, N, Kp], Y [y_rows, N]")
    (T, N, K), rows, y_rows = W.shape, X.shape[0], Y.shape[0]
    if K % 128:
        raise ValueError("codes lie in rows of whole blocks of 128")
    yp, ldy = _rows(Y, "Y", (y_rows, N), d)
    M = gather.shape[0] if gather is not None else scatter.shape[0] if scatter is not None else rows
    gp = None if gather is None else _flat(gather, "gather", (M,), d, t.int32)
    sp = None if scatter is None else _flat(scatter, "scatter", (M,), d, t.int32)
    _check(_lib.rgnn_typed_linear_int8(
        _flat(X, "X", (rows, K), d, t.int8), _flat(x_scales, "x_scales", (rows,), d, t.float32), rows, gp,
        _flat(type_ptr, "type_ptr", (T + 1,), d, t.int64), T, M, _flat(W, "W", (T, N, K), d, t.int8),
        _flat(w_scales, "w_scales", (T, N), d, t.float32), K, N, t.floats[Y.dtype], yp, y_rows, ldy, sp, _stream_of(stream, d, t)))


class Dropout:
    """What rms_norm, its backward and dropout drop: a value with probability p, by the numbers of a
    counter-based generator.  rng: device int64 [2], seed and offset, read when the kernels run; call: the number
    of the call within a step.  The backward pass takes the forward's Dropout and the same rng."""

    def __init__(self, p: float, rng, call: int = 0):
        import torch
        if rng.dtype != torch.int64 or rng.dim() != 1 or rng.shape[0] != 2 or not rng.is_contiguous():
            raise ValueError("rng must be contiguous int64 [2]")
        if not 0 <= p <= 1:
            raise ValueError("p must lie in [0, 1]")
        if not -2 ** 63 <= call < 2 ** 63:
            raise ValueError("call must be a 64-bit number")
        self.p, self.rng, self.call = float(p), rng, int(call)

    def _args(self, device: int):
        rng = self.rng
        if rng.get_device() != device:
            raise ValueError("rng must be on the tensors' device")
        return rng.data_ptr(), self.call, self.p


def dropout(X, Y, dropout: Dropout, residual=None, stream=None):
    """Y = [residual +] D(X); X, Y fp32, bf16 or fp16, residual of Y's type.  Y may be X or residual.  With the
    output's gradient as X and no residual: the gradient of x."""
    t = _torch()
    floats = t.floats
    d = _device_of(X, t)
    if X.dim() != 2:
        raise ValueError("X must be a matrix")
    rows, cols = shape = X.shape
    xp, ldx = _rows(X, "X", shape, d)
    yp, ldy = _rows(Y, "Y", shape, d)
    rp = ldr = 0
    if residual is not None:
        if residual.dtype != Y.dtype:
            raise ValueError("residual must be of Y's type")
        rp, ldr = _rows(residual, "residual", shape, d)
    _check(_lib.rgnn_dropout(_DROPOUT_PACK(xp, rp, yp, rows, ldx, ldr, ldy, *dropout._args(d), cols, floats[X.dtype], floats[Y.dtype]),
                             _stream_of(stream, d, t)))


def rms_norm(X, weight, Y, eps=1e-6, residual=None, sum=None, scales=None, rstd=None, dropout=None, stream=None):
    """r = [residual +] D(X), Y = r / sqrt(mean(r^2) + eps) * weight for each row; weight [cols] or None.
    sum: takes r (of residual's type; of any without one); rstd: float32 [rows], takes the root's inverse.  Y fp32,
    bf16 or fp16; or float8_e4m3fn codes [rows, Kp] with scales uint8 [rows, Ks] for typed_linear_fp8; or int8 codes
    [rows, Kp] with scales float32 [rows] for typed_linear_int8.  Y may be X, sum may be residual.  A call's 16-bit tensors are of
    one type."""
    t = _torch()
    floats = t.floats
    d = _device_of(X, t)
    if X.dim() != 2:
        raise ValueError("X must be a matrix")
    rows, cols = shape = X.shape
    xp, ldx = _rows(X, "X", shape, d)
    rp = ldr = sp = lds = wp = scp = sdp = 0
    x_type = sum_type = floats[X.dtype]
    if residual is not None:
        rp, ldr = _rows(residual, "residual", shape, d)
        sum_type = floats[residual.dtype]
    if sum is not None:
        sp, lds = _rows(sum, "sum", shape, d)
        if residual is None:
            sum_type = floats[sum.dtype]
        elif sum.dtype != residual.dtype:
            raise ValueError("sum must be of residual's type")
    w_type = F32
    if weight is not None:
        wp, w_type = _flat(weight, "weight", (cols,), d), floats[weight.dtype]
    if rstd is not None:
        sdp = _flat(rstd, "rstd", (rows,), d, t.float32)
    code = floats.get(Y.dtype)
    if code is not None:
        if scales is not None:
            raise ValueError("scales are for 8-bit codes")
        yp, ldy = _rows(Y, "Y", shape, d)
    else:
        if scales is None:
            raise ValueError("Y must be fp32, bf16 or fp16, or 8-bit codes with scales")
        Kp, Ks = fp8_widths(cols)
        if Y.dtype == t.int8:
            code, ldy, scp = I8, Kp, _flat(scales, "scales", (rows,), d, t.float32)
        else:
            code, ldy, scp = F8_E4M3, Kp, _flat(scales, "scales", (rows, Ks), d, t.uint8)
        yp = _flat(Y, "codes", (rows, Kp), d, t.int8 if code == I8 else t.e4m3)
    _check(_lib.rgnn_rms_norm(_NORM_PACK(xp, rp, sp, wp, yp, scp, sdp, rows, ldx, ldr, lds, ldy, eps,
                                         *(_NO_DROPOUT if dropout is None else dropout._args(d)), cols, x_type, sum_type,
                                         w_type, code), _stream_of(stream, d, t)))


def rms_norm_backward_workspace_size(rows: int, cols: int) -> int:
    n = ctypes.c_size_t()
    _check(_lib.rgnn_rms_norm_backward_workspace_size(rows, cols, ctypes.byref(n)))
    return n.value


def rms_norm_backward(dY, sum, rstd, weight, d_sum=None, d_residual=None, dX=None, dW=None, ws=None, dropout=None,
                      stream=None):
    """The gradients of rms_norm: sum and rstd as it wrote them (sum: X itself without residual and dropout), d_sum
    the gradient that reaches the sum by other ways.  d_residual (sum's type), dX and dW [cols] are written where
    given; dW needs the workspace ws.  d_residual may be d_sum, dX may be dY."""
    t = _torch()
    floats = t.floats
    d = _device_of(dY, t)
    if dY.dim() != 2:
        raise ValueError("dY must be a matrix")
    rows, cols = shape = dY.shape
    yp, ldy = _rows(dY, "dY", shape, d)
    sp, lds = _rows(sum, "sum", shape, d)
    gp = ldg = rp = ldr = xp = ldx = wp = dwp = wsp = ws_bytes = 0
    w_type = x_type = dw_type = F32
    if d_sum is not None:
        if d_sum.dtype != sum.dtype:
            raise ValueError("d_sum must be of sum's type")
        gp, ldg = _rows(d_sum, "d_sum", shape, d)
    if d_residual is not None:
        if d_residual.dtype != sum.dtype:
            raise ValueError("d_residual must be of sum's type")
        rp, ldr = _rows(d_residual, "d_residual", shape, d)
    if dX is not None:
        (xp, ldx), x_type = _rows(dX, "dX", shape, d), floats[dX.dtype]
    if weight is not None:
        wp, w_type = _flat(weight, "weight", (cols,), d), floats[weight.dtype]
    if dW is not None:
        dwp, dw_type = _flat(dW, "dW", (cols,), d), floats[dW.dtype]
    if ws is not None:
        if ws.get_device() != d or not ws.is_contiguous():
            raise ValueError("the workspace must be contiguous, on the tensors' device")
        wsp, ws_bytes = ws.data_ptr(), ws.numel() * ws.element_size()
    _check(_lib.rgnn_rms_norm_backward(
        _NORM_BACKWARD_PACK(yp, sp, _flat(rstd, "rstd", (rows,), d, t.float32), wp, gp, rp, xp, dwp, wsp, rows, ldy, lds, ldg,
                            ldr, ldx, ws_bytes, *(_NO_DROPOUT if dropout is None else dropout._args(d)), cols, floats[dY.dtype],
                            floats[sum.dtype], w_type, x_type, dw_type), _stream_of(stream, d, t)))


class AdamwTensors:
    """The tensors of adamw_step, checked once and kept: lists of parameters,
    gradients (the buffers that the backward calls write) and states m, v, fp32, or int8
    and uint8 with m_scale, v_scale (fp32, one for each 256 elements); copies: None, or a
    tensor or None for each parameter, which takes the new value in its own type.

    Their memory is kept too, and a step refuses a tensor that has been given other memory since
    (`.data = `, `set_`, `resize_`): make the list again then.  Gradients that are new tensors after each
    backward pass need a list of their own each time; a captured graph holds the addresses of its capture."""

    def __init__(self, params, grads, m, v, m_scale=None, v_scale=None, copies=None):
        import torch
        n = len(params)
        m_scale, v_scale, copies = (x if x is not None else [None] * n for x in (m_scale, v_scale, copies))
        lists = (params, grads, m, v, m_scale, v_scale, copies)
        _need(all(len(x) == n for x in lists), "lists must have one length")
        self._kept = [(k, t) for k, x in enumerate(zip(*lists)) for t in x if t is not None]
        self._array = (AdamwTensor * max(n, 1))()
        self._n = n
        self.device = params[0].get_device() if n else None
        device, codes = self.device, _dtype_codes()
        pack, at, size_of = _ADAMW_PACK.pack_into, 0, _ADAMW_PACK.size
        for k, (p, g, a, b, sa, sb, c) in enumerate(zip(*lists)):
            size, eight = p.numel(), a.dtype == torch.int8
            for t in (p, g, a, b, sa, sb, c):
                if t is not None and (t.get_device() != device or device < 0 or not t.is_contiguous()):
                    raise ValueError(f"tensor {k}: tensors must be contiguous, on a GPU and on one device")
            if g.numel() != size or a.numel() != size or b.numel() != size or (c is not None and c.numel() != size):
                raise ValueError(f"tensor {k}: lengths differ")
            if eight:
                blocks = -(-size // 256)
                _need(b.dtype == torch.uint8 and all(t is not None and t.dtype == torch.float32 and
                                                     t.numel() == blocks for t in (sa, sb)),
                      f"tensor {k}: 8-bit states are int8 and uint8 with fp32 scales [{blocks}]")
            elif a.dtype != torch.float32 or b.dtype != torch.float32 or sa is not None or sb is not None:
                raise ValueError(f"tensor {k}: states are fp32 without scales, or int8 and uint8 with them")
            try:
                types = codes[p.dtype], codes[g.dtype], F32 if c is None else codes[c.dtype]
            except KeyError:
                raise ValueError(f"tensor {k}: parameter, gradient and copy must be fp32, bf16 or fp16") from None
            pack(self._array, at, p.data_ptr(), g.data_ptr(), a.data_ptr(), b.data_ptr(),
                 0 if sa is None else sa.data_ptr(), 0 if sb is None else sb.data_ptr(),
                 0 if c is None else c.data_ptr(), size, *types, 8 if eight else 32)
            at += size_of
        # with the storages kept, no other memory can come to lie at these addresses
        self._storages = [t.untyped_storage() for _, t in self._kept]
        self._where = [t.data_ptr for _, t in self._kept]
        self._addresses = [where() for where in self._where]

    def _check_addresses(self):
        now = [where() for where in self._where]
        if now != self._addresses:
            k = next(k for (k, _), a, b in zip(self._kept, now, self._addresses) if a != b)
            raise ValueError(f"tensor {k}: its memory has moved since the list was made; make the list again")


def adamw_step(tensors: AdamwTensors, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01,
               grad_scale=None, stream=None):
    """One AdamW step.  step: the step's number from 1, or a device int64 [1] that
    holds it; grad_scale: None or a device fp32 [1]."""
    import torch
    d = tensors.device
    if d is None:
        return
    if d != torch.cuda.current_device():
        raise ValueError(f"tensors are on device {d}, the current one is {torch.cuda.current_device()}")
    tensors._check_addresses()
    step_dev = None
    if isinstance(step, torch.Tensor):
        if step.dtype != torch.int64 or step.numel() != 1 or step.get_device() != d:
            raise ValueError("step must be a number or a device int64 [1]")
        step, step_dev = 0, step.data_ptr()
    if grad_scale is not None:
        if grad_scale.dtype != torch.float32 or grad_scale.numel() != 1 or grad_scale.get_device() != d:
            raise ValueError("grad_scale must be a device fp32 [1]")
        grad_scale = grad_scale.data_ptr()
    hyper = AdamwHyper(lr, beta1, beta2, eps, weight_decay)
    _check(_lib.rgnn_adamw_step(tensors._array, tensors._n, ctypes.byref(hyper), step, step_dev, grad_scale,
                                _stream_on(stream, d)))


def profile_enable(on: bool):
    _check(_lib.rgnn_profile_enable(1 if on else 0))


def profile_reset():
    _check(_lib.rgnn_profile_reset())


def profile_read() -> dict:
    """{kernel name: (launches, total ms)} of the launches recorded while enabled."""
    n = ctypes.c_int32()
    _check(_lib.rgnn_profile_count(ctypes.byref(n)))
    out = {}
    buf = ctypes.create_string_buffer(128)
    for i in range(n.value):
        cnt, ms = ctypes.c_int64(), ctypes.c_double()
        _check(_lib.rgnn_profile_read(i, buf, 128, ctypes.byref(cnt), ctypes.byref(ms)))
        out[buf.value.decode()] = (cnt.value, ms.value)
    return out


def version() -> str:
    return _lib.rgnn_version().decode()
