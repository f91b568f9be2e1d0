"""ctypes binding of libftc.so: argument marshalling only.

Every function here has the name of the C entry point it calls (include/ftc.h).  Tensors
are torch CUDA tensors used purely as device buffers; outputs and workspaces are
allocated with torch.empty and handed to the library as raw pointers.  All work is
enqueued on torch's current stream.  There is no CPU or PyTorch fallback: if the shared
library is missing, lib() raises.
"""
import collections
import ctypes as C
import os
import struct

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libftc.so")

FTC_F32, FTC_F16, FTC_BF16 = 0, 1, 2
FTC_PATH_AUTO, FTC_PATH_VALU, FTC_PATH_MFMA = 0, 1, 2
FTC_OK, FTC_EINVAL, FTC_EUNSUPPORTED, FTC_EALIGN, FTC_EWORKSPACE, FTC_EHIP = 0, -1, -2, -3, -4, -5

_DTYPES = {torch.float32: FTC_F32, torch.float16: FTC_F16, torch.bfloat16: FTC_BF16}

_I, _P, _Z, _F, _D = C.c_int32, C.c_void_p, C.c_size_t, C.c_float, C.c_double

# (restype, argtypes) of every export, in the order of include/ftc.h; with these set, ctypes
# rejects a call with the wrong number of arguments instead of passing garbage.
_SIGNATURES = {
    "ftc_version": (_I, []),
    "ftc_last_error": (C.c_char_p, []),
    "ftc_validate_csr": (_I, [_P, _P, _P]),
    "ftc_build_windows_workspace_bytes": (_Z, [_I, _I, _I, _I]),
    "ftc_build_windows": (_I, [_P, _P, _P, _Z, _P]),
    "ftc_build_windows_concurrent": (_I, [_P, _P, _P, _Z, _P, _P]),
    "ftc_gcn_norm": (_I, [_P, _P, _P, _P, _P]),
    "ftc_spmm_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_spmm": (_I, [_P, _P, _P, _P, _I, _I, _I, _P, _I, _I, _P, _I, _I, _P, _Z, _P]),
    "ftc_spmm_noalloc": (_I, [_P, _P, _P, _P, _I, _I, _I, _P, _I, _I, _P, _I, _I, _P]),
    "ftc_sddmm_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_sddmm": (_I, [_P, _P, _P, _P, _I, _I, _I, _P, _P, _F, _I, _P, _I, _P, _Z, _P]),
    "ftc_row_rnorm": (_I, [_I, _P, _I, _I, _I, _P, _P]),
    "ftc_edge_softmax_workspace_bytes": (_Z, [_I, _I]),
    "ftc_edge_softmax": (_I, [_P, _P, _P, _P, _P, _Z, _P]),
    "ftc_update_gemm": (_I, [_I, _P, _I, _I, _I, _P, _I, _P, _I, _I, _P, _I, _P]),
    "ftc_gcn_layer_workspace_bytes": (_Z, [_I, _I, _I, _I]),
    "ftc_gcn_layer": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _P, _I, _I, _P, _I, _I, _I, _P, _Z, _P]),
    "ftc_agnn_layer_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_agnn_layer": (_I, [_P, _P, _P, _I, _I, _I, _F, _P, _I, _I, _P, _P, _P, _I, _I, _P, _Z, _P]),
    "ftc_transpose_index": (_I, [_P, _P, _P, _P, _P]),
    "ftc_edge_softmax_backward": (_I, [_P, _P, _P, _P, _P, _P, _Z, _P]),
    "ftc_weight_grad_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_weight_grad": (_I, [_I, _P, _I, _I, _I, _P, _I, _I, _P, _P, _Z, _P]),
    "ftc_update_gemm_backward_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_update_gemm_backward": (_I, [_I, _P, _I, _I, _I, _P, _I, _P, _I, _I, _P, _I, _P, _I, _I, _P, _P, _Z, _P]),
    "ftc_gcn_layer_backward_workspace_bytes": (_Z, [_I, _I, _I, _I]),
    "ftc_gcn_layer_backward": (_I, [_P, _P, _P, _P, _P, _I, _I, _I, _P, _I, _P, _I, _I, _P, _I, _P, _I, _P, _I, _P,
                                    _Z, _P]),
    "ftc_agnn_layer_backward_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_agnn_layer_backward": (_I, [_P, _P, _P, _P, _I, _I, _I, _F, _P, _P, _I, _P, _I, _I, _P, _I, _P, _Z, _P]),
    "ftc_agnn_layer_backward_fused_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_agnn_layer_backward_fused": (_I, [_P, _P, _P, _I, _I, _I, _F, _P, _P, _I, _I, _P, _I, _P, _I, _I, _P, _P, _P, _Z, _P]),
    "ftc_embedding": (_I, [_I, _P, _I, _P, _I, _I, _I, _F, _P, _I, _I, _P]),
    "ftc_embedding_backward_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_embedding_backward": (_I, [_I, _P, _I, _P, _I, _I, _I, _F, _P, _I, _I, _P, _Z, _P]),
    "ftc_linear_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_linear": (_I, [_I, _P, _I, _I, _I, _P, _I, _P, _I, _P, _I, _P, _I, _P, _I, _I, _P, _Z, _P]),
    "ftc_linear_backward_workspace_bytes": (_Z, [_I, _I, _I]),
    "ftc_linear_backward": (_I, [_I, _P, _I, _I, _I, _P, _I, _P, _I, _P, _I, _P, _I, _P, _I, _I, _P, _P, _I, _P, _Z, _P]),
    "ftc_grad_norm_workspace_bytes": (_Z, [_I]),
    "ftc_grad_norm": (_I, [_P, _I, _D, _P, _P, _Z, _P]),
    "ftc_clip_grad_norm": (_I, [_P, _I, _D, _D, _P, _P, _Z, _P]),
    "ftc_grouped_linear_workspace_bytes": (_Z, [_I, _I, _I, _I]),
    "ftc_grouped_linear": (_I, [_I, _P, _I, _P, _I, _I, _I, _P, _I, _P, _I, _P, _I, _P, _I, _P, _I, _I, _P, _Z, _P]),
    "ftc_grouped_linear_backward_workspace_bytes": (_Z, [_I, _I, _I, _I]),
    "ftc_grouped_linear_backward": (_I, [_I, _P, _I, _P, _I, _I, _I, _P, _I, _P, _I, _P, _I, _P, _I, _P, _I, _I, _P, _P, _I, _P, _Z, _P]),
    "ftc_block_norm": (_I, [_P, _P, _I, _P, _I, _P, _P]),
    "ftc_block_norm_backward_workspace_bytes": (_Z, [_I, _I]),
    "ftc_block_norm_backward": (_I, [_P, _P, _P, _I, _P, _I, _P, _P, _Z, _P]),
    "ftc_graph_attention_workspace_bytes": (_Z, [_I, _I, _I, _I, _I, _I]),
    "ftc_graph_attention": (_I, [_I, _P, _I, _P, _I, _I, _I, _I, _I, _P, _I, _P, _I, _P, _I, _P, _F, _P, _I, _P, _P, _Z, _P]),
    "ftc_graph_attention_backward_workspace_bytes": (_Z, [_I, _I, _I, _I, _I, _I]),
    "ftc_graph_attention_backward": (_I, [_I, _P, _I, _P, _I, _I, _I, _I, _I, _P, _I, _P, _I, _P, _I, _P, _F, _P, _I, _P, _P, _I,
                                          _P, _I, _P, _I, _P, _I, _P, _Z, _P]),
    "ftc_reorder_workspace_bytes": (_Z, [_I, _I]),
    "ftc_degree_order": (_I, [_P, _I, _P, _P, _P, _Z, _P]),
    "ftc_order_by_key": (_I, [_I, _P, _P, _P, _P, _P, _Z, _P]),
    "ftc_label_propagation": (_I, [_P, _I, _P, _P, _Z, _P]),
    "ftc_permute_graph": (_I, [_P, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "ftc_permute_rows": (_I, [_I, _P, _I, _I, _I, _P, _P, _I, _P]),
    "ftc_degree_stats": (_I, [_P, _P, _P]),
    "ftc_plan_graph": (_I, [_I, _I, C.c_int64, C.c_int64, _I, _I, _P]),
}
EXPORTS = list(_SIGNATURES)


class FtcError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libftc error {code}: {msg}")
        self.code = code


class ftc_csr(C.Structure):
    _fields_ = [("n", C.c_int32), ("nnz", C.c_int32), ("row_ptr", C.c_void_p), ("col_idx", C.c_void_p)]


class ftc_windows(C.Structure):
    _fields_ = [("blk_h", C.c_int32), ("blk_w", C.c_int32), ("n_windows", C.c_int32),
                ("edge_to_row", C.c_void_p), ("edge_to_col", C.c_void_p),
                ("block_partition", C.c_void_p), ("win_col_ptr", C.c_void_p),
                ("win_cols", C.c_void_p), ("summary", C.c_void_p)]


_lib = None


def lib():
    """Load libftc.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(code):
    if code != FTC_OK:
        raise FtcError(code, lib().ftc_last_error().decode())


# Numbers and pointers go to the library as plain ints: the signatures above convert them.  A small call is bound by what
# happens here (one SpMM on 2048 nodes: 8.7 us from Python with a ctypes object per argument and a torch.cuda.Stream per call).
def _ptr(t):
    return t.data_ptr() if t is not None else None


# not part of torch's public interface: without it the handle comes from a stream object
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


# torch.cuda.current_device() without its check that CUDA is initialised, which a tensor on the GPU implies
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream():
    """Handle of torch's current stream on the current device."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dt(t):
    return _DTYPES[t.dtype]


class Graph:
    """Device CSR adjacency (int32) plus its C descriptor."""

    def __init__(self, row_ptr, col_idx):
        assert row_ptr.dtype == torch.int32 and col_idx.dtype == torch.int32
        assert row_ptr.is_cuda and col_idx.is_cuda and row_ptr.is_contiguous() and col_idx.is_contiguous()
        self.row_ptr, self.col_idx = row_ptr, col_idx
        self.n = row_ptr.numel() - 1
        self.nnz = col_idx.numel()
        self.c = ftc_csr(self.n, self.nnz, row_ptr.data_ptr(), col_idx.data_ptr() if self.nnz else 0)

    @staticmethod
    def from_numpy(row_ptr, col_idx, device="cuda"):
        return Graph(torch.from_numpy(row_ptr).to(device=device, dtype=torch.int32),
                     torch.from_numpy(col_idx).to(device=device, dtype=torch.int32))


class Windows:
    """Device arrays of the sparse graph transformation plus their C descriptor."""

    def __init__(self, g, blk_h=16, blk_w=8):
        dev = g.row_ptr.device
        self.blk_h, self.blk_w = blk_h, blk_w
        self.n_windows = (g.n + blk_h - 1) // blk_h
        i32 = dict(dtype=torch.int32, device=dev)
        self.edge_to_row = torch.empty(g.nnz, **i32)
        self.edge_to_col = torch.empty(g.nnz, **i32)
        self.block_partition = torch.empty(self.n_windows, **i32)
        self.win_col_ptr = torch.empty(self.n_windows + 1, **i32)
        self.win_cols = torch.empty(g.nnz, **i32)
        self.summary = torch.empty(2, dtype=torch.int64, device=dev)
        self.c = ftc_windows(blk_h, blk_w, self.n_windows, self.edge_to_row.data_ptr(),
                             self.edge_to_col.data_ptr(), self.block_partition.data_ptr(),
                             self.win_col_ptr.data_ptr(), self.win_cols.data_ptr(),
                             self.summary.data_ptr())


def _workspace(nbytes, device):
    # torch's caching allocator returns 512-byte aligned blocks
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _wref(w):
    return C.byref(w.c) if w is not None else None


def ftc_version():
    return lib().ftc_version()


def ftc_validate_csr(g):
    flag = torch.empty(1, dtype=torch.int32, device=g.row_ptr.device)
    _check(lib().ftc_validate_csr(C.byref(g.c), _ptr(flag), _stream()))
    return flag


class ftc_side_streams(C.Structure):
    _fields_ = [("stream", C.c_void_p * 3), ("fork", C.c_void_p), ("join", C.c_void_p * 3)]


class SideStreams:
    """Three streams and four events for ftc_build_windows_concurrent, created through torch (device plumbing
    only) on the current device at the default priority; keeps them alive as long as the object lives."""

    def __init__(self):
        self.streams = [torch.cuda.Stream() for _ in range(3)]
        self.events = [torch.cuda.Event(enable_timing=False) for _ in range(4)]
        for ev, st in zip(self.events, [torch.cuda.current_stream()] + self.streams):
            ev.record(st)              # torch creates the event handle at its first record
        self.c = ftc_side_streams()
        for i in range(3):
            self.c.stream[i] = self.streams[i].cuda_stream
            self.c.join[i] = self.events[1 + i].cuda_event
        self.c.fork = self.events[0].cuda_event


def ftc_build_windows(g, blk_h=16, blk_w=8, out=None, ws=None):
    w = out if out is not None else Windows(g, blk_h, blk_w)
    if ws is None:
        ws = _workspace(lib().ftc_build_windows_workspace_bytes(g.n, g.nnz, w.c.blk_h, w.c.blk_w), g.row_ptr.device)
    _check(lib().ftc_build_windows(C.byref(g.c), C.byref(w.c), _ptr(ws), ws.numel(), _stream()))
    return w


def ftc_build_windows_concurrent(g, side, blk_h=16, blk_w=8, out=None, ws=None):
    """side: a SideStreams (or None: the same as ftc_build_windows)."""
    w = out if out is not None else Windows(g, blk_h, blk_w)
    if ws is None:
        ws = _workspace(lib().ftc_build_windows_workspace_bytes(g.n, g.nnz, w.c.blk_h, w.c.blk_w), g.row_ptr.device)
    _check(lib().ftc_build_windows_concurrent(C.byref(g.c), C.byref(w.c), _ptr(ws), ws.numel(),
                                              C.byref(side.c) if side is not None else None, _stream()))
    return w


def ftc_gcn_norm(g, w=None, want_vals=True, want_dinv=True):
    dev = g.row_ptr.device
    vals = torch.empty(g.nnz, dtype=torch.float32, device=dev) if want_vals else None
    dinv = torch.empty(g.n, dtype=torch.float32, device=dev) if want_dinv else None
    _check(lib().ftc_gcn_norm(C.byref(g.c), _wref(w), _ptr(vals), _ptr(dinv), _stream()))
    return vals, dinv


def ftc_spmm(g, w, vals, X, out=None, out_dtype=torch.float32, relu=False, path=FTC_PATH_AUTO, ws=None,
             out_scale=None):
    D = X.shape[1]
    if out is None:
        out = torch.empty((g.n, D), dtype=out_dtype, device=X.device)
    if ws is None:
        ws = _workspace(lib().ftc_spmm_workspace_bytes(g.n, g.nnz, D), X.device)
    _check(lib().ftc_spmm(C.byref(g.c), _wref(w), _ptr(vals), _ptr(X), X.stride(0),
                          _dt(X), D, _ptr(out), out.stride(0),
                          _dt(out), _ptr(out_scale), 1 if relu else 0, path,
                          _ptr(ws), ws.numel(), _stream()))
    return out


def ftc_spmm_noalloc(g, w, vals, X, out, relu=False, path=FTC_PATH_AUTO, out_scale=None):
    """ftc_spmm on the library's built-in scratch buffer; `out` is the caller's (nothing is allocated here)."""
    D = X.shape[1]
    _check(lib().ftc_spmm_noalloc(C.byref(g.c), _wref(w), _ptr(vals), _ptr(X), X.stride(0),
                                  _dt(X), D, _ptr(out), out.stride(0),
                                  _dt(out), _ptr(out_scale), 1 if relu else 0, path,
                                  _stream()))
    return out


def ftc_sddmm(g, w, X, Y, row_scale=None, col_scale=None, alpha=1.0, out=None, path=FTC_PATH_AUTO, ws=None,
              cosine=False):
    D = X.shape[1]
    assert Y.shape[1] == D and X.stride(0) == Y.stride(0) and X.dtype == Y.dtype
    if out is None:
        out = torch.empty(g.nnz, dtype=torch.float32, device=X.device)
    if ws is None:
        ws = _workspace(lib().ftc_sddmm_workspace_bytes(g.n, g.nnz, D), X.device)
    _check(lib().ftc_sddmm(C.byref(g.c), _wref(w), _ptr(X), _ptr(Y), X.stride(0),
                           _dt(X), D, _ptr(row_scale), _ptr(col_scale),
                           alpha, 1 if cosine else 0, _ptr(out), path, _ptr(ws),
                           ws.numel(), _stream()))
    return out


def ftc_row_rnorm(H, out=None):
    if out is None:
        out = torch.empty(H.shape[0], dtype=torch.float32, device=H.device)
    _check(lib().ftc_row_rnorm(H.shape[0], _ptr(H), H.stride(0), _dt(H),
                               H.shape[1], _ptr(out), _stream()))
    return out


def ftc_edge_softmax(g, w, e_in, out=None, ws=None):
    if out is None:
        out = torch.empty_like(e_in)
    if ws is None:
        ws = _workspace(lib().ftc_edge_softmax_workspace_bytes(g.n, g.nnz) if w is not None else 0, e_in.device)
    _check(lib().ftc_edge_softmax(C.byref(g.c), _wref(w), _ptr(e_in), _ptr(out), _ptr(ws),
                                  ws.numel(), _stream()))
    return out


def ftc_update_gemm(X, W, out=None, out_dtype=torch.float32, relu=False, row_scale=None):
    n, d_in = X.shape
    d_out = W.shape[1]
    assert W.shape[0] == d_in and W.is_contiguous() and W.dtype == X.dtype
    if out is None:
        out = torch.empty((n, d_out), dtype=out_dtype, device=X.device)
    _check(lib().ftc_update_gemm(n, _ptr(X), X.stride(0), _dt(X),
                                 d_in, _ptr(W), d_out, _ptr(out),
                                 out.stride(0), _dt(out), _ptr(row_scale),
                                 1 if relu else 0, _stream()))
    return out


def ftc_gcn_layer(g, w, vals, X, W, relu=False, out=None, out_dtype=torch.float32, path=FTC_PATH_AUTO,
                  ws=None, dinv=None):
    n, d_in = X.shape
    d_out = W.shape[1]
    assert W.shape[0] == d_in and W.is_contiguous() and W.dtype == X.dtype
    if out is None:
        out = torch.empty((n, d_out), dtype=out_dtype, device=X.device)
    if ws is None:
        ws = _workspace(lib().ftc_gcn_layer_workspace_bytes(g.n, g.nnz, d_in, d_out), X.device)
    _check(lib().ftc_gcn_layer(C.byref(g.c), _wref(w), _ptr(vals), _ptr(dinv), _ptr(X), X.stride(0),
                               _dt(X), d_in, _ptr(W), d_out,
                               1 if relu else 0, _ptr(out), out.stride(0),
                               _dt(out), path, _ptr(ws), ws.numel(),
                               _stream()))
    return out


def ftc_agnn_layer(g, w, H, beta=1.0, out=None, out_dtype=torch.float32, edge_p=None, path=FTC_PATH_AUTO,
                   ws=None, row_z=None, out_f32=None):
    n, D = H.shape
    if out is None:
        out = torch.empty((n, D), dtype=out_dtype, device=H.device)
    if ws is None:
        ws = _workspace(lib().ftc_agnn_layer_workspace_bytes(g.n, g.nnz, D), H.device)
    _check(lib().ftc_agnn_layer(C.byref(g.c), _wref(w), _ptr(H), H.stride(0), _dt(H),
                                D, beta, _ptr(out), out.stride(0),
                                _dt(out), _ptr(edge_p), _ptr(row_z), _ptr(out_f32),
                                out_f32.stride(0) if out_f32 is not None else 0, path, _ptr(ws),
                                ws.numel(), _stream()))
    return out


# ---- backward pass (gradients are fp32 tensors) ----------------------------------------------------
def ftc_transpose_index(g, w=None):
    T = torch.empty(g.nnz, dtype=torch.int32, device=g.row_ptr.device)
    flag = torch.empty(1, dtype=torch.int32, device=g.row_ptr.device)
    _check(lib().ftc_transpose_index(C.byref(g.c), _wref(w), _ptr(T), _ptr(flag), _stream()))
    return T, flag


def ftc_edge_softmax_backward(g, w, p, dp, out=None, ws=None):
    if out is None:
        out = torch.empty_like(dp)
    if ws is None:
        ws = _workspace(lib().ftc_edge_softmax_workspace_bytes(g.n, g.nnz), dp.device)
    _check(lib().ftc_edge_softmax_backward(C.byref(g.c), _wref(w), _ptr(p), _ptr(dp), _ptr(out), _ptr(ws),
                                           ws.numel(), _stream()))
    return out


def ftc_weight_grad(X, G, ws=None):
    n, d_in = X.shape
    d_out = G.shape[1]
    assert G.dtype == torch.float32 and G.shape[0] == n
    dW = torch.empty((d_in, d_out), dtype=torch.float32, device=X.device)
    if ws is None:
        ws = _workspace(lib().ftc_weight_grad_workspace_bytes(n, d_in, d_out), X.device)
    _check(lib().ftc_weight_grad(n, _ptr(X), X.stride(0), _dt(X), d_in,
                                 _ptr(G), G.stride(0), d_out, _ptr(dW), _ptr(ws),
                                 ws.numel(), _stream()))
    return dW


def ftc_update_gemm_backward(X, W, dZ, Z=None, want_dX=True, dx_dtype=torch.float32, dX=None, ws=None):
    n, d_in = X.shape
    d_out = W.shape[1]
    assert dZ.dtype == torch.float32 and dZ.shape == (n, d_out)
    if dX is None and want_dX:
        dX = torch.empty((n, d_in), dtype=dx_dtype, device=X.device)
    dW = torch.empty((d_in, d_out), dtype=torch.float32, device=X.device)
    if ws is None:
        ws = _workspace(lib().ftc_update_gemm_backward_workspace_bytes(n, d_in, d_out), X.device)
    _check(lib().ftc_update_gemm_backward(
        n, _ptr(X), X.stride(0), _dt(X), d_in, _ptr(W), d_out,
        _ptr(Z), Z.stride(0) if Z is not None else 0, _dt(Z) if Z is not None else 0, _ptr(dZ),
        dZ.stride(0), _ptr(dX), dX.stride(0) if dX is not None else 0,
        _dt(dX) if dX is not None else 0, _ptr(dW), _ptr(ws), ws.numel(), _stream()))
    return dX, dW


def ftc_gcn_layer_backward(gT, wT, valsT, X, W, dY, Y=None, dinv=None, want_dX=True, path=FTC_PATH_AUTO, ws=None):
    n, d_in = X.shape
    d_out = W.shape[1]
    assert dY.dtype == torch.float32 and dY.shape == (n, d_out)
    dX = torch.empty((n, d_in), dtype=torch.float32, device=X.device) if want_dX else None
    dW = torch.empty((d_in, d_out), dtype=torch.float32, device=X.device)
    if ws is None:
        ws = _workspace(lib().ftc_gcn_layer_backward_workspace_bytes(gT.n, gT.nnz, d_in, d_out), X.device)
    _check(lib().ftc_gcn_layer_backward(
        C.byref(gT.c), _wref(wT), _ptr(valsT), _ptr(dinv), _ptr(X), X.stride(0), _dt(X),
        d_in, _ptr(W), d_out, _ptr(Y), Y.stride(0) if Y is not None else 0,
        _dt(Y) if Y is not None else 0, _ptr(dY), dY.stride(0), _ptr(dX),
        dX.stride(0) if dX is not None else 0, _ptr(dW), path, _ptr(ws), ws.numel(),
        _stream()))
    return dX, dW


def ftc_agnn_layer_backward(g, w, T, H, p, dY, beta=1.0, dH=None, dh_dtype=torch.float32, dbeta=None,
                            path=FTC_PATH_AUTO, ws=None):
    n, D = H.shape
    assert dY.dtype == H.dtype and dY.shape == H.shape and dY.stride(0) == H.stride(0)
    if dH is None:
        dH = torch.empty((n, D), dtype=dh_dtype, device=H.device)
    if dbeta is None:
        dbeta = torch.empty(1, dtype=torch.float32, device=H.device)
    if ws is None:
        ws = _workspace(lib().ftc_agnn_layer_backward_workspace_bytes(g.n, g.nnz, D), H.device)
    _check(lib().ftc_agnn_layer_backward(
        C.byref(g.c), _wref(w), _ptr(T), _ptr(H), H.stride(0), _dt(H), D,
        beta, _ptr(p), _ptr(dY), dY.stride(0), _ptr(dH), dH.stride(0),
        _dt(dH), _ptr(dbeta), path, _ptr(ws), ws.numel(), _stream()))
    return dH, dbeta


def ftc_agnn_layer_backward_fused(g, w, H, row_z, Y, dY, beta=1.0, dH=None, dh_dtype=torch.float32, dbeta=None, ws=None,
                                  pattern_flag=None):
    n, D = H.shape
    assert dY.dtype == H.dtype and dY.shape == H.shape and dY.stride(0) == H.stride(0) and Y.shape == H.shape
    if dH is None:
        dH = torch.empty((n, D), dtype=dh_dtype, device=H.device)
    if dbeta is None:
        dbeta = torch.empty(1, dtype=torch.float32, device=H.device)
    if ws is None:
        ws = _workspace(lib().ftc_agnn_layer_backward_fused_workspace_bytes(g.n, g.nnz, D), H.device)
    _check(lib().ftc_agnn_layer_backward_fused(
        C.byref(g.c), _wref(w), _ptr(H), H.stride(0), _dt(H), D, beta,
        _ptr(row_z), _ptr(Y), Y.stride(0), _dt(Y), _ptr(dY), dY.stride(0), _ptr(dH),
        dH.stride(0), _dt(dH), _ptr(dbeta), _ptr(pattern_flag), _ptr(ws), ws.numel(),
        _stream()))
    return dH, dbeta


# ---- graph transformer ----------------------------------------------------------------------------------
FTC_ACT_NONE, FTC_ACT_RELU, FTC_ACT_GELU, FTC_ACT_SILU = 0, 1, 2, 3


def _here(*tensors):
    """Handle of the current stream; the tensors are on its device."""
    dev = _current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{dev}")
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(dev)


def _ld(t, rows, cols, dtype=None):
    """Leading dimension of a rows x cols matrix whose rows are contiguous."""
    if t.shape != (rows, cols) or (dtype is not None and t.dtype != dtype):
        raise ValueError(f"expected {rows} x {cols}" + (f" of {dtype}" if dtype is not None else "") + f", got {tuple(t.shape)} of {t.dtype}")
    st, sc = t.stride()
    if cols > 1 and sc != 1:
        raise ValueError("rows must be contiguous")
    return st if rows > 1 else max(st, cols)


def _vector(t, numel, dtypes):
    if t.dim() != 1 or (numel is not None and t.numel() != numel) or t.dtype not in dtypes or not t.is_contiguous():
        raise ValueError(f"expected a contiguous vector of {numel} {dtypes}, got {tuple(t.shape)} of {t.dtype}")


def ftc_embedding(ids, E, scale=1.0, out=None, out_dtype=None):
    """scale * E[ids], zeros for ids outside the table; out in E's type unless given."""
    n, (vocab, D) = ids.numel(), E.shape
    if out is None:
        out = torch.empty((n, D), dtype=out_dtype or E.dtype, device=E.device)
    _vector(ids, n, (torch.int32,))
    stream = _here(ids, E, out)
    _check(lib().ftc_embedding(n, _ptr(ids), vocab, _ptr(E), _ld(E, vocab, D), _dt(E), D, scale, _ptr(out), _ld(out, n, D), _dt(out),
                               stream))
    return out


def ftc_embedding_backward(ids, dOut, vocab, scale=1.0, dE=None, de_dtype=torch.float32, ws=None):
    n, D = dOut.shape
    if dE is None:
        dE = torch.empty((vocab, D), dtype=de_dtype, device=dOut.device)
    if ws is None:
        ws = _workspace(lib().ftc_embedding_backward_workspace_bytes(n, vocab, D), dOut.device)
    _vector(ids, n, (torch.int32,))
    stream = _here(ids, dOut, dE, ws)
    _check(lib().ftc_embedding_backward(n, _ptr(ids), vocab, _ptr(dOut), _ld(dOut, n, D), _dt(dOut), D, scale, _ptr(dE),
                                        _ld(dE, vocab, D), _dt(dE), _ptr(ws), ws.numel(), stream))
    return dE


def slope_like(t):
    """A tensor of t's shape for the activation slopes that ftc_linear keeps for inputs of t's type."""
    return torch.empty(t.shape, dtype=torch.float32 if t.dtype == torch.float32 else torch.int16, device=t.device)


def ftc_linear(X, W, bias=None, act=FTC_ACT_NONE, residual=None, out=None, out_dtype=None, slope=None, ws=None):
    """act(X W + bias) + residual; out in X's type unless given.  slope: see slope_like."""
    n, d_in = X.shape
    d_out = W.shape[1]
    if out is None:
        out = torch.empty((n, d_out), dtype=out_dtype or X.dtype, device=X.device)
    if ws is None:
        ws = _workspace(lib().ftc_linear_workspace_bytes(n, d_in, d_out), X.device)
    stream = _here(X, W, bias, residual, out, slope, ws)
    _ld(W, d_in, d_out, X.dtype)
    if not W.is_contiguous():
        raise ValueError("W must be contiguous")
    if bias is not None:
        _vector(bias, d_out, (X.dtype,))
    sdt = torch.float32 if X.dtype == torch.float32 else torch.int16
    _check(lib().ftc_linear(n, _ptr(X), _ld(X, n, d_in), _dt(X), d_in, _ptr(W), d_out, _ptr(bias), act, _ptr(residual),
                            _ld(residual, n, d_out, X.dtype) if residual is not None else 0, _ptr(slope),
                            _ld(slope, n, d_out, sdt) if slope is not None else 0, _ptr(out), _ld(out, n, d_out), _dt(out), _ptr(ws),
                            ws.numel(), stream))
    return out


def ftc_linear_backward(X, W, dZ, slope=None, want_dX=True, want_dW=True, want_db=True, dX=None, dx_dtype=None, dW=None, db=None,
                        dw_dtype=torch.float32, dX_add=None, ws=None):
    """(dX, dW, db); dX in X's type unless given, dX_add (may be dX) added to it; dW and db share a type (dw_dtype where they are not given)."""
    n, d_in = X.shape
    d_out = W.shape[1]
    if dX is None and want_dX:
        dX = torch.empty((n, d_in), dtype=dx_dtype or X.dtype, device=X.device)
    wdt = dW.dtype if dW is not None else db.dtype if db is not None else dw_dtype
    if dW is None and want_dW:
        dW = torch.empty((d_in, d_out), dtype=wdt, device=X.device)
    if db is None and want_db:
        db = torch.empty(d_out, dtype=wdt, device=X.device)
    if ws is None:
        ws = _workspace(lib().ftc_linear_backward_workspace_bytes(n, d_in, d_out), X.device)
    stream = _here(X, W, dZ, slope, dX_add, dX, dW, db, ws)
    _ld(W, d_in, d_out, X.dtype)
    if not W.is_contiguous() or (dW is not None and not dW.is_contiguous()):
        raise ValueError("W and dW must be contiguous")
    if dW is not None:
        _ld(dW, d_in, d_out, wdt)
    if db is not None:
        _vector(db, d_out, (wdt,))
    sdt = torch.float32 if X.dtype == torch.float32 else torch.int16
    _check(lib().ftc_linear_backward(n, _ptr(X), _ld(X, n, d_in), _dt(X), d_in, _ptr(W), d_out, _ptr(slope),
                                     _ld(slope, n, d_out, sdt) if slope is not None else 0, _ptr(dZ), _ld(dZ, n, d_out, X.dtype),
                                     _ptr(dX_add), _ld(dX_add, n, d_in, X.dtype) if dX_add is not None else 0, _ptr(dX),
                                     _ld(dX, n, d_in) if dX is not None else 0, _dt(dX) if dX is not None else 0, _ptr(dW),
                                     _ptr(db), _DTYPES[wdt], _ptr(ws), ws.numel(), stream))
    return dX, dW, db


def _contiguous(t, shape, dtype):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"expected a contiguous {shape} tensor of {dtype}, got {tuple(t.shape)} of {t.dtype}")


def ftc_grouped_linear(X, W, group_ptr, bias=None, act=FTC_ACT_NONE, residual=None, out=None, out_dtype=None, slope=None, ws=None):
    """act(X W[g] + bias[g]) + residual for the rows group_ptr[g] .. group_ptr[g+1] of every group g; W groups x d_in x d_out, bias groups x d_out, group_ptr
    int32.  out in X's type unless given; rows of no group keep what out has there.  slope: see slope_like."""
    (n, d_in), (groups, _, d_out), dt, L = X.shape, W.shape, X.dtype, lib()
    if out is None:
        out = torch.empty((n, d_out), dtype=out_dtype or dt, device=X.device)
    if ws is None:
        ws = _workspace(L.ftc_grouped_linear_workspace_bytes(n, groups, d_in, d_out), X.device)
    stream = _here(X, W, group_ptr, bias, residual, out, slope, ws)
    _vector(group_ptr, groups + 1, (torch.int32,))
    _contiguous(W, (groups, d_in, d_out), dt)
    if bias is not None:
        _contiguous(bias, (groups, d_out), dt)
    ldr = _ld(residual, n, d_out, dt) if residual is not None else 0
    lds = _ld(slope, n, d_out, torch.float32 if dt == torch.float32 else torch.int16) if slope is not None else 0
    _check(L.ftc_grouped_linear(n, group_ptr.data_ptr(), groups, X.data_ptr(), _ld(X, n, d_in), _dt(X), d_in, W.data_ptr(), d_out, _ptr(bias), act,
                                _ptr(residual), ldr, _ptr(slope), lds, out.data_ptr(), _ld(out, n, d_out), _dt(out), ws.data_ptr(), ws.numel(), stream))
    return out


def ftc_grouped_linear_backward(X, W, group_ptr, dZ, slope=None, want_dX=True, want_dW=True, want_db=True, dX=None, dx_dtype=None, dW=None, db=None,
                                dw_dtype=torch.float32, dX_add=None, ws=None):
    """(dX, dW, db) of ftc_grouped_linear, with the types that ftc_linear_backward has; rows of no group keep what dX has there."""
    (n, d_in), (groups, _, d_out) = X.shape, W.shape
    if dX is None and want_dX:
        dX = torch.empty((n, d_in), dtype=dx_dtype or X.dtype, device=X.device)
    wdt = dW.dtype if dW is not None else db.dtype if db is not None else dw_dtype
    if dW is None and want_dW:
        dW = torch.empty((groups, d_in, d_out), dtype=wdt, device=X.device)
    if db is None and want_db:
        db = torch.empty((groups, d_out), dtype=wdt, device=X.device)
    if ws is None:
        ws = _workspace(lib().ftc_grouped_linear_backward_workspace_bytes(n, groups, d_in, d_out), X.device)
    stream = _here(X, W, group_ptr, dZ, slope, dX_add, dX, dW, db, ws)
    _vector(group_ptr, groups + 1, (torch.int32,))
    _contiguous(W, (groups, d_in, d_out), X.dtype)
    if dW is not None:
        _contiguous(dW, (groups, d_in, d_out), wdt)
    if db is not None:
        _contiguous(db, (groups, d_out), wdt)
    sdt = torch.float32 if X.dtype == torch.float32 else torch.int16
    _check(lib().ftc_grouped_linear_backward(n, _ptr(group_ptr), groups, _ptr(X), _ld(X, n, d_in), _dt(X), d_in, _ptr(W), d_out, _ptr(slope),
                                             _ld(slope, n, d_out, sdt) if slope is not None else 0, _ptr(dZ), _ld(dZ, n, d_out, X.dtype),
                                             _ptr(dX_add), _ld(dX_add, n, d_in, X.dtype) if dX_add is not None else 0, _ptr(dX),
                                             _ld(dX, n, d_in) if dX is not None else 0, _dt(dX) if dX is not None else 0, _ptr(dW),
                                             _ptr(db), _DTYPES[wdt], _ptr(ws), ws.numel(), stream))
    return dX, dW, db


class ftc_grad(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("ldo", C.c_int64),
                ("dtype", C.c_int32)]


def _as_matrix(t):
    """(rows, cols, ld) of a contiguous tensor of any shape, or of a matrix whose rows are contiguous."""
    if t.is_contiguous():
        return 1, t.numel(), t.numel()
    if t.dim() != 2 or t.stride(1) != 1 and t.shape[1] > 1 or t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError(f"expected a contiguous tensor or a matrix with contiguous rows, got strides {t.stride()}")
    return t.shape[0], t.shape[1], t.stride(0)


def _overlap(a, b):
    """Whether two tensors as (address, bytes of a number, rows, cols, ld) share memory; rows of one distance can lie beside each other."""
    (pa, ea, ra, ca, la), (pb, eb, rb, cb, lb) = a, b
    end = lambda p, e, r, c, ld: p + ((r - 1) * ld + c) * e
    if end(*a) <= pb or end(*b) <= pa:
        return False
    if la * ea != lb * eb or ra == 1 or rb == 1:
        return True
    d = (pb - pa) % (la * ea)   # where a row of b begins in a row of a, and where a row of a begins in a row of b
    return d < ca * ea or (la * ea - d) % (la * ea) < cb * eb


class GradList:
    """Gradients (and where the clipped ones go: `out`, in place unless given) and their descriptors for ftc_grad_norm and ftc_clip_grad_norm: for a program whose
    gradients stay where they are.  The tensors share no memory, but that a gradient may be its own `out`."""

    def __init__(self, grads, out=None):
        self.grads = list(grads)
        self.out = self.grads if out is None else list(out)
        if len(self.out) != len(self.grads):
            raise ValueError(f"{len(self.out)} outputs for {len(self.grads)} gradients")
        devices = {t.device for t in self.grads + self.out}
        if len(devices) > 1:
            raise ValueError(f"gradients and outputs on {len(devices)} devices")
        self.first = self.grads[0] if self.grads else None   # stands for all of them
        self.c = (ftc_grad * len(self.grads))()
        spans = []
        for i, (g, o) in enumerate(zip(self.grads, self.out)):
            if o.shape != g.shape or o.dtype != g.dtype:
                raise ValueError(f"gradient {i} is {tuple(g.shape)} of {g.dtype}, its output {tuple(o.shape)} of {o.dtype}")
            if g.is_contiguous() and o.is_contiguous():
                (rows, cols, ld), (_, _, ldo) = _as_matrix(g), _as_matrix(o)
            else:
                two = lambda t: (t.shape[0], t.shape[1], t.stride(0) if t.shape[0] > 1 else t.shape[1]) if t.dim() == 2 and t.is_contiguous() else _as_matrix(t)
                if g.dim() != 2:
                    raise ValueError(f"gradient {i}: a tensor that is not a matrix, and its output, are contiguous")
                (rows, cols, ld), (_, _, ldo) = two(g), two(o)
            self.c[i] = ftc_grad(_ptr(g), _ptr(o), rows, cols, ld, ldo, _dt(g))
            if g.numel():
                e = g.element_size()
                spans.append((g.data_ptr(), e, rows, cols, ld))
                if o.data_ptr() != g.data_ptr() or ld != ldo:
                    spans.append((o.data_ptr(), e, rows, cols, ldo))
        spans.sort()
        ends = []                    # those that reach beyond the next one's beginning
        for s in spans:
            ends = [t for t in ends if t[0] + ((t[2] - 1) * t[4] + t[3]) * t[1] > s[0]]
            if any(_overlap(t, s) for t in ends):
                raise ValueError("two of the gradients and outputs share memory")
            ends.append(s)

    def workspace_bytes(self):
        return lib().ftc_grad_norm_workspace_bytes(len(self.grads))


def _grad_call(grads, norm, ws):
    if not isinstance(grads, GradList):
        grads = GradList(grads)
    dev = norm.device if norm is not None else grads.first.device if grads.grads else "cuda"
    if norm is None:
        norm = torch.empty(1, dtype=torch.float32, device=dev)
    _vector(norm, 1, (torch.float32,))
    if ws is None:
        ws = _workspace(grads.workspace_bytes(), dev)
    return grads, norm, ws, _here(norm, ws, grads.first)


def ftc_grad_norm(grads, scale=1.0, norm=None, ws=None):
    """|scale| times the norm over all gradients (a GradList, or tensors), one fp32 number on the device."""
    grads, norm, ws, stream = _grad_call(grads, norm, ws)
    _check(lib().ftc_grad_norm(grads.c, len(grads.grads), scale, _ptr(norm), _ptr(ws), ws.numel(), stream))
    return norm


def ftc_clip_grad_norm(grads, max_norm, scale=1.0, norm=None, ws=None):
    """scale min(1, max_norm / norm) times every gradient (a GradList, or tensors: in place), norm as ftc_grad_norm has it, which is what comes back."""
    grads, norm, ws, stream = _grad_call(grads, norm, ws)
    _check(lib().ftc_clip_grad_norm(grads.c, len(grads.grads), max_norm, scale, _ptr(norm), _ptr(ws), ws.numel(), stream))
    return norm


FTC_NORM_NONE, FTC_NORM_RMS, FTC_NORM_LAYER = 0, 1, 2


class ftc_block(C.Structure):
    _fields_ = [("n", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32), ("post", C.c_int32), ("pre", C.c_int32), ("eps", C.c_float),
                ("x_scale", C.c_float), ("X", C.c_void_p), ("F", C.c_void_p), ("gate", C.c_void_p), ("post_w", C.c_void_p),
                ("post_b", C.c_void_p), ("pre_w", C.c_void_p), ("pre_b", C.c_void_p), ("ldx", C.c_int32), ("ldf", C.c_int32),
                ("ldg", C.c_int32)]


class ftc_block_grads(C.Structure):
    _fields_ = [("dX", C.c_void_p), ("dF", C.c_void_p), ("dgate", C.c_void_p), ("dpost_w", C.c_void_p), ("dpost_b", C.c_void_p),
                ("dpre_w", C.c_void_p), ("dpre_b", C.c_void_p), ("lddx", C.c_int32), ("lddf", C.c_int32), ("lddg", C.c_int32),
                ("dw_dtype", C.c_int32)]


BlockGrads = collections.namedtuple("BlockGrads", "dX dF dgate dpost_w dpost_b dpre_w dpre_b")


# ftc_block as bytes: a call on a few rows is bound by what happens here (a ctypes structure of these 17 fields takes 1.2 us more)
_BLOCK = struct.Struct("@5i2f7P3i0P")


def _block(X, F, x_scale, post, post_w, post_b, gate, pre, pre_w, pre_b, eps):
    n, d = X.shape
    dt, row, ldg = X.dtype, (d,), 0
    for v in (post_w, post_b, pre_w, pre_b):
        if v is not None and (v.shape != row or v.dtype != dt or not v.is_contiguous()):
            _vector(v, d, (dt,))
    if gate is not None:
        if gate.dim() == 1:
            _vector(gate, d, (dt,))
        else:
            ldg = _ld(gate, n, d, dt)
            if ldg < d:
                raise ValueError("the rows of gate overlap (one gate for all rows is a vector)")
    at = lambda t: 0 if t is None else t.data_ptr()
    return _BLOCK.pack(n, d, _DTYPES[dt], post, pre, eps, x_scale, X.data_ptr(), at(F), at(gate), at(post_w), at(post_b), at(pre_w), at(pre_b),
                       _ld(X, n, d), 0 if F is None else _ld(F, n, d, dt), ldg)


def _stats(stats, n):
    if stats.dtype != torch.float32 or stats.shape != (n, 4) or not stats.is_contiguous():
        raise ValueError("stats is a contiguous n x 4 fp32 tensor")


def ftc_block_norm(X, F=None, x_scale=1.0, post=FTC_NORM_NONE, post_w=None, post_b=None, gate=None, pre=FTC_NORM_RMS, pre_w=None,
                   pre_b=None, eps=1e-5, H=None, U=None, stats=None):
    """(H, U): h = x_scale X + gate Npost(F) and Npre(h), in X's type.  gate: d numbers, or n x d.  H is None without F unless it is given, U without
    a norm `pre`.  stats: n x 4 fp32, for the backward pass."""
    n, d = X.shape
    if H is None and (F is not None or pre == FTC_NORM_NONE):
        H = torch.empty((n, d), dtype=X.dtype, device=X.device)
    if U is None and pre != FTC_NORM_NONE:
        U = torch.empty((n, d), dtype=X.dtype, device=X.device)
    if stats is not None:
        _stats(stats, n)
    stream = _here(X, F, post_w, post_b, gate, pre_w, pre_b, H, U, stats)
    b = _block(X, F, x_scale, post, post_w, post_b, gate, pre, pre_w, pre_b, eps)
    _check(lib().ftc_block_norm(b, _ptr(H), _ld(H, n, d, X.dtype) if H is not None else 0, _ptr(U),
                                _ld(U, n, d, X.dtype) if U is not None else 0, _ptr(stats), stream))
    return H, U


def ftc_block_norm_backward(X, stats, dH=None, dU=None, F=None, x_scale=1.0, post=FTC_NORM_NONE, post_w=None, post_b=None, gate=None,
                            pre=FTC_NORM_RMS, pre_w=None, pre_b=None, eps=1e-5, dX=None, dF=None, dgate=None, dpost_w=None, dpost_b=None,
                            dpre_w=None, dpre_b=None, want=("dX", "dF", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b"),
                            dw_dtype=torch.float32, ws=None):
    """BlockGrads, the block as ftc_block_norm was given it.  Of the names in `want` those come back that the block has, the others as None; dX, dF and
    the gradient of an n x d gate in X's type, the other ones in dw_dtype unless one of them is given, whose type is that of all."""
    n, d = X.shape
    dt, rows = X.dtype, gate is not None and gate.dim() != 1
    vectors = [t for t in ((None if rows else dgate), dpost_w, dpost_b, dpre_w, dpre_b) if t is not None]
    wdt = vectors[0].dtype if vectors else dw_dtype
    for v in vectors:
        _vector(v, d, (wdt,))

    def out(t, name, there, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=X.device) if t is None and there and name in want else t
    dX, dF = out(dX, "dX", True, (n, d), dt), out(dF, "dF", F is not None, (n, d), dt)
    dgate = out(dgate, "dgate", gate is not None, (n, d) if rows else d, dt if rows else wdt)
    dpost_w, dpost_b = out(dpost_w, "dpost_w", post_w is not None, d, wdt), out(dpost_b, "dpost_b", post_b is not None, d, wdt)
    dpre_w, dpre_b = out(dpre_w, "dpre_w", pre_w is not None, d, wdt), out(dpre_b, "dpre_b", pre_b is not None, d, wdt)
    if ws is None:
        ws = _workspace(lib().ftc_block_norm_backward_workspace_bytes(n, d), X.device)
    if stats is not None:
        _stats(stats, n)
    stream = _here(X, F, post_w, post_b, gate, pre_w, pre_b, stats, dH, dU, dX, dF, dgate, dpost_w, dpost_b, dpre_w, dpre_b, ws)
    b = _block(X, F, x_scale, post, post_w, post_b, gate, pre, pre_w, pre_b, eps)
    ld = lambda t: _ld(t, n, d, dt) if t is not None else 0
    g = ftc_block_grads(_ptr(dX), _ptr(dF), _ptr(dgate), _ptr(dpost_w), _ptr(dpost_b), _ptr(dpre_w), _ptr(dpre_b), ld(dX), ld(dF),
                        ld(dgate) if rows else 0, _DTYPES[wdt])
    _check(lib().ftc_block_norm_backward(b, _ptr(stats), _ptr(dH), ld(dH), _ptr(dU), ld(dU), C.byref(g), _ptr(ws), ws.numel(), stream))
    return BlockGrads(dX, dF, dgate, dpost_w, dpost_b, dpre_w, dpre_b)


def _attention_sizes(Q, K, V, q_ptr, kv_ptr, heads, kv_heads, kv_mask):
    if heads < 1 or Q.dim() != 2 or Q.shape[1] % heads:
        raise ValueError("Q has heads * D columns")
    n_q, D, n_kv, graphs = Q.shape[0], Q.shape[1] // heads, K.shape[0], q_ptr.numel() - 1
    _vector(q_ptr, graphs + 1, (torch.int32,))
    _vector(kv_ptr, graphs + 1, (torch.int32,))
    if kv_mask is not None:
        _vector(kv_mask, n_kv, (torch.uint8, torch.bool))
    return n_q, n_kv, graphs, heads, kv_heads, D


def ftc_graph_attention(Q, K, V, q_ptr, kv_ptr, heads, kv_heads=None, scale=None, kv_mask=None, out=None, lse=None, ws=None):
    """Attention inside every graph of a packed batch; Q n_q x (heads D), K and V n_kv x (kv_heads D).  scale: 1 / sqrt(D) unless
    given.  lse: n_q x heads fp32, for the backward pass."""
    kv_heads = heads if kv_heads is None else kv_heads
    sizes = n_q, n_kv, graphs, _, _, D = _attention_sizes(Q, K, V, q_ptr, kv_ptr, heads, kv_heads, kv_mask)
    if out is None:
        out = torch.empty((n_q, heads * D), dtype=Q.dtype, device=Q.device)
    if ws is None:
        ws = _workspace(lib().ftc_graph_attention_workspace_bytes(*sizes), Q.device)
    stream = _here(Q, K, V, q_ptr, kv_ptr, kv_mask, out, lse, ws)
    dt = Q.dtype
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != (n_q, heads) or not lse.is_contiguous()):
        raise ValueError("lse is a contiguous n_q x heads fp32 tensor")
    _check(lib().ftc_graph_attention(n_q, _ptr(q_ptr), n_kv, _ptr(kv_ptr), graphs, heads, kv_heads, D, _DTYPES[dt],
                                     _ptr(Q), _ld(Q, n_q, heads * D), _ptr(K), _ld(K, n_kv, kv_heads * D, dt), _ptr(V),
                                     _ld(V, n_kv, kv_heads * D, dt), _ptr(kv_mask), D ** -0.5 if scale is None else scale, _ptr(out),
                                     _ld(out, n_q, heads * D, dt), _ptr(lse), _ptr(ws), ws.numel(), stream))
    return out


def ftc_graph_attention_backward(Q, K, V, q_ptr, kv_ptr, out, lse, dOut, heads, kv_heads=None, scale=None, kv_mask=None, dQ=None,
                                 dK=None, dV=None, ws=None):
    """(dQ, dK, dV) in Q's type."""
    kv_heads = heads if kv_heads is None else kv_heads
    sizes = n_q, n_kv, graphs, _, _, D = _attention_sizes(Q, K, V, q_ptr, kv_ptr, heads, kv_heads, kv_mask)
    dt = Q.dtype
    new = lambda t: torch.empty(t.shape, dtype=dt, device=Q.device)
    dQ, dK, dV = dQ if dQ is not None else new(Q), dK if dK is not None else new(K), dV if dV is not None else new(V)
    if ws is None:
        ws = _workspace(lib().ftc_graph_attention_backward_workspace_bytes(*sizes), Q.device)
    stream = _here(Q, K, V, q_ptr, kv_ptr, kv_mask, out, lse, dOut, dQ, dK, dV, ws)
    if lse.dtype != torch.float32 or lse.shape != (n_q, heads) or not lse.is_contiguous():
        raise ValueError("lse is a contiguous n_q x heads fp32 tensor")
    hd, kd = heads * D, kv_heads * D
    _check(lib().ftc_graph_attention_backward(
        n_q, _ptr(q_ptr), n_kv, _ptr(kv_ptr), graphs, heads, kv_heads, D, _DTYPES[dt], _ptr(Q), _ld(Q, n_q, hd), _ptr(K), _ld(K, n_kv, kd, dt),
        _ptr(V), _ld(V, n_kv, kd, dt), _ptr(kv_mask), D ** -0.5 if scale is None else scale, _ptr(out), _ld(out, n_q, hd, dt), _ptr(lse),
        _ptr(dOut), _ld(dOut, n_q, hd, dt), _ptr(dQ), _ld(dQ, n_q, hd, dt), _ptr(dK), _ld(dK, n_kv, kd, dt), _ptr(dV),
        _ld(dV, n_kv, kd, dt), _ptr(ws), ws.numel(), stream))
    return dQ, dK, dV


# ---- locality reordering ------------------------------------------------------------------------------
FTC_ORDER_DEGREE, FTC_ORDER_DEGREE_CLASSES, FTC_ORDER_COMMUNITIES = 0, 1, 2


def ftc_degree_order(g, mode=FTC_ORDER_DEGREE, ws=None):
    dev = g.row_ptr.device
    perm = torch.empty(g.n, dtype=torch.int32, device=dev)
    inv = torch.empty(g.n, dtype=torch.int32, device=dev)
    if ws is None:
        ws = _workspace(lib().ftc_reorder_workspace_bytes(g.n, g.nnz), dev)
    _check(lib().ftc_degree_order(C.byref(g.c), mode, _ptr(perm), _ptr(inv), _ptr(ws),
                                  ws.numel(), _stream()))
    return perm, inv


def ftc_order_by_key(keys, ws=None):
    """Returns (perm, inv, flag): ascending keys, ties by id."""
    n = keys.numel()
    dev = keys.device
    perm = torch.empty(n, dtype=torch.int32, device=dev)
    inv = torch.empty(n, dtype=torch.int32, device=dev)
    flag = torch.empty(1, dtype=torch.int32, device=dev)
    if ws is None:
        ws = _workspace(lib().ftc_reorder_workspace_bytes(n, 0), dev)
    _check(lib().ftc_order_by_key(n, _ptr(keys), _ptr(perm), _ptr(inv), _ptr(flag), _ptr(ws),
                                  ws.numel(), _stream()))
    return perm, inv, flag


def ftc_label_propagation(g, rounds=10, ws=None):
    dev = g.row_ptr.device
    labels = torch.empty(g.n, dtype=torch.int32, device=dev)
    if ws is None:
        ws = _workspace(lib().ftc_reorder_workspace_bytes(g.n, g.nnz), dev)
    _check(lib().ftc_label_propagation(C.byref(g.c), rounds, _ptr(labels), _ptr(ws), ws.numel(),
                                       _stream()))
    return labels


def ftc_permute_graph(g, perm, inv, ws=None):
    """Returns (relabelled Graph, flag tensor: 0 if (perm, inv) is a permutation and its inverse)."""
    dev = g.row_ptr.device
    row_ptr = torch.empty(g.n + 1, dtype=torch.int32, device=dev)
    col_idx = torch.empty(g.nnz, dtype=torch.int32, device=dev)
    flag = torch.empty(1, dtype=torch.int32, device=dev)
    if ws is None:
        ws = _workspace(lib().ftc_reorder_workspace_bytes(g.n, g.nnz), dev)
    _check(lib().ftc_permute_graph(C.byref(g.c), _ptr(perm), _ptr(inv), _ptr(row_ptr), _ptr(col_idx), _ptr(flag),
                                   _ptr(ws), ws.numel(), _stream()))
    return Graph(row_ptr, col_idx), flag


def ftc_permute_rows(X, index, out=None):
    n, D = X.shape
    if out is None:
        out = torch.empty((n, D), dtype=X.dtype, device=X.device)
    _check(lib().ftc_permute_rows(n, _ptr(X), X.stride(0), _dt(X), D,
                                  _ptr(index), _ptr(out), out.stride(0), _stream()))
    return out


# ---- per-graph plan -------------------------------------------------------------------------------------
FTC_ORDER_NONE = -1


class ftc_plan(C.Structure):
    _fields_ = [("skew", C.c_double), ("reuse", C.c_double), ("reorder", C.c_int32), ("agnn_single_pass", C.c_int32),
                ("agnn_backward_single_pass", C.c_int32), ("spmm_mfma_windows", C.c_int32),
                ("sddmm_mfma_windows", C.c_int32), ("mfma_min_reuse", C.c_float)]


def ftc_degree_stats(g):
    stats = torch.empty(2, dtype=torch.int64, device=g.row_ptr.device)
    _check(lib().ftc_degree_stats(C.byref(g.c), _ptr(stats), _stream()))
    return stats


def ftc_plan_graph(n, nnz, sum_deg_sq, sum_uniq, D, dtype):
    """Host-only: the per-graph choices as a dict (dtype: a torch dtype)."""
    plan = ftc_plan()
    _check(lib().ftc_plan_graph(n, nnz, C.c_int64(int(sum_deg_sq)), C.c_int64(int(sum_uniq)),
                                D, _DTYPES[dtype], C.byref(plan)))
    return {name: getattr(plan, name) for name, _ in ftc_plan._fields_}
