"""Thin ctypes binding of librtlynx.so: argument marshalling only.

Same entry points as include/rtlynx.h. Tensors are torch CUDA tensors (used for device memory
and the current stream); every step of the path runs inside the library's HIP kernels. There is
no fallback: a missing library or a non-zero status raises.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librtlynx.so")

COMP_NONE, COMP_GROUP, COMP_ROW, COMP_TENSOR = 0, 1, 2, 3
COMP = {"none": COMP_NONE, "group": COMP_GROUP, "row": COMP_ROW, "tensor": COMP_TENSOR}

SYMBOLS = ["rtl_sparsify_pack_workspace", "rtl_sparsify_pack", "rtl_packed_linear_workspace",
           "rtl_packed_linear", "rtl_sparse_linear_workspace", "rtl_sparse_linear", "rtl_sparse_linear_static",
           "rtl_sparse_lora_linear_workspace", "rtl_sparse_lora_linear",
           "rtl_dense_linear_workspace", "rtl_dense_linear",
           "rtl_quantize_fp8", "rtl_sparsify_pack_fp8_workspace", "rtl_sparsify_pack_fp8",
           "rtl_sparse_linear_fp8_workspace", "rtl_sparse_linear_fp8",
           "rtl_sparse_lora_linear_fp8_workspace", "rtl_sparse_lora_linear_fp8",
           "rtl_quantize_mxfp4", "rtl_dequantize_mxfp4", "rtl_mxfp4_packed_linear_workspace", "rtl_mxfp4_packed_linear",
           "rtl_mxfp4_linear_workspace", "rtl_mxfp4_linear",
           "rtl_grouped_clear", "rtl_grouped_linear", "rtl_grouped_linear_dgrad", "rtl_grouped_linear_wgrad_workspace", "rtl_grouped_linear_wgrad",
           "rtl_grouped_mxfp4_linear_workspace", "rtl_grouped_mxfp4_linear",
           "rtl_diag_matrix_rate", "rtl_diag_fill_rate", "rtl_diag_pack_sweep", "rtl_diag_tile_plan", "rtl_init", "rtl_status_str", "rtl_version"]

_lib = None


class RtlError(RuntimeError):
    def __init__(self, status, where):
        self.status = int(status)
        super().__init__("%s failed: %s" % (where, status_str(status)))


def lib():
    """Load librtlynx.so (built in-tree by paper_2605_26632_amd/build.py). Raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("librtlynx.so is not built: run `python -m paper_2605_26632_amd.build` "
                               "(or __graft_entry__.build()) first; there is no fallback path")
        L = C.CDLL(LIB_PATH)
        i64, vp, sz, fl, ci = C.c_int64, C.c_void_p, C.c_size_t, C.c_float, C.c_int
        L.rtl_sparsify_pack_workspace.argtypes = [i64, i64, ci]
        L.rtl_sparsify_pack_workspace.restype = sz
        L.rtl_sparsify_pack.argtypes = [vp, i64, i64, i64, ci, fl, vp, vp, vp, vp, sz, vp]
        L.rtl_sparsify_pack.restype = ci
        L.rtl_packed_linear_workspace.argtypes = [i64, i64, i64]
        L.rtl_packed_linear_workspace.restype = sz
        L.rtl_packed_linear.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, vp, sz, vp]
        L.rtl_packed_linear.restype = ci
        L.rtl_sparse_linear_workspace.argtypes = [i64, i64, i64, ci]
        L.rtl_sparse_linear_workspace.restype = sz
        L.rtl_sparse_linear.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, ci, fl, vp, sz, vp]
        L.rtl_sparse_linear.restype = ci
        L.rtl_sparse_linear_static.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, ci, fl, vp]
        L.rtl_sparse_linear_static.restype = ci
        L.rtl_sparse_lora_linear_workspace.argtypes = [i64, i64, i64, i64, ci]
        L.rtl_sparse_lora_linear_workspace.restype = sz
        L.rtl_sparse_lora_linear.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i64,
                                             i64, i64, ci, fl, vp, sz, vp]
        L.rtl_sparse_lora_linear.restype = ci
        L.rtl_dense_linear_workspace.argtypes = [i64, i64, i64]
        L.rtl_dense_linear_workspace.restype = sz
        L.rtl_dense_linear.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, vp, sz, vp]
        L.rtl_dense_linear.restype = ci
        L.rtl_quantize_fp8.argtypes = [vp, i64, i64, i64, vp, i64, vp]
        L.rtl_quantize_fp8.restype = ci
        L.rtl_sparsify_pack_fp8_workspace.argtypes = [i64, i64, ci]
        L.rtl_sparsify_pack_fp8_workspace.restype = sz
        L.rtl_sparsify_pack_fp8.argtypes = [vp, i64, i64, i64, ci, fl, vp, vp, vp, vp, vp, sz, vp]
        L.rtl_sparsify_pack_fp8.restype = ci
        L.rtl_sparse_linear_fp8_workspace.argtypes = [i64, i64, i64, ci]
        L.rtl_sparse_linear_fp8_workspace.restype = sz
        L.rtl_sparse_linear_fp8.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, ci, fl, vp, sz, vp]
        L.rtl_sparse_linear_fp8.restype = ci
        L.rtl_diag_matrix_rate.argtypes = [ci, vp, i64, ci, vp, vp, vp]
        L.rtl_diag_matrix_rate.restype = ci
        L.rtl_diag_fill_rate.argtypes = [vp, sz, i64, ci, vp, vp, vp]
        L.rtl_diag_fill_rate.restype = ci
        L.rtl_sparse_lora_linear_fp8_workspace.argtypes = [i64, i64, i64, i64, ci]
        L.rtl_sparse_lora_linear_fp8_workspace.restype = sz
        L.rtl_sparse_lora_linear_fp8.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i64, i64,
                                                 i64, ci, fl, vp, sz, vp]
        L.rtl_sparse_lora_linear_fp8.restype = ci
        L.rtl_quantize_mxfp4.argtypes = [vp, i64, i64, i64, vp, i64, vp, vp, i64, vp, vp]
        L.rtl_quantize_mxfp4.restype = ci
        L.rtl_dequantize_mxfp4.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp]
        L.rtl_dequantize_mxfp4.restype = ci
        L.rtl_mxfp4_packed_linear_workspace.argtypes = [i64, i64, i64]
        L.rtl_mxfp4_packed_linear_workspace.restype = sz
        L.rtl_mxfp4_packed_linear.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, vp, sz, vp]
        L.rtl_mxfp4_packed_linear.restype = ci
        L.rtl_mxfp4_linear_workspace.argtypes = [i64, i64, i64]
        L.rtl_mxfp4_linear_workspace.restype = sz
        L.rtl_mxfp4_linear.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, vp, sz, vp]
        L.rtl_mxfp4_linear.restype = ci
        L.rtl_grouped_clear.argtypes = [vp, vp] + [i64] * 4 + [vp]
        L.rtl_grouped_clear.restype = ci
        L.rtl_grouped_linear.argtypes = [vp, vp, vp, vp, vp] + [i64] * 8 + [vp]
        L.rtl_grouped_linear.restype = ci
        L.rtl_grouped_linear_dgrad.argtypes = [vp, vp, vp, vp] + [i64] * 8 + [vp]
        L.rtl_grouped_linear_dgrad.restype = ci
        L.rtl_grouped_linear_wgrad_workspace.argtypes = [i64] * 4
        L.rtl_grouped_linear_wgrad_workspace.restype = sz
        L.rtl_grouped_linear_wgrad.argtypes = [vp, vp, vp, vp, vp, ci] + [i64] * 8 + [vp, sz, vp]
        L.rtl_grouped_linear_wgrad.restype = ci
        L.rtl_grouped_mxfp4_linear_workspace.argtypes = [i64] * 4
        L.rtl_grouped_mxfp4_linear_workspace.restype = sz
        L.rtl_grouped_mxfp4_linear.argtypes = [vp] * 6 + [i64] * 8 + [vp, sz, vp]
        L.rtl_grouped_mxfp4_linear.restype = ci
        L.rtl_diag_pack_sweep.argtypes = [vp, i64, i64, i64, ci, fl, vp, sz, vp]
        L.rtl_diag_pack_sweep.restype = ci
        L.rtl_diag_tile_plan.argtypes = [i64, i64, ci, C.POINTER(C.c_int64)]
        L.rtl_diag_tile_plan.restype = ci
        L.rtl_init.argtypes = []
        L.rtl_init.restype = ci
        L.rtl_status_str.argtypes = [ci]
        L.rtl_status_str.restype = C.c_char_p
        L.rtl_version.restype = C.c_char_p
        _lib = L
    return _lib


def status_str(status):
    return lib().rtl_status_str(int(status)).decode()


def version():
    return lib().rtl_version().decode()


def init():
    """rtl_init: one-time set-up of the current device (required only before HIP-graph capture)."""
    _check(lib().rtl_init(), "rtl_init")


# Per-call marshalling is what the smallest linears wait for (a call at [256, 512, 512] keeps the GPU busy for
# 7.5 us): addresses go to ctypes as plain integers (argtypes make them pointers) and the current stream is
# taken as its handle, without a Stream object around it (4 us of a 13 us call).
def _p(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check(status, where):
    if status != 0:
        raise RtlError(status, where)


def _need_cuda(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise ValueError("librtlynx takes device tensors only")


def _ws(nbytes, device):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def sparsify_pack(X, comp=COMP_GROUP, eps=1e-8, out=None):
    """rtl_sparsify_pack: X bf16 [M,K] -> (vals bf16 [M,K/2], meta u8 [M,K/8], scale fp32 or None)."""
    _need_cuda(X)
    assert X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    M, K = X.shape
    dev = X.device
    if out is None:
        vals = torch.empty((M, K // 2), dtype=torch.bfloat16, device=dev)
        meta = torch.empty((M, K // 8), dtype=torch.uint8, device=dev)
    else:
        vals, meta = out
    scale = None
    if comp == COMP_ROW:
        scale = torch.empty((M,), dtype=torch.float32, device=dev)
    elif comp == COMP_TENSOR:
        scale = torch.empty((1,), dtype=torch.float32, device=dev)
    L = lib()
    nws = L.rtl_sparsify_pack_workspace(M, K, comp)
    ws = _ws(nws, dev)
    st = L.rtl_sparsify_pack(_p(X), M, K, X.stride(0), comp, eps, _p(vals), _p(meta), _p(scale),
                             _p(ws), ws.numel(), _stream())
    _check(st, "rtl_sparsify_pack")
    return vals, meta, scale


def packed_linear(vals, meta, W, bias=None, row_scale=None, tensor_scale=None, out=None, ws=None):
    """rtl_packed_linear: Y = decode(vals, meta) W^T (* scales) (+ bias), bf16 [M,N]."""
    _need_cuda(vals, meta, W)
    M, K = vals.shape[0], vals.shape[1] * 2
    N = W.shape[0]
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=W.device) if out is None else out
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_packed_linear_workspace(M, N, K), W.device)
    st = L.rtl_packed_linear(_p(vals), _p(meta), _p(row_scale), _p(tensor_scale), _p(W), _p(bias),
                             _p(Y), M, N, K, W.stride(0), Y.stride(0), _p(ws), ws.numel(), _stream())
    _check(st, "rtl_packed_linear")
    return Y


def sparse_linear_workspace(M, N, K, comp=COMP_GROUP):
    return int(lib().rtl_sparse_linear_workspace(M, N, K, comp))


def sparse_linear(X, W, bias=None, comp=COMP_GROUP, eps=1e-8, out=None, ws=None):
    """rtl_sparse_linear: Y = compensate(sparsify_2:4(X)) W^T (+ bias), bf16 [M,N]."""
    _need_cuda(X, W)
    M, K = X.shape
    N = W.shape[0]
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device) if out is None else out
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_sparse_linear_workspace(M, N, K, comp), X.device)
    st = L.rtl_sparse_linear(_p(X), _p(W), _p(bias), _p(Y), M, N, K, X.stride(0), W.stride(0),
                             Y.stride(0), comp, eps, _p(ws), ws.numel(), _stream())
    _check(st, "rtl_sparse_linear")
    return Y


STATIC_SCRATCH_BYTES = 64 * 1024 * 1024     # RTL_STATIC_SCRATCH_BYTES of the header


def sparse_linear_static(X, W, Y, bias=None, comp=COMP_GROUP, eps=1e-8):
    """rtl_sparse_linear_static: rtl_sparse_linear on the library's fixed scratch; the caller passes
    inputs and the output, nothing is allocated (not by the library, not here)."""
    _need_cuda(X, W, Y)
    M, K = X.shape
    N = W.shape[0]
    st = lib().rtl_sparse_linear_static(_p(X), _p(W), _p(bias), _p(Y), M, N, K, X.stride(0), W.stride(0),
                                        Y.stride(0), comp, eps, _stream())
    _check(st, "rtl_sparse_linear_static")
    return Y


def sparse_lora_linear_workspace(M, N, K, R=64, comp=COMP_GROUP):
    return int(lib().rtl_sparse_lora_linear_workspace(M, N, K, R, comp))


def sparse_lora_linear(X, W, LA, LB, bias=None, comp=COMP_GROUP, eps=1e-8, out=None, ws=None):
    """rtl_sparse_lora_linear: Y = compensate(sparsify_2:4(X)) W^T + X (L_A L_B)^T (+ bias)."""
    _need_cuda(X, W, LA, LB)
    M, K = X.shape
    N, R = LA.shape
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device) if out is None else out
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_sparse_lora_linear_workspace(M, N, K, R, comp), X.device)
    st = L.rtl_sparse_lora_linear(_p(X), _p(W), _p(LA), _p(LB), _p(bias), _p(Y), M, N, K, R,
                                  X.stride(0), W.stride(0), LA.stride(0), LB.stride(0), Y.stride(0),
                                  comp, eps, _p(ws), ws.numel(), _stream())
    _check(st, "rtl_sparse_lora_linear")
    return Y


def dense_linear(X, W, bias=None, out=None, ws=None):
    """rtl_dense_linear: Y = X W^T (+ bias), bf16 [M,N]."""
    _need_cuda(X, W)
    M, K = X.shape
    N = W.shape[0]
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device) if out is None else out
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_dense_linear_workspace(M, N, K), X.device)
    st = L.rtl_dense_linear(_p(X), _p(W), _p(bias), _p(Y), M, N, K, X.stride(0), W.stride(0),
                            Y.stride(0), _p(ws), ws.numel(), _stream())
    _check(st, "rtl_dense_linear")
    return Y


# ---- FP8 (E4M3) composition; codes travel as uint8 tensors ----------------------------------

def quantize_fp8(W, out=None):
    """rtl_quantize_fp8: bf16 [rows, cols] -> E4M3 codes (uint8), direct cast."""
    _need_cuda(W)
    assert W.dtype == torch.bfloat16 and W.dim() == 2 and W.stride(1) == 1
    rows, cols = W.shape
    Wq = torch.empty((rows, cols), dtype=torch.uint8, device=W.device) if out is None else out
    st = lib().rtl_quantize_fp8(_p(W), rows, cols, W.stride(0), _p(Wq), Wq.stride(0), _stream())
    _check(st, "rtl_quantize_fp8")
    return Wq


def sparsify_pack_fp8(X, x_scale, comp=COMP_GROUP, eps=1e-8, out=None):
    """rtl_sparsify_pack_fp8: X bf16 [M,K], x_scale fp32 [1] -> (vals u8 [M,K/2], meta u8 [M,K/8], scale)."""
    _need_cuda(X, x_scale)
    assert X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    assert x_scale.dtype == torch.float32
    M, K = X.shape
    dev = X.device
    if out is None:
        vals = torch.empty((M, K // 2), dtype=torch.uint8, device=dev)
        meta = torch.empty((M, K // 8), dtype=torch.uint8, device=dev)
    else:
        vals, meta = out
    scale = None
    if comp == COMP_ROW:
        scale = torch.empty((M,), dtype=torch.float32, device=dev)
    elif comp == COMP_TENSOR:
        scale = torch.empty((1,), dtype=torch.float32, device=dev)
    L = lib()
    ws = _ws(L.rtl_sparsify_pack_fp8_workspace(M, K, comp), dev)
    st = L.rtl_sparsify_pack_fp8(_p(X), M, K, X.stride(0), comp, eps, _p(x_scale), _p(vals), _p(meta),
                                 _p(scale), _p(ws), ws.numel(), _stream())
    _check(st, "rtl_sparsify_pack_fp8")
    return vals, meta, scale


def sparse_linear_fp8_workspace(M, N, K, comp=COMP_GROUP):
    return int(lib().rtl_sparse_linear_fp8_workspace(M, N, K, comp))


def sparse_linear_fp8(X, Wq, x_scale, bias=None, comp=COMP_GROUP, eps=1e-8, out=None, ws=None):
    """rtl_sparse_linear_fp8: Y = x_scale * (e4m3(S(X) / x_scale) Wq^T) (+ bias), bf16 [M,N]."""
    _need_cuda(X, Wq, x_scale)
    assert Wq.dtype == torch.uint8 and x_scale.dtype == torch.float32
    M, K = X.shape
    N = Wq.shape[0]
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device) if out is None else out
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_sparse_linear_fp8_workspace(M, N, K, comp), X.device)
    st = L.rtl_sparse_linear_fp8(_p(X), _p(Wq), _p(x_scale), _p(bias), _p(Y), M, N, K, X.stride(0),
                                 Wq.stride(0), Y.stride(0), comp, eps, _p(ws), ws.numel(), _stream())
    _check(st, "rtl_sparse_linear_fp8")
    return Y


def sparse_lora_linear_fp8_workspace(M, N, K, R=64, comp=COMP_GROUP):
    return int(lib().rtl_sparse_lora_linear_fp8_workspace(M, N, K, R, comp))


def sparse_lora_linear_fp8(X, Wq, x_scale, LA, LB, bias=None, comp=COMP_GROUP, eps=1e-8, out=None, ws=None):
    """rtl_sparse_lora_linear_fp8: Y = x_scale * (e4m3(S(X) / x_scale) Wq^T) + X (L_A L_B)^T (+ bias), bf16 [M,N]."""
    _need_cuda(X, Wq, x_scale, LA, LB)
    assert Wq.dtype == torch.uint8 and x_scale.dtype == torch.float32
    assert LA.dtype == torch.bfloat16 and LB.dtype == torch.bfloat16
    M, K = X.shape
    N, R = LA.shape
    assert Wq.shape == (N, K) and LB.shape == (R, K)
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=X.device) if out is None else out
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_sparse_lora_linear_fp8_workspace(M, N, K, R, comp), X.device)
    st = L.rtl_sparse_lora_linear_fp8(_p(X), _p(Wq), _p(x_scale), _p(LA), _p(LB), _p(bias), _p(Y), M, N, K, R,
                                      X.stride(0), Wq.stride(0), LA.stride(0), LB.stride(0), Y.stride(0), comp, eps,
                                      _p(ws), ws.numel(), _stream())
    _check(st, "rtl_sparse_lora_linear_fp8")
    return Y


# ---- microscaled 4-bit floating point (MXFP4): uint8 tensors, two codes to a byte -----------------

# These checks run on every call and a small product takes the GPU less time than they do: each property of a tensor is asked for once.

def _here(*ts):
    """Number of the current device, which has to hold all of the tensors: the launch goes to its current stream."""
    dev = torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -1
    for t in ts:
        if t is not None and (t.get_device() != dev or dev < 0):
            raise ValueError("librtlynx takes tensors of the current device (%d) only, not of %s" % (dev, t.device))
    return dev


def _matrix(t, dtype, name):
    """(rows, columns, row stride). torch leaves any stride there for a single row."""
    stride = t.stride()
    if len(stride) != 2 or t.dtype is not dtype:
        raise ValueError("%s: %s matrix expected" % (name, dtype))
    rows, cols = t.shape
    if stride[1] != 1 and cols > 1:
        raise ValueError("%s: contiguous rows expected" % name)
    return rows, cols, stride[0] if rows > 1 else cols


def _stack(t, dtype, name):
    """(matrices, rows, columns, row stride, matrix stride)."""
    stride = t.stride()
    if len(stride) != 3 or t.dtype is not dtype:
        raise ValueError("%s: stack of %s matrices expected" % (name, dtype))
    n, rows, cols = t.shape
    if stride[2] != 1 and cols > 1:
        raise ValueError("%s: contiguous rows expected" % name)
    return n, rows, cols, stride[1] if rows > 1 else cols, stride[0] if n > 1 else 0


def _whole(t, shape, dtype, name):
    """A contiguous tensor of just this shape, or None."""
    if t is not None and (t.shape != shape or t.dtype is not dtype or not t.is_contiguous()):
        raise ValueError("%s: contiguous %s tensor of shape %s expected" % (name, dtype, tuple(shape)))


def _output(out, rows, cols, dtype, like):
    """(out or a new tensor, its row stride)."""
    if out is None:
        return torch.empty(rows, cols, dtype=dtype, device=like.device), cols
    m, n, ld = _matrix(out, dtype, "out")
    if m != rows or n != cols:
        raise ValueError("out: shape (%d, %d) expected" % (rows, cols))
    return out, ld


def _on(dev):
    return torch._C._cuda_getCurrentRawStream(dev)


def mxfp4_scales_shape(rows, cols):
    """Shape of the scale bytes of a [rows, cols] matrix: byte of block b = col // 32 of row r at [b // 8, r, b % 8]."""
    return ((cols + 255) // 256, rows, 8)


def quantize_mxfp4(X, along="cols", out=None):
    """rtl_quantize_mxfp4: bf16 [rows, cols] -> codes and scales, blocks of 32 along its rows ("cols": (Q [rows, cols/2], S)),
    down its columns ("rows": (Qt [cols, R/2], St) of X^T, R = rows rounded up to a multiple of 32) or both in one pass
    ((Q, S, Qt, St)). uint8 tensors; S has mxfp4_scales_shape."""
    if along not in ("cols", "rows", "both"):
        raise ValueError("along: 'cols', 'rows' or 'both'")
    dev = _here(X, *(out or ()))
    rows, cols, ld = _matrix(X, torch.bfloat16, "X")
    u8, pad = torch.uint8, (rows + 31) // 32 * 32
    if out is not None and len(out) != (4 if along == "both" else 2):
        raise ValueError("out: %d tensors expected" % (4 if along == "both" else 2))
    q = s = qt = st = None
    ldq = ldqt = 0
    if along != "rows":
        q, ldq = _output(out and out[0], rows, cols // 2, u8, X)
        shape = mxfp4_scales_shape(rows, cols)
        s = out[1] if out else torch.empty(*shape, dtype=u8, device=X.device)
        _whole(s, shape, u8, "out")
    if along != "cols":
        qt, ldqt = _output(out and out[-2], cols, pad // 2, u8, X)
        shape = mxfp4_scales_shape(cols, pad)
        st = out[-1] if out else torch.empty(*shape, dtype=u8, device=X.device)
        _whole(st, shape, u8, "out")
    _check(lib().rtl_quantize_mxfp4(_p(X), rows, cols, ld, _p(q), ldq, _p(s), _p(qt), ldqt, _p(st), _on(dev)), "rtl_quantize_mxfp4")
    return (q, s, qt, st) if along == "both" else (q, s) if along == "cols" else (qt, st)


def dequantize_mxfp4(Q, S, out=None):
    """rtl_dequantize_mxfp4: codes [rows, cols/2] and scales -> bf16 [rows, cols]."""
    dev = _here(Q, S, out)
    rows, half, ldq = _matrix(Q, torch.uint8, "Q")
    _whole(S, mxfp4_scales_shape(rows, half * 2), torch.uint8, "S")
    X, ld = _output(out, rows, half * 2, torch.bfloat16, Q)
    _check(lib().rtl_dequantize_mxfp4(_p(Q), ldq, _p(S), rows, half * 2, _p(X), ld, _on(dev)), "rtl_dequantize_mxfp4")
    return X


def mxfp4_packed_linear_workspace(M, N, K):
    return int(lib().rtl_mxfp4_packed_linear_workspace(M, N, K))


def mxfp4_packed_linear(Xq, Xs, Wq, Ws, bias=None, out=None, ws=None):
    """rtl_mxfp4_packed_linear: Y = Xq Wq^T (+ bias) on codes and scales of quantize_mxfp4, bf16 [M,N]."""
    dev = _here(Xq, Xs, Wq, Ws, bias, out, ws)
    M, half, ldx = _matrix(Xq, torch.uint8, "Xq")
    N, half_w, ldw = _matrix(Wq, torch.uint8, "Wq")
    K = half * 2
    if half_w != half:
        raise ValueError("Xq and Wq differ in K")
    _whole(Xs, mxfp4_scales_shape(M, K), torch.uint8, "Xs")
    _whole(Ws, mxfp4_scales_shape(N, K), torch.uint8, "Ws")
    _whole(bias, (N,), torch.bfloat16, "bias")
    Y, ldy = _output(out, M, N, torch.bfloat16, Wq)
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_mxfp4_packed_linear_workspace(M, N, K), Wq.device)
    st = L.rtl_mxfp4_packed_linear(_p(Xq), _p(Xs), _p(Wq), _p(Ws), _p(bias), _p(Y), M, N, K, ldx, ldw, ldy, _p(ws), _bytes(ws), _on(dev))
    _check(st, "rtl_mxfp4_packed_linear")
    return Y


def _bytes(ws):
    return ws.numel() * ws.element_size() if ws.is_contiguous() else 0


def mxfp4_linear_workspace(M, N, K):
    return int(lib().rtl_mxfp4_linear_workspace(M, N, K))


def mxfp4_linear(X, Wq, Ws, bias=None, out=None, ws=None):
    """rtl_mxfp4_linear: Y = mxfp4(X) Wq^T (+ bias), X bf16 [M,K] quantised in the call, bf16 [M,N]."""
    dev = _here(X, Wq, Ws, bias, out, ws)
    M, K, ldx = _matrix(X, torch.bfloat16, "X")
    N, half, ldw = _matrix(Wq, torch.uint8, "Wq")
    if half * 2 != K:
        raise ValueError("X and Wq differ in K")
    _whole(Ws, mxfp4_scales_shape(N, K), torch.uint8, "Ws")
    _whole(bias, (N,), torch.bfloat16, "bias")
    Y, ldy = _output(out, M, N, torch.bfloat16, X)
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_mxfp4_linear_workspace(M, N, K), X.device)
    st = L.rtl_mxfp4_linear(_p(X), _p(Wq), _p(Ws), _p(bias), _p(Y), M, N, K, ldx, ldw, ldy, _p(ws), _bytes(ws), _on(dev))
    _check(st, "rtl_mxfp4_linear")
    return Y


# ---- linears grouped by expert: rows offsets[e] .. offsets[e + 1] of the activation belong to weight e ------------
# `out` of the row-wise results: rows of no expert keep what it held; without `out` they are zeros.

def _rows_output(out, rows, cols, like, offsets, E, dev):
    """(out, or a new tensor with zeros in the rows of no expert, its row stride)."""
    Y, ld = _output(out, rows, cols, torch.bfloat16, like)
    if out is None:
        _check(lib().rtl_grouped_clear(_p(offsets), _p(Y), rows, E, cols, ld, _on(dev)), "rtl_grouped_clear")
    return Y, ld


def grouped_clear(offsets, out):
    """rtl_grouped_clear: zeros into the rows of `out` (bf16 [T,N]) that belong to no expert."""
    dev = _here(offsets, out)
    T, N, ld = _matrix(out, torch.bfloat16, "out")
    E = offsets.numel() - 1
    if E < 0:
        raise ValueError("offsets: at least one number expected")
    _whole(offsets, (E + 1,), torch.int32, "offsets")
    _check(lib().rtl_grouped_clear(_p(offsets), _p(out), T, E, N, ld, _on(dev)), "rtl_grouped_clear")
    return out


def grouped_linear(X, offsets, W, bias=None, out=None):
    """rtl_grouped_linear: Y[rows of e] = X[rows of e] W[e]^T (+ bias[e]); X bf16 [T,K], offsets int32 [E+1] on the device,
    W bf16 [E,N,K], bias [E,N]; bf16 [T,N]."""
    dev = _here(X, offsets, W, bias, out)
    T, K, ldx = _matrix(X, torch.bfloat16, "X")
    E, N, K_w, ldw, stride = _stack(W, torch.bfloat16, "W")
    if K_w != K:
        raise ValueError("X and W differ in K")
    _whole(offsets, (E + 1,), torch.int32, "offsets")
    _whole(bias, (E, N), torch.bfloat16, "bias")
    Y, ldy = _rows_output(out, T, N, X, offsets, E, dev)
    st = lib().rtl_grouped_linear(_p(X), _p(offsets), _p(W), _p(bias), _p(Y), T, E, N, K, ldx, ldw, stride, ldy, _on(dev))
    _check(st, "rtl_grouped_linear")
    return Y


def grouped_linear_dgrad(dY, offsets, W, out=None):
    """rtl_grouped_linear_dgrad: dX[rows of e] = dY[rows of e] W[e]; bf16 [T,K]."""
    dev = _here(dY, offsets, W, out)
    T, N, lddy = _matrix(dY, torch.bfloat16, "dY")
    E, N_w, K, ldw, stride = _stack(W, torch.bfloat16, "W")
    if N_w != N:
        raise ValueError("dY and W differ in N")
    _whole(offsets, (E + 1,), torch.int32, "offsets")
    dX, ldx = _rows_output(out, T, K, dY, offsets, E, dev)
    st = lib().rtl_grouped_linear_dgrad(_p(dY), _p(offsets), _p(W), _p(dX), T, E, N, K, lddy, ldw, stride, ldx, _on(dev))
    _check(st, "rtl_grouped_linear_dgrad")
    return dX


def grouped_linear_wgrad_workspace(T, E, N, K):
    return int(lib().rtl_grouped_linear_wgrad_workspace(T, E, N, K))


def grouped_linear_wgrad(dY, X, offsets, with_bias=False, dtype=torch.bfloat16, out=None, ws=None):
    """rtl_grouped_linear_wgrad: (dW [E,N,K], db [E,N] or None), dW[e] = dY[rows of e]^T X[rows of e], db[e] the sum of the rows of
    dY, in bf16 or float32. `out`: the two tensors (the second None without a bias); they then settle with_bias and dtype."""
    dW, db = out if out is not None else (None, None)
    dev = _here(dY, X, offsets, dW, db, ws)
    T, N, lddy = _matrix(dY, torch.bfloat16, "dY")
    T_x, K, ldx = _matrix(X, torch.bfloat16, "X")
    if T_x != T:
        raise ValueError("dY and X differ in rows")
    E = offsets.numel() - 1
    if E < 0:
        raise ValueError("offsets: at least one number expected")
    _whole(offsets, (E + 1,), torch.int32, "offsets")
    if out is None:
        dW = torch.empty((E, N, K), dtype=dtype, device=dY.device)
        db = torch.empty((E, N), dtype=dtype, device=dY.device) if with_bias else None
    dtype = dW.dtype
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise ValueError("gradients in bf16 or float32")
    e, n, k, lddw, stride = _stack(dW, dtype, "dW")
    if e != E or n != N or k != K:
        raise ValueError("dW: shape (%d, %d, %d) expected" % (E, N, K))
    _whole(db, (E, N), dtype, "db")
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_grouped_linear_wgrad_workspace(T, E, N, K), dY.device)
    st = L.rtl_grouped_linear_wgrad(_p(dY), _p(X), _p(offsets), _p(dW), _p(db), 1 if dtype is torch.float32 else 0, T, E, N, K,
                                    lddy, ldx, lddw, stride, _p(ws), _bytes(ws), _on(dev))
    _check(st, "rtl_grouped_linear_wgrad")
    return dW, db


def grouped_mxfp4_linear_workspace(T, E, N, K):
    return int(lib().rtl_grouped_mxfp4_linear_workspace(T, E, N, K))


def grouped_mxfp4_linear(X, offsets, Wq, Ws, bias=None, out=None, ws=None):
    """rtl_grouped_mxfp4_linear: grouped_linear with X quantised in the call and 4-bit weights: Wq uint8 [E,N,K/2], Ws the scales of
    the [E*N, K] matrix of all rows (what quantize_mxfp4(W.view(E * N, K)) returns); bf16 [T,N]."""
    dev = _here(X, offsets, Wq, Ws, bias, out, ws)
    T, K, ldx = _matrix(X, torch.bfloat16, "X")
    E, N, half, ldw, stride = _stack(Wq, torch.uint8, "Wq")
    if half * 2 != K:
        raise ValueError("X and Wq differ in K")
    _whole(offsets, (E + 1,), torch.int32, "offsets")
    _whole(Ws, mxfp4_scales_shape(E * N, K), torch.uint8, "Ws")
    _whole(bias, (E, N), torch.bfloat16, "bias")
    Y, ldy = _rows_output(out, T, N, X, offsets, E, dev)
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_grouped_mxfp4_linear_workspace(T, E, N, K), X.device)
    st = L.rtl_grouped_mxfp4_linear(_p(X), _p(offsets), _p(Wq), _p(Ws), _p(bias), _p(Y), T, E, N, K, ldx, ldw, stride, ldy, _p(ws), _bytes(ws), _on(dev))
    _check(st, "rtl_grouped_mxfp4_linear")
    return Y


# ---- diagnostics ------------------------------------------------------------------------------

def diag_matrix_rate(kind, operands, iters, blocks=1024):
    """rtl_diag_matrix_rate: enqueue the issue-rate probe; returns (clocks uint64[2] as an int64 tensor,
    executed flops of the launch). Timing is the caller's (events around the call)."""
    _need_cuda(operands)
    assert operands.numel() * operands.element_size() >= 3072
    clocks = torch.zeros(2, dtype=torch.int64, device=operands.device)
    sink = torch.zeros(1, dtype=torch.float32, device=operands.device)
    st = lib().rtl_diag_matrix_rate(int(kind), _p(operands), int(iters), int(blocks), _p(clocks), _p(sink), _stream())
    _check(st, "rtl_diag_matrix_rate")
    return clocks, float(blocks) * 4 * 4 * iters * 2 * 32 * 32 * 16


def diag_pack_sweep(X, comp=COMP_GROUP, eps=1e-8, ws=None):
    """rtl_diag_pack_sweep: the sparsification sweep as rtl_sparse_linear launches it, alone (for timing);
    the compressed operand lands in the head of `ws` (an rtl_sparse_linear workspace)."""
    _need_cuda(X)
    assert X.dtype == torch.bfloat16 and X.dim() == 2 and X.stride(1) == 1
    M, K = X.shape
    L = lib()
    if ws is None:
        ws = _ws(L.rtl_sparse_linear_workspace(M, 1, K, comp), X.device)
    _check(L.rtl_diag_pack_sweep(_p(X), M, K, X.stride(0), comp, eps, _p(ws), ws.numel(), _stream()),
           "rtl_diag_pack_sweep")
    return ws


def diag_tile_plan(M, N, dense=False):
    """rtl_diag_tile_plan: dict(body_width, body_rows, body_tiles, tail_tiles) for an [M, N] output."""
    out = (C.c_int64 * 4)()
    _check(lib().rtl_diag_tile_plan(int(M), int(N), int(bool(dense)), out), "rtl_diag_tile_plan")
    return dict(body_width=int(out[0]), body_rows=int(out[1]), body_tiles=int(out[2]), tail_tiles=int(out[3]))


def diag_fill_rate(region, iters, blocks=256):
    """rtl_diag_fill_rate: enqueue the L2 -> LDS streaming probe on `region` (a uint8 device tensor);
    returns (clocks int64[2] tensor, bytes moved by the launch)."""
    _need_cuda(region)
    nbytes = region.numel() * region.element_size()
    clocks = torch.zeros(2, dtype=torch.int64, device=region.device)
    sink = torch.zeros(1, dtype=torch.float32, device=region.device)
    st = lib().rtl_diag_fill_rate(_p(region), nbytes, int(iters), int(blocks), _p(clocks), _p(sink), _stream())
    _check(st, "rtl_diag_fill_rate")
    return clocks, float(blocks) * 8 * iters * 8192
