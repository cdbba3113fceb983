"""Python binding of ``libxtc.so``, the MI355X (gfx950) tiled dense contraction.

Argument marshalling only: every step of the computation runs in the HIP
kernels of ``libxtc.so``.  The functions ``xtc_matmul``, ``xtc_conv2d_nchw``,
``xtc_matmul_relu``, ``xtc_conv2d_nchw_relu``, ``xtc_default_schedule``, ``xtc_sched_check``, ``xtc_sched_list``,
``xtc_status_str`` mirror the C ABI of ``include/xtc.h`` one to one (pointers
are Python ints holding device addresses; the stream is a ``hipStream_t`` as
an int, 0 for the null stream).  ``matmul`` and ``conv2d_nchw`` are
conveniences over torch device tensors (torch provides memory and the
current stream, nothing else); the plain calls among theirs go through
``_binding.so`` (csrc/torch_binding.cpp), which saves the interpreter's share
of a call.  ``rmsnorm``, ``rmsnorm_backward``, ``quantize_fp8``, ``matmul_fp8``,
``matmul_grouped``, ``matmul_grouped_wgrad``, ``matmul_grouped_fp8``, ``layernorm``,
``linear``, ``route_experts``, ``combine_experts``, their ``_backward`` forms,
``linear_wgrad`` and ``activation_backward`` likewise
stand for the entry points of those names.  None of them records an autograd
graph: a result does not require a gradient whatever its operands do, and the
gradients are calls of their own.

If the library has not been built, importing this package raises
``ImportError``: there is no fallback implementation.  Without the native
binding (not built, or for another torch) it warns, and the conveniences check
their arguments and call the same library from Python.
"""
from __future__ import annotations

import ctypes
import os
from collections import namedtuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libxtc.so")

XTC_F32 = 0
XTC_BF16 = 1
XTC_FP8 = 2
XTC_NO_ACTIVATION = 0
XTC_RELU = 1
XTC_GELU = 2
XTC_GELU_TANH = 3
XTC_SILU = 4
XTC_OP_MATMUL = 0
XTC_OP_CONV2D = 1

XTC_OK = 0
XTC_ERR_NULL_POINTER = 1
XTC_ERR_BAD_SHAPE = 2
XTC_ERR_BAD_LEADING_DIM = 3
XTC_ERR_BAD_DTYPE = 4
XTC_ERR_BAD_SCHEDULE = 5
XTC_ERR_UNSUPPORTED_SCHEDULE = 6
XTC_ERR_TOO_LARGE = 7
XTC_ERR_HIP = 8
XTC_ERR_MISALIGNED = 9


class Sched(ctypes.Structure):
    """``xtc_sched``: see include/xtc.h for the meaning of each field."""
    _fields_ = [(n, ctypes.c_int32) for n in (
        "size", "block_m", "block_n", "block_k", "wave_m", "wave_n",
        "mfma_m", "mfma_n", "mfma_k", "lds_stages", "lds_pad", "unroll_k",
        "raster", "xcd_remap", "k_order", "k_split")]

    def __init__(self, **kw):
        super().__init__()
        self.size = ctypes.sizeof(Sched)
        self.k_split = 1
        for k, v in kw.items():
            setattr(self, k, v)

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_ if n != "size"}

    def __repr__(self):
        d = self.as_dict()
        return ("Sched(block=%dx%dx%d wave=%dx%d mfma=%dx%dx%d stages=%d pad=%d unroll=%d "
                "raster=%d xcd=%d k_order=%d k_split=%d)" % (
                    d["block_m"], d["block_n"], d["block_k"], d["wave_m"], d["wave_n"],
                    d["mfma_m"], d["mfma_n"], d["mfma_k"], d["lds_stages"], d["lds_pad"],
                    d["unroll_k"], d["raster"], d["xcd_remap"], d["k_order"], d["k_split"]))


class XtcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = "%s: %s (status %d)" % (where, xtc_status_str(status), status)
        if status == XTC_ERR_HIP:
            msg += ", hipError %d" % _lib.xtc_last_hip_error()
        super().__init__(msg)


def _load():
    # torch ships its own HIP runtime (same soname as ROCm's).  Loading torch
    # first makes libxtc.so bind to that one runtime; loaded the other way
    # round, the process would map two runtimes, and torch's device memory
    # and streams would be invalid handles for the library's launches.
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libxtc.so is not built (expected at %s); run `python paper_2512_16512_amd/build.py`"
            % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    i64, vp, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int32
    sp = ctypes.POINTER(Sched)
    lib.xtc_matmul.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, i32, sp, vp]
    lib.xtc_matmul.restype = i32
    lib.xtc_conv2d_nchw.argtypes = [i64] * 11 + [vp, vp, vp, i32, sp, vp]
    lib.xtc_conv2d_nchw.restype = i32
    lib.xtc_matmul_relu.argtypes = lib.xtc_matmul.argtypes
    lib.xtc_matmul_relu.restype = i32
    lib.xtc_conv2d_nchw_relu.argtypes = lib.xtc_conv2d_nchw.argtypes
    lib.xtc_conv2d_nchw_relu.restype = i32
    f32 = ctypes.c_float
    lib.xtc_rmsnorm.argtypes = [i64, i64, vp, i64, vp, i64, vp, f32, vp, i64, vp, i64, vp, i64, vp, i32, i32, i32, vp]
    lib.xtc_rmsnorm.restype = i32
    lib.xtc_rmsnorm_backward.argtypes = [i64, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, vp, i64, i32, i32, vp]
    lib.xtc_rmsnorm_backward.restype = i32
    lib.xtc_rmsnorm_backward_workspace.argtypes = [i64, i64]
    lib.xtc_rmsnorm_backward_workspace.restype = i64
    lib.xtc_layernorm.argtypes = [i64, i64, vp, i64, vp, i64, vp, vp, f32, vp, i64, vp, i64, vp, i64, vp, vp, i32, i32,
                                  i32, vp]
    lib.xtc_layernorm.restype = i32
    lib.xtc_layernorm_backward.argtypes = [i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, i64, i32,
                                           i32, vp]
    lib.xtc_layernorm_backward.restype = i32
    lib.xtc_layernorm_backward_workspace.argtypes = [i64, i64]
    lib.xtc_layernorm_backward_workspace.restype = i64
    lib.xtc_quantize_fp8.argtypes = [i64, i64, vp, i64, i64, vp, i64, vp, i64, i32, vp]
    lib.xtc_quantize_fp8.restype = i32
    lib.xtc_matmul_fp8.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, i32, i32, vp]
    lib.xtc_matmul_fp8.restype = i32
    lib.xtc_linear.argtypes = [i64] * 3 + [vp, i64, vp, i64, i32, vp, i32, vp, i64, i32, i32, vp, i64, vp, i64, vp, i64,
                                           i32, i32, vp]
    lib.xtc_linear.restype = i32
    lib.xtc_linear_workspace.argtypes = [i64] * 3 + [vp, i64, vp, i64, i32]
    lib.xtc_linear_workspace.restype = i64
    lib.xtc_linear_wgrad.argtypes = [i64] * 3 + [vp, i64, vp, i64, vp, i64, vp, i64, i32, i32, vp]
    lib.xtc_linear_wgrad.restype = i32
    lib.xtc_linear_wgrad_workspace.argtypes = [i64] * 3 + [vp, i64, vp, i64]
    lib.xtc_linear_wgrad_workspace.restype = i64
    lib.xtc_activation_backward.argtypes = [i64] * 2 + [vp, i64, i32, vp, i64, i32, i32, vp, i64, vp, vp, i64, vp]
    lib.xtc_activation_backward.restype = i32
    lib.xtc_activation_backward_workspace.argtypes = [i64] * 2
    lib.xtc_activation_backward_workspace.restype = i64
    lib.xtc_route_experts.argtypes = [i64] * 3 + [vp, i64] + [vp] * 9 + [i64, i32, vp]
    lib.xtc_route_experts.restype = i32
    lib.xtc_route_experts_workspace.argtypes = [i64] * 2
    lib.xtc_route_experts_workspace.restype = i64
    lib.xtc_route_experts_backward.argtypes = [i64] * 3 + [vp, vp, i64, vp, vp, vp, f32, vp, i64, i32, i32, vp]
    lib.xtc_route_experts_backward.restype = i32
    lib.xtc_combine_experts.argtypes = [i64] * 4 + [vp, i64, vp, vp, vp, i64, i32, vp, i64, i32, i32, vp]
    lib.xtc_combine_experts.restype = i32
    lib.xtc_combine_experts_backward.argtypes = [i64] * 3 + [vp, i64, i32, vp, i64, vp, vp, vp, vp, i64, vp, i32, vp]
    lib.xtc_combine_experts_backward.restype = i32
    lib.xtc_matmul_grouped.argtypes = [i64] * 4 + [vp, i64, vp, i64, i64, i32, vp, vp, i64, i32, i32, i32, vp]
    lib.xtc_matmul_grouped.restype = i32
    lib.xtc_matmul_grouped_wgrad.argtypes = [i64] * 4 + [vp, i64, vp, i64, vp, vp, i64, i64, i32, i32, vp]
    lib.xtc_matmul_grouped_wgrad.restype = i32
    lib.xtc_matmul_grouped_fp8.argtypes = [i64] * 4 + [vp, i64, vp, i64, vp, i64, i64, vp, i64, i64, vp, vp, i64,
                                                       i32, i32, vp]
    lib.xtc_matmul_grouped_fp8.restype = i32
    lib.xtc_default_schedule.argtypes = [i32, i32, i64, i64, i64, sp]
    lib.xtc_default_schedule.restype = i32
    lib.xtc_sched_check.argtypes = [i32, i32, sp]
    lib.xtc_sched_check.restype = i32
    lib.xtc_sched_occupancy.argtypes = [i32, i32, i64, sp, ctypes.POINTER(i32)]
    lib.xtc_sched_occupancy.restype = i32
    lib.xtc_sched_list.argtypes = [i32, i32, sp, i32]
    lib.xtc_sched_list.restype = i32
    lib.xtc_status_str.argtypes = [i32]
    lib.xtc_status_str.restype = ctypes.c_char_p
    lib.xtc_last_hip_error.argtypes = []
    lib.xtc_last_hip_error.restype = i32
    lib.xtc_conv_max_k.argtypes = []
    lib.xtc_conv_max_k.restype = i64
    lib.xtc_version.argtypes = []
    lib.xtc_version.restype = i32
    return lib


_lib = _load()


def _load_binding():
    # needs torch; without it the conveniences below cannot be called either
    try:
        import torch  # noqa: F401
    except ImportError:
        return None
    try:
        from . import _binding
    except ImportError as e:
        import warnings
        warnings.warn("the native binding does not load (%s): matmul() and conv2d_nchw() take 6 us longer "
                      "per call; run `python paper_2512_16512_amd/build.py`" % e, RuntimeWarning, stacklevel=3)
        return None
    return _binding


_fast = _load_binding()

# Every symbol include/xtc.h declares.
EXPORTS = ("xtc_matmul", "xtc_conv2d_nchw", "xtc_matmul_relu", "xtc_conv2d_nchw_relu",
           "xtc_rmsnorm", "xtc_rmsnorm_backward", "xtc_rmsnorm_backward_workspace", "xtc_layernorm",
           "xtc_layernorm_backward", "xtc_layernorm_backward_workspace", "xtc_quantize_fp8",
           "xtc_matmul_fp8", "xtc_linear", "xtc_linear_workspace", "xtc_linear_wgrad", "xtc_linear_wgrad_workspace",
           "xtc_activation_backward", "xtc_activation_backward_workspace", "xtc_matmul_grouped", "xtc_matmul_grouped_wgrad", "xtc_matmul_grouped_fp8",
           "xtc_route_experts", "xtc_route_experts_workspace", "xtc_route_experts_backward", "xtc_combine_experts",
           "xtc_combine_experts_backward", "xtc_default_schedule", "xtc_sched_occupancy", "xtc_sched_check",
           "xtc_sched_list", "xtc_status_str", "xtc_last_hip_error", "xtc_conv_max_k",
           "xtc_version")


def _sp(sched):
    return ctypes.byref(sched) if sched is not None else None


# ------------------------------------------------------------- raw C ABI


def xtc_matmul(M, N, K, A, lda, B, ldb, C, ldc, dtype, sched=None, stream=0) -> int:
    return _lib.xtc_matmul(M, N, K, A, lda, B, ldb, C, ldc, dtype, _sp(sched), stream)


def xtc_conv2d_nchw(N, C, H, W, OC, R, S, stride_h, stride_w, pad_h, pad_w, X, Wt, Y, dtype,
                    sched=None, stream=0) -> int:
    return _lib.xtc_conv2d_nchw(N, C, H, W, OC, R, S, stride_h, stride_w, pad_h, pad_w, X, Wt, Y,
                                dtype, _sp(sched), stream)


def xtc_matmul_relu(M, N, K, A, lda, B, ldb, C, ldc, dtype, sched=None, stream=0) -> int:
    return _lib.xtc_matmul_relu(M, N, K, A, lda, B, ldb, C, ldc, dtype, _sp(sched), stream)


def xtc_conv2d_nchw_relu(N, C, H, W, OC, R, S, stride_h, stride_w, pad_h, pad_w, X, Wt, Y, dtype,
                         sched=None, stream=0) -> int:
    return _lib.xtc_conv2d_nchw_relu(N, C, H, W, OC, R, S, stride_h, stride_w, pad_h, pad_w, X,
                                     Wt, Y, dtype, _sp(sched), stream)


def xtc_rmsnorm(T, D, X, ldx, R, ldr, W, eps, Y, ldy, S, lds, H, ldh, rstd, dtype, w_dtype, out_dtype, stream=0) -> int:
    return _lib.xtc_rmsnorm(T, D, X, ldx, R, ldr, W, eps, Y, ldy, S, lds, H, ldh, rstd, dtype, w_dtype, out_dtype,
                            stream)


def xtc_rmsnorm_backward(T, D, DY, lddy, X, ldx, W, rstd, DR, lddr, DX, lddx, DW, workspace, workspace_bytes, dtype,
                         w_dtype, stream=0) -> int:
    return _lib.xtc_rmsnorm_backward(T, D, DY, lddy, X, ldx, W, rstd, DR, lddr, DX, lddx, DW, workspace,
                                     workspace_bytes, dtype, w_dtype, stream)


def xtc_rmsnorm_backward_workspace(T, D) -> int:
    return _lib.xtc_rmsnorm_backward_workspace(T, D)


def xtc_layernorm(T, D, X, ldx, R, ldr, W, B, eps, Y, ldy, S, lds, H, ldh, mean, rstd, dtype, w_dtype, out_dtype,
                  stream=0) -> int:
    return _lib.xtc_layernorm(T, D, X, ldx, R, ldr, W, B, eps, Y, ldy, S, lds, H, ldh, mean, rstd, dtype, w_dtype,
                              out_dtype, stream)


def xtc_layernorm_backward(T, D, DY, lddy, X, ldx, W, mean, rstd, DR, lddr, DX, lddx, DW, DB, workspace,
                           workspace_bytes, dtype, w_dtype, stream=0) -> int:
    return _lib.xtc_layernorm_backward(T, D, DY, lddy, X, ldx, W, mean, rstd, DR, lddr, DX, lddx, DW, DB, workspace,
                                       workspace_bytes, dtype, w_dtype, stream)


def xtc_layernorm_backward_workspace(T, D) -> int:
    return _lib.xtc_layernorm_backward_workspace(T, D)


def xtc_quantize_fp8(M, K, X, ldx, block_rows, Q, ldq, S, lds, dtype, stream=0) -> int:
    return _lib.xtc_quantize_fp8(M, K, X, ldx, block_rows, Q, ldq, S, lds, dtype, stream)


def xtc_matmul_fp8(M, N, K, A, lda, SA, ldsa, B, ldb, SB, ldsb, C, ldc, out_dtype, relu=0, stream=0) -> int:
    return _lib.xtc_matmul_fp8(M, N, K, A, lda, SA, ldsa, B, ldb, SB, ldsb, C, ldc, out_dtype, relu, stream)


def xtc_linear(T, N, K, A, lda, B, ldb, transpose_b, bias, bias_dtype, R, ldr, r_dtype, activation, C, ldc, Z, ldz,
               workspace, workspace_bytes, dtype, out_dtype, stream=0) -> int:
    return _lib.xtc_linear(T, N, K, A, lda, B, ldb, transpose_b, bias, bias_dtype, R, ldr, r_dtype, activation, C, ldc,
                           Z, ldz, workspace, workspace_bytes, dtype, out_dtype, stream)


def xtc_linear_workspace(T, N, K, A, lda, B, ldb, transpose_b) -> int:
    return _lib.xtc_linear_workspace(T, N, K, A, lda, B, ldb, transpose_b)


def xtc_linear_wgrad(T, N, K, A, lda, DY, lddy, DB, lddb, workspace, workspace_bytes, dtype, out_dtype, stream=0) -> int:
    return _lib.xtc_linear_wgrad(T, N, K, A, lda, DY, lddy, DB, lddb, workspace, workspace_bytes, dtype, out_dtype,
                                 stream)


def xtc_linear_wgrad_workspace(T, N, K, A, lda, DY, lddy) -> int:
    return _lib.xtc_linear_wgrad_workspace(T, N, K, A, lda, DY, lddy)


def xtc_activation_backward(T, N, DY, lddy, dy_dtype, Z, ldz, z_dtype, activation, DZ, lddz, DB, workspace,
                            workspace_bytes, stream=0) -> int:
    return _lib.xtc_activation_backward(T, N, DY, lddy, dy_dtype, Z, ldz, z_dtype, activation, DZ, lddz, DB, workspace,
                                        workspace_bytes, stream)


def xtc_activation_backward_workspace(T, N) -> int:
    return _lib.xtc_activation_backward_workspace(T, N)


def xtc_matmul_grouped(G, T, N, K, A, lda, B, ldb, stride_b, transpose_b, ends, C, ldc, dtype, out_dtype, relu=0,
                       stream=0) -> int:
    return _lib.xtc_matmul_grouped(G, T, N, K, A, lda, B, ldb, stride_b, transpose_b, ends, C, ldc, dtype, out_dtype,
                                   relu, stream)


def xtc_matmul_grouped_wgrad(G, T, N, K, A, lda, DY, lddy, ends, DB, lddb, stride_db, dtype, out_dtype,
                             stream=0) -> int:
    return _lib.xtc_matmul_grouped_wgrad(G, T, N, K, A, lda, DY, lddy, ends, DB, lddb, stride_db, dtype, out_dtype,
                                         stream)


def xtc_matmul_grouped_fp8(G, T, N, K, A, lda, SA, ldsa, B, ldb, stride_b, SB, ldsb, stride_sb, ends, C, ldc,
                           out_dtype, relu=0, stream=0) -> int:
    return _lib.xtc_matmul_grouped_fp8(G, T, N, K, A, lda, SA, ldsa, B, ldb, stride_b, SB, ldsb, stride_sb, ends, C,
                                       ldc, out_dtype, relu, stream)


def xtc_route_experts(T, E, top, scores, lds, mask, expert, p, row, token, counts, ends, loss, workspace,
                      workspace_bytes, dtype, stream=0) -> int:
    return _lib.xtc_route_experts(T, E, top, scores, lds, mask, expert, p, row, token, counts, ends, loss, workspace,
                                  workspace_bytes, dtype, stream)


def xtc_route_experts_workspace(T, E) -> int:
    return _lib.xtc_route_experts_workspace(T, E)


def xtc_route_experts_backward(T, E, top, DP, scores, lds, expert, p, counts, dloss, DS, ldds, dtype, out_dtype,
                               stream=0) -> int:
    return _lib.xtc_route_experts_backward(T, E, top, DP, scores, lds, expert, p, counts, dloss, DS, ldds, dtype,
                                           out_dtype, stream)


def xtc_combine_experts(T, top, D, R, rows, ldrows, row, p, RES, ldr, r_dtype, C, ldc, dtype, out_dtype,
                        stream=0) -> int:
    return _lib.xtc_combine_experts(T, top, D, R, rows, ldrows, row, p, RES, ldr, r_dtype, C, ldc, dtype, out_dtype,
                                    stream)


def xtc_combine_experts_backward(T, top, D, DOUT, lddo, dout_dtype, rows, ldrows, row, token, p, DROWS, lddr, DP, dtype,
                                 stream=0) -> int:
    return _lib.xtc_combine_experts_backward(T, top, D, DOUT, lddo, dout_dtype, rows, ldrows, row, token, p, DROWS,
                                             lddr, DP, dtype, stream)


def xtc_default_schedule(op, dtype, M, N, K) -> Sched:
    s = Sched()
    st = _lib.xtc_default_schedule(op, dtype, M, N, K, ctypes.byref(s))
    if st != XTC_OK:
        raise XtcError(st, "xtc_default_schedule")
    return s


def xtc_sched_check(op, dtype, sched) -> int:
    return _lib.xtc_sched_check(op, dtype, _sp(sched))


def xtc_sched_occupancy(op, dtype, K, sched) -> int:
    """Workgroups of the instance ``sched`` names that one CU holds at once."""
    n = ctypes.c_int32(0)
    st = _lib.xtc_sched_occupancy(op, dtype, K, _sp(sched), ctypes.byref(n))
    if st != XTC_OK:
        raise XtcError(st, "xtc_sched_occupancy")
    return n.value


def xtc_sched_list(op, dtype):
    n = _lib.xtc_sched_list(op, dtype, None, 0)
    if n < 0:
        return []
    arr = (Sched * n)()
    _lib.xtc_sched_list(op, dtype, arr, n)
    return list(arr)


def xtc_status_str(status) -> str:
    return _lib.xtc_status_str(status).decode()


def xtc_last_hip_error() -> int:
    return _lib.xtc_last_hip_error()


def xtc_conv_max_k() -> int:
    return _lib.xtc_conv_max_k()


def xtc_version() -> int:
    return _lib.xtc_version()


# ------------------------------------------------------- torch conveniences


def _stream(torch, device):
    return torch.cuda.current_stream(device).cuda_stream


def _dtype_code(torch, t):
    if t.dtype == torch.float32:
        return XTC_F32
    if t.dtype == torch.bfloat16:
        return XTC_BF16
    raise TypeError("unsupported dtype %s (float32 or bfloat16)" % t.dtype)


def _check_rowmajor(t, name):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError("%s must be a 2-D row-major tensor (unit column stride)" % name)


def matmul(a, b, out=None, sched=None, relu=False):
    """``out = a @ b`` on the GPU (``relu(a @ b)`` fused when ``relu``).
    ``a`` [M,K] and ``b`` [K,N] are both float32 or both bfloat16 CUDA tensors
    with unit column stride; ``out`` is float32 [M,N] (allocated when None).
    Enqueued on torch's current stream."""
    if sched is None and _fast is not None:
        c = _fast.matmul(a, b, out, relu)
        if c is not None:
            return c
    import torch
    _check_rowmajor(a, "a")
    _check_rowmajor(b, "b")
    if a.dtype != b.dtype:
        raise TypeError("a and b must have the same dtype")
    if not (a.is_cuda and b.is_cuda):
        raise ValueError("a and b must be CUDA (HIP) tensors")
    M, K = a.shape
    K2, N = b.shape
    if K2 != K:
        raise ValueError("inner dimensions differ: %d vs %d" % (K, K2))
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=a.device)
    _check_rowmajor(out, "out")
    if out.dtype != torch.float32 or tuple(out.shape) != (M, N):
        raise ValueError("out must be float32 [M, N]")
    lda = a.stride(0) if M > 1 else max(K, 1)
    ldb = b.stride(0) if K > 1 else max(N, 1)
    ldc = out.stride(0) if M > 1 else max(N, 1)
    fn = xtc_matmul_relu if relu else xtc_matmul
    st = fn(M, N, K, a.data_ptr(), lda, b.data_ptr(), ldb, out.data_ptr(), ldc,
            _dtype_code(torch, a), sched, _stream(torch, a.device))
    if st != XTC_OK:
        raise XtcError(st, fn.__name__)
    return out


def conv2d_nchw(x, w, stride=1, pad=0, out=None, sched=None, relu=False):
    """Zero-padded cross-correlation of NCHW ``x`` with OIHW ``w`` (both
    float32 or both bfloat16, contiguous CUDA tensors) into a float32 NCHW
    ``out`` (relu fused into the epilogue when ``relu``)."""
    if sched is None and _fast is not None:
        y = _fast.conv2d_nchw(x, w, stride, pad, out, relu)
        if y is not None:
            return y
    import torch
    if x.dim() != 4 or w.dim() != 4 or not x.is_contiguous() or not w.is_contiguous():
        raise ValueError("x and w must be contiguous 4-D tensors")
    if x.dtype != w.dtype:
        raise TypeError("x and w must have the same dtype")
    N, C, H, W = x.shape
    OC, C2, R, S = w.shape
    if C2 != C:
        raise ValueError("channel counts differ")
    sh, sw = (stride, stride) if isinstance(stride, int) else stride
    ph, pw = (pad, pad) if isinstance(pad, int) else pad
    OH = (H + 2 * ph - R) // sh + 1
    OW = (W + 2 * pw - S) // sw + 1
    if out is None:
        out = torch.empty((N, OC, max(OH, 0), max(OW, 0)), dtype=torch.float32, device=x.device)
    if not out.is_contiguous() or tuple(out.shape) != (N, OC, OH, OW):
        raise ValueError("out must be a contiguous [N, OC, OH, OW] tensor")
    fn = xtc_conv2d_nchw_relu if relu else xtc_conv2d_nchw
    st = fn(N, C, H, W, OC, R, S, sh, sw, ph, pw, x.data_ptr(), w.data_ptr(), out.data_ptr(),
            _dtype_code(torch, x), sched, _stream(torch, x.device))
    if st != XTC_OK:
        raise XtcError(st, fn.__name__)
    return out


# --------------------------------------- norms, 8-bit and grouped products


#: What ``layernorm`` returns: as ``RmsNorm``, and each row's ``mean`` (float32).
LayerNorm = namedtuple("LayerNorm", "out scale residual mean rstd")

#: What ``rmsnorm`` returns.  ``out``: the normed rows, in x's type or as
#: float8_e4m3fn with ``scale`` (else None); ``residual``: x plus the residual
#: (x itself when there was none); ``rstd``: one float32 a row, for the gradient.
RmsNorm = namedtuple("RmsNorm", "out scale residual rstd")


def _matrix(t, name, dtypes, shape=None, device=None):
    """Checks a [rows, cols] operand (of a family: [.., rows, cols]) with unit column stride."""
    if t.dtype not in dtypes:
        raise TypeError("%s must be %s, not %s" % (name, " or ".join(str(d).split(".")[1] for d in dtypes), t.dtype))
    if t.dim() != (2 if shape is None else len(shape)) or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError("%s must be a %d-D tensor with unit stride along its last axis"
                         % (name, 2 if shape is None else len(shape)))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be %s, not %s" % (name, list(shape), list(t.shape)))
    if not t.is_cuda or (device is not None and t.device != device):
        raise ValueError("%s must be a CUDA (HIP) tensor%s" % (name, "" if device is None else " on %s" % device))


def _vector(t, name, dtypes, length, device):
    if t.dtype not in dtypes:
        raise TypeError("%s must be %s, not %s" % (name, " or ".join(str(d).split(".")[1] for d in dtypes), t.dtype))
    if t.dim() != 1 or t.shape[0] != length or not t.is_contiguous():
        raise ValueError("%s must be a contiguous vector of %d values" % (name, length))
    if t.device != device:
        raise ValueError("%s must be on %s" % (name, device))


def _ld(t):
    """Row stride of a matrix in elements; where it has one row at most, its length."""
    return t.stride(-2) if t.shape[-2] > 1 else max(t.shape[-1], 1)


def _family(t):
    """Elements between the matrices of [G, rows, cols]."""
    return t.stride(0) if t.shape[0] > 1 else 0


def _ptr(t):
    return None if t is None else t.data_ptr()


def _blocks_of(n):
    return -(-n // 128)


def _on(torch, device):
    """The context in which launches go to ``device``."""
    return torch.cuda.device(device)


def _check(st, where):
    if st != XTC_OK:
        raise XtcError(st, where)


def rmsnorm(x, weight, residual=None, eps=1e-6, quantize=False):
    """Root-mean-square norm of each row of ``x`` (plus ``residual``): ``RmsNorm(out, scale, residual, rstd)``.

    ``x`` and ``residual`` [T, D] are float32 or bfloat16 CUDA tensors with unit column stride, ``weight`` [D] is of
    the same type or float32.  ``out`` is of x's type, or with ``quantize`` float8_e4m3fn with a float32 ``scale`` for
    each 128 columns.  ``rstd`` of rows without columns is NaN.  Enqueued on torch's current stream."""
    if _fast is not None:
        r = _fast.rmsnorm(x, weight, residual, eps, quantize)
        if r is not None:
            return RmsNorm._make(r)
    import torch
    kinds = (torch.float32, torch.bfloat16)
    _matrix(x, "x", kinds)
    T, D = x.shape
    _vector(weight, "weight", (torch.float32, x.dtype), D, x.device)
    if residual is not None:
        _matrix(residual, "residual", (x.dtype,), (T, D), x.device)
    out = torch.empty((T, D), dtype=torch.float8_e4m3fn if quantize else x.dtype, device=x.device)
    scale = torch.empty((T, _blocks_of(D)), dtype=torch.float32, device=x.device) if quantize else None
    total = x if residual is None else torch.empty((T, D), dtype=x.dtype, device=x.device)
    rstd = torch.empty(T, dtype=torch.float32, device=x.device)
    if D == 0:
        rstd.fill_(float("nan"))     # the mean of nothing, 0/0 (the library's call does nothing)
    code = _dtype_code(torch, x)
    _check(xtc_rmsnorm(T, D, x.data_ptr(), _ld(x), _ptr(residual), 0 if residual is None else _ld(residual),
                       weight.data_ptr(), eps, out.data_ptr(), max(D, 1), _ptr(scale), _blocks_of(D),
                       None if residual is None else total.data_ptr(), D, rstd.data_ptr(), code,
                       _dtype_code(torch, weight), XTC_FP8 if quantize else code, _stream(torch, x.device)),
           "xtc_rmsnorm")
    return RmsNorm(out, scale, total, rstd)


def rmsnorm_backward(dy, x, weight, rstd, dresidual=None):
    """``(dx, dweight)`` of ``rmsnorm``: ``x`` is the sum that was normed (its result's ``residual``), ``dresidual`` the
    gradient that reaches that sum from elsewhere.  ``dx`` (x's type) is the gradient of x and of the residual,
    ``dweight`` float32."""
    if _fast is not None:
        r = _fast.rmsnorm_backward(dy, x, weight, rstd, dresidual)
        if r is not None:
            return r
    import torch
    _matrix(x, "x", (torch.float32, torch.bfloat16))
    T, D = x.shape
    _matrix(dy, "dy", (x.dtype,), (T, D), x.device)
    _vector(weight, "weight", (torch.float32, x.dtype), D, x.device)
    _vector(rstd, "rstd", (torch.float32,), T, x.device)
    if dresidual is not None:
        _matrix(dresidual, "dresidual", (x.dtype,), (T, D), x.device)
    dx = torch.empty((T, D), dtype=x.dtype, device=x.device)
    dweight = torch.empty(D, dtype=torch.float32, device=x.device)
    size = xtc_rmsnorm_backward_workspace(T, D)
    work = torch.empty(max(size, 0), dtype=torch.uint8, device=x.device)
    _check(xtc_rmsnorm_backward(T, D, dy.data_ptr(), _ld(dy), x.data_ptr(), _ld(x), weight.data_ptr(),
                                rstd.data_ptr(), _ptr(dresidual), 0 if dresidual is None else _ld(dresidual),
                                dx.data_ptr(), max(D, 1), dweight.data_ptr(), work.data_ptr(), size,
                                _dtype_code(torch, x), _dtype_code(torch, weight), _stream(torch, x.device)),
           "xtc_rmsnorm_backward")
    return dx, dweight


def layernorm(x, weight, bias=None, residual=None, eps=1e-5, quantize=False):
    """Layer norm of each row of ``x`` (plus ``residual``): ``LayerNorm(out, scale, residual, mean, rstd)``.

    Operands and results as for ``rmsnorm``; ``bias`` [D] is of the weight's type.  ``mean`` and ``rstd`` of rows
    without columns are NaN.  Enqueued on torch's current stream."""
    if _fast is not None:
        r = _fast.layernorm(x, weight, bias, residual, eps, quantize)
        if r is not None:
            return LayerNorm._make(r)
    import torch
    kinds = (torch.float32, torch.bfloat16)
    _matrix(x, "x", kinds)
    T, D = x.shape
    _vector(weight, "weight", (torch.float32, x.dtype), D, x.device)
    if bias is not None:
        _vector(bias, "bias", (weight.dtype,), D, x.device)
    if residual is not None:
        _matrix(residual, "residual", (x.dtype,), (T, D), x.device)
    out = torch.empty((T, D), dtype=torch.float8_e4m3fn if quantize else x.dtype, device=x.device)
    scale = torch.empty((T, _blocks_of(D)), dtype=torch.float32, device=x.device) if quantize else None
    total = x if residual is None else torch.empty((T, D), dtype=x.dtype, device=x.device)
    mean, rstd = (torch.empty(T, dtype=torch.float32, device=x.device) for _ in range(2))
    if D == 0:
        mean.fill_(float("nan"))     # the means of nothing, 0/0 (the library's call does nothing)
        rstd.fill_(float("nan"))
    code = _dtype_code(torch, x)
    with _on(torch, x.device):
        _check(xtc_layernorm(T, D, x.data_ptr(), _ld(x), _ptr(residual), 0 if residual is None else _ld(residual),
                             weight.data_ptr(), _ptr(bias), eps, out.data_ptr(), max(D, 1), _ptr(scale), _blocks_of(D),
                             None if residual is None else total.data_ptr(), D, mean.data_ptr(), rstd.data_ptr(), code,
                             _dtype_code(torch, weight), XTC_FP8 if quantize else code, _stream(torch, x.device)),
               "xtc_layernorm")
    return LayerNorm(out, scale, total, mean, rstd)


def layernorm_backward(dy, x, weight, mean, rstd, dresidual=None):
    """``(dx, dweight, dbias)`` of ``layernorm``: ``x`` is the sum that was normed (its result's ``residual``),
    ``dresidual`` the gradient that reaches that sum from elsewhere.  ``dx`` (x's type) is the gradient of x and of the
    residual, ``dweight`` and ``dbias`` are float32."""
    if _fast is not None:
        r = _fast.layernorm_backward(dy, x, weight, mean, rstd, dresidual)
        if r is not None:
            return r
    import torch
    _matrix(x, "x", (torch.float32, torch.bfloat16))
    T, D = x.shape
    _matrix(dy, "dy", (x.dtype,), (T, D), x.device)
    _vector(weight, "weight", (torch.float32, x.dtype), D, x.device)
    _vector(mean, "mean", (torch.float32,), T, x.device)
    _vector(rstd, "rstd", (torch.float32,), T, x.device)
    if dresidual is not None:
        _matrix(dresidual, "dresidual", (x.dtype,), (T, D), x.device)
    dx = torch.empty((T, D), dtype=x.dtype, device=x.device)
    dweight, dbias = (torch.empty(D, dtype=torch.float32, device=x.device) for _ in range(2))
    size = xtc_layernorm_backward_workspace(T, D)
    work = torch.empty(max(size, 0), dtype=torch.uint8, device=x.device)
    with _on(torch, x.device):
        _check(xtc_layernorm_backward(T, D, dy.data_ptr(), _ld(dy), x.data_ptr(), _ld(x), weight.data_ptr(),
                                      mean.data_ptr(), rstd.data_ptr(), _ptr(dresidual),
                                      0 if dresidual is None else _ld(dresidual), dx.data_ptr(), max(D, 1),
                                      dweight.data_ptr(), dbias.data_ptr(), work.data_ptr(), size,
                                      _dtype_code(torch, x), _dtype_code(torch, weight), _stream(torch, x.device)),
               "xtc_layernorm_backward")
    return dx, dweight, dbias


def quantize_fp8(x, block_rows=1):
    """``(q, scale)``: the matrix ``x`` (float32 or bfloat16) as float8_e4m3fn with a float32 scale for each
    ``block_rows`` x 128 values; 1 for activations, 128 for weights."""
    if _fast is not None:
        r = _fast.quantize_fp8(x, block_rows)
        if r is not None:
            return r
    import torch
    _matrix(x, "x", (torch.float32, torch.bfloat16))
    if block_rows not in (1, 128):
        raise ValueError("block_rows must be 1 or 128")
    M, K = x.shape
    q = torch.empty((M, K), dtype=torch.float8_e4m3fn, device=x.device)
    scale = torch.empty((-(-M // block_rows), _blocks_of(K)), dtype=torch.float32, device=x.device)
    _check(xtc_quantize_fp8(M, K, x.data_ptr(), _ld(x), block_rows, q.data_ptr(), max(K, 1), scale.data_ptr(),
                            _blocks_of(K), _dtype_code(torch, x), _stream(torch, x.device)), "xtc_quantize_fp8")
    return q, scale


def _out_code(torch, dtype):
    if dtype is None or dtype == torch.float32:
        return XTC_F32
    if dtype == torch.bfloat16:
        return XTC_BF16
    raise TypeError("dtype must be float32 or bfloat16, not %s" % dtype)


def _result(torch, shape, out, dtype, device):
    """The output tensor of a product and its type's code."""
    if out is None:
        code = _out_code(torch, dtype)
        return torch.empty(shape, dtype=torch.bfloat16 if code else torch.float32, device=device), code
    _matrix(out, "out", (torch.float32, torch.bfloat16) if dtype is None else (dtype,), shape, device)
    return out, _out_code(torch, out.dtype)


def matmul_fp8(a, a_scale, b, b_scale, out=None, relu=False, dtype=None):
    """``out = A @ B.T`` (``relu`` fused) of block-scaled operands: ``a`` [M, K] with ``a_scale`` [M, ceil(K/128)] and
    ``b`` [N, K] with ``b_scale`` [ceil(N/128), ceil(K/128)], float8_e4m3fn and float32, as ``quantize_fp8`` gives them
    with ``block_rows`` 1 and 128.  ``out`` [M, N] is float32 or bfloat16 (``dtype``, when allocated here; float32
    unless given).  A float32 result has float32 sums.  For a bfloat16 one each eight consecutive products lose what lies
    more than 13 binary places below their largest: far below the result's rounding, but for sums that cancel, where
    the error can be 2^-10 of the largest product of each eight."""
    if _fast is not None:
        r = _fast.matmul_fp8(a, a_scale, b, b_scale, out, relu, dtype)
        if r is not None:
            return r
    import torch
    e4m3, f32 = (torch.float8_e4m3fn,), (torch.float32,)
    _matrix(a, "a", e4m3)
    M, K = a.shape
    _matrix(b, "b", e4m3, None, a.device)
    N = b.shape[0]
    if b.shape[1] != K:
        raise ValueError("inner dimensions differ: %d vs %d" % (K, b.shape[1]))
    _matrix(a_scale, "a_scale", f32, (M, _blocks_of(K)), a.device)
    _matrix(b_scale, "b_scale", f32, (_blocks_of(N), _blocks_of(K)), a.device)
    out, code = _result(torch, (M, N), out, dtype, a.device)
    _check(xtc_matmul_fp8(M, N, K, a.data_ptr(), _ld(a), a_scale.data_ptr(), _ld(a_scale), b.data_ptr(), _ld(b),
                          b_scale.data_ptr(), _ld(b_scale), out.data_ptr(), _ld(out), code, int(relu),
                          _stream(torch, a.device)), "xtc_matmul_fp8")
    return out


_ACTIVATIONS = {None: XTC_NO_ACTIVATION, "relu": XTC_RELU, "gelu": XTC_GELU, "gelu_tanh": XTC_GELU_TANH,
                "silu": XTC_SILU}


def _activation(name):
    if name not in _ACTIVATIONS:
        raise ValueError("activation must be None, 'relu', 'gelu', 'gelu_tanh' or 'silu', not %r" % (name,))
    return _ACTIVATIONS[name]


def linear(a, b, bias=None, residual=None, activation=None, transpose_b=False, keep=False, out=None, dtype=None):
    """``out = act(a @ b + bias) + residual``, all of it in one kernel and float32, rounded once.

    ``a`` [T, K] and ``b`` [K, N] ([N, K] with ``transpose_b``) are bfloat16, ``bias`` [N] and ``residual`` [T, N] float32
    or bfloat16 each.  ``activation``: None, "relu", "gelu" (by the error function), "gelu_tanh" or "silu".  ``out``
    [T, N] is float32 or bfloat16 (``dtype``, when allocated here; float32 unless given), and may be ``residual`` itself.
    With ``keep`` the result is ``(out, z)``, z = a @ b + bias in out's type for ``activation_backward``.  The gradient of
    ``a`` is the same call on z's gradient with the other ``transpose_b``."""
    code_act = _activation(activation)
    if _fast is not None:
        r = _fast.linear(a, b, bias, residual, code_act, transpose_b, keep, out, dtype)
        if r is not None:
            return r
    import torch
    bf16, either = (torch.bfloat16,), (torch.float32, torch.bfloat16)
    _matrix(a, "a", bf16)
    T, K = a.shape
    _matrix(b, "b", bf16, None, a.device)
    N = b.shape[0 if transpose_b else 1]
    if b.shape[1 if transpose_b else 0] != K:
        raise ValueError("inner dimensions differ: %d vs %d" % (K, b.shape[1 if transpose_b else 0]))
    if bias is not None:
        _vector(bias, "bias", either, N, a.device)
    if residual is not None:
        _matrix(residual, "residual", either, (T, N), a.device)
    out, code = _result(torch, (T, N), out, dtype, a.device)
    z = torch.empty((T, N), dtype=out.dtype, device=a.device) if keep else None
    size = xtc_linear_workspace(T, N, K, a.data_ptr(), _ld(a), b.data_ptr(), _ld(b), int(transpose_b))
    work = torch.empty(max(size, 0), dtype=torch.uint8, device=a.device)
    with _on(torch, a.device):
        _check(xtc_linear(T, N, K, a.data_ptr(), _ld(a), b.data_ptr(), _ld(b), int(transpose_b), _ptr(bias),
                          XTC_F32 if bias is None else _dtype_code(torch, bias), _ptr(residual),
                          0 if residual is None else _ld(residual),
                          XTC_F32 if residual is None else _dtype_code(torch, residual), code_act, out.data_ptr(),
                          _ld(out), _ptr(z), max(N, 1), work.data_ptr(), size, XTC_BF16, code, _stream(torch, a.device)),
               "xtc_linear")
    return (out, z) if keep else out


def linear_wgrad(a, dy, out=None, dtype=None):
    """The gradient of ``linear``'s ``b`` [K, N] (float32 or bfloat16: ``dtype``): ``a.T @ dy``, of ``a`` [T, K] and the
    gradient ``dy`` [T, N] of a @ b, both bfloat16.  Of a ``b`` that is [N, K]: ``linear_wgrad(dy, a)``."""
    if _fast is not None:
        r = _fast.linear_wgrad(a, dy, out, dtype)
        if r is not None:
            return r
    import torch
    bf16 = (torch.bfloat16,)
    _matrix(a, "a", bf16)
    T, K = a.shape
    _matrix(dy, "dy", bf16, None, a.device)
    N = dy.shape[1]
    if dy.shape[0] != T:
        raise ValueError("a and dy have %d and %d rows" % (T, dy.shape[0]))
    out, code = _result(torch, (K, N), out, dtype, a.device)
    size = xtc_linear_wgrad_workspace(T, N, K, a.data_ptr(), _ld(a), dy.data_ptr(), _ld(dy))
    work = torch.empty(max(size, 0), dtype=torch.uint8, device=a.device)
    with _on(torch, a.device):
        _check(xtc_linear_wgrad(T, N, K, a.data_ptr(), _ld(a), dy.data_ptr(), _ld(dy), out.data_ptr(), _ld(out),
                                work.data_ptr(), size, XTC_BF16, code, _stream(torch, a.device)), "xtc_linear_wgrad")
    return out


def activation_backward(dy, z, activation):
    """``(dz, dbias)`` of ``linear``: ``dy`` [T, N] is the gradient of its result, ``z`` what it kept (float32 or bfloat16
    each; z is not read where ``activation`` is None).  ``dz = dy * act'(z)`` is bfloat16, as ``linear`` and
    ``linear_wgrad`` take it; ``dbias`` [N], its column sums before that rounding, float32."""
    code_act = _activation(activation)
    if _fast is not None:
        r = _fast.activation_backward(dy, z, code_act)
        if r is not None:
            return r
    import torch
    either = (torch.float32, torch.bfloat16)
    _matrix(dy, "dy", either)
    T, N = dy.shape
    if activation is None:
        z = dy
    _matrix(z, "z", either, (T, N), dy.device)
    dz = torch.empty((T, N), dtype=torch.bfloat16, device=dy.device)
    dbias = torch.empty(N, dtype=torch.float32, device=dy.device)
    size = xtc_activation_backward_workspace(T, N)
    work = torch.empty(max(size, 0), dtype=torch.uint8, device=dy.device)
    with _on(torch, dy.device):
        _check(xtc_activation_backward(T, N, dy.data_ptr(), _ld(dy), _dtype_code(torch, dy), z.data_ptr(), _ld(z),
                                       _dtype_code(torch, z), code_act, dz.data_ptr(), max(N, 1), dbias.data_ptr(),
                                       work.data_ptr(), size, _stream(torch, dy.device)), "xtc_activation_backward")
    return dz, dbias


def matmul_grouped(a, b, ends, transpose_b=False, out=None, relu=False, dtype=None):
    """``out[i] = a[i] @ b[g]`` (``relu`` fused) for the rows ``i`` of group ``g``, which end before ``ends[g]``.

    ``a`` [T, K] and ``b`` [G, K, N] ([G, N, K] with ``transpose_b``) are bfloat16, ``ends`` [G] int32, ascending, on
    the same device; rows past ``ends[-1]`` are zeros in ``out`` [T, N] (float32 or bfloat16: ``dtype``).  The
    gradient of ``a`` is the same call on out's gradient with the other ``transpose_b``."""
    if _fast is not None:
        r = _fast.matmul_grouped(a, b, ends, transpose_b, out, relu, dtype)
        if r is not None:
            return r
    import torch
    bf16 = (torch.bfloat16,)
    _matrix(a, "a", bf16)
    T, K = a.shape
    if b.dim() != 3:
        raise ValueError("b must be a 3-D tensor")
    G, N = b.shape[0], b.shape[1 if transpose_b else 2]
    _matrix(b, "b", bf16, (G, N, K) if transpose_b else (G, K, N), a.device)
    _vector(ends, "ends", (torch.int32,), G, a.device)
    out, code = _result(torch, (T, N), out, dtype, a.device)
    _check(xtc_matmul_grouped(G, T, N, K, a.data_ptr(), _ld(a), b.data_ptr(), _ld(b), _family(b), int(transpose_b),
                              ends.data_ptr(), out.data_ptr(), _ld(out), XTC_BF16, code, int(relu),
                              _stream(torch, a.device)), "xtc_matmul_grouped")
    return out


def matmul_grouped_wgrad(a, dy, ends, out=None, dtype=None):
    """The gradient of ``matmul_grouped``'s ``b`` [G, K, N] (float32 or bfloat16: ``dtype``): ``a[rows].T @ dy[rows]``
    over each group's rows, zeros for an empty group.  ``a`` [T, K] and ``dy`` [T, N] are bfloat16."""
    if _fast is not None:
        r = _fast.matmul_grouped_wgrad(a, dy, ends, out, dtype)
        if r is not None:
            return r
    import torch
    bf16 = (torch.bfloat16,)
    _matrix(a, "a", bf16)
    T, K = a.shape
    _matrix(dy, "dy", bf16, None, a.device)
    N = dy.shape[1]
    if dy.shape[0] != T:
        raise ValueError("a and dy have %d and %d rows" % (T, dy.shape[0]))
    if ends.dim() != 1:
        raise ValueError("ends must be a vector")
    G = ends.shape[0]
    _vector(ends, "ends", (torch.int32,), G, a.device)
    out, code = _result(torch, (G, K, N), out, dtype, a.device)
    _check(xtc_matmul_grouped_wgrad(G, T, N, K, a.data_ptr(), _ld(a), dy.data_ptr(), _ld(dy), ends.data_ptr(),
                                    out.data_ptr(), _ld(out), _family(out), XTC_BF16, code,
                                    _stream(torch, a.device)), "xtc_matmul_grouped_wgrad")
    return out


def matmul_grouped_fp8(a, a_scale, b, b_scale, ends, out=None, relu=False, dtype=None):
    """``matmul_grouped`` of block-scaled operands: ``a`` [T, K] with ``a_scale`` [T, ceil(K/128)], ``b`` [G, N, K] with
    ``b_scale`` [G, ceil(N/128), ceil(K/128)] (float8_e4m3fn and float32); ``out`` [T, N], its sums as ``matmul_fp8``'s."""
    if _fast is not None:
        r = _fast.matmul_grouped_fp8(a, a_scale, b, b_scale, ends, out, relu, dtype)
        if r is not None:
            return r
    import torch
    e4m3, f32 = (torch.float8_e4m3fn,), (torch.float32,)
    _matrix(a, "a", e4m3)
    T, K = a.shape
    if b.dim() != 3:
        raise ValueError("b must be a 3-D tensor")
    G, N = b.shape[:2]
    _matrix(b, "b", e4m3, (G, N, K), a.device)
    _matrix(a_scale, "a_scale", f32, (T, _blocks_of(K)), a.device)
    _matrix(b_scale, "b_scale", f32, (G, _blocks_of(N), _blocks_of(K)), a.device)
    _vector(ends, "ends", (torch.int32,), G, a.device)
    out, code = _result(torch, (T, N), out, dtype, a.device)
    _check(xtc_matmul_grouped_fp8(G, T, N, K, a.data_ptr(), _ld(a), a_scale.data_ptr(), _ld(a_scale), b.data_ptr(),
                                  _ld(b), _family(b), b_scale.data_ptr(), _ld(b_scale), _family(b_scale),
                                  ends.data_ptr(), out.data_ptr(), _ld(out), code, int(relu),
                                  _stream(torch, a.device)), "xtc_matmul_grouped_fp8")
    return out


# ----------------------------------------------- the routing of a mixture


#: What ``route_experts`` returns.  ``expert``, ``p``, ``row`` [T, top]: each token's experts (the highest score first),
#: their weights, and the place of each choice among the rows sorted by expert; ``token`` [T * top]: the token of each of
#: these rows; ``counts``, ``ends`` [E]: the rows of each expert and where they end (``matmul_grouped``'s ``ends``);
#: ``loss``: the balance loss, a float32 scalar.  Places and counts are int32.  They may share one storage, which lives as
#: long as any of them.
Routing = namedtuple("Routing", "expert p row token counts ends loss")


def _block(t, name, dtype, shape, device):
    """Checks a contiguous operand."""
    if t.dtype != dtype:
        raise TypeError("%s must be %s, not %s" % (name, str(dtype).split(".")[1], t.dtype))
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError("%s must be contiguous %s" % (name, list(shape)))
    if t.device != device:
        raise ValueError("%s must be on %s" % (name, device))


def route_experts(scores, top, mask=None):
    """The ``top`` experts of each token: ``Routing(expert, p, row, token, counts, ends, loss)``.

    ``scores`` [T, E] are float32 or bfloat16, E at most 1024 and ``top`` at most 16.  ``p`` is the softmax over a token's
    chosen scores; of equal scores the lowest expert comes first.  Tokens where the boolean ``mask`` [T] is false go to
    no expert: their ``expert`` and ``row`` are -1, their ``p`` zeros, and ``token`` is -1 for the rows behind ``ends[-1]``.
    A score of -inf has the weight 0: its expert is chosen only where fewer than ``top`` others are left.
    The balance loss is ``E / (top * n**2) * sum_e counts[e] * sum_t softmax(scores[t])[e]`` over the n tokens that are
    left (1 where every expert has as many).  Nothing waits for the GPU."""
    if _fast is not None:
        r = _fast.route_experts(scores, top, mask)
        if r is not None:
            return Routing._make(r)
    import torch
    _matrix(scores, "scores", (torch.float32, torch.bfloat16))
    T, E = scores.shape
    if mask is not None:
        _block(mask, "mask", torch.bool, (T,), scores.device)
    if not 1 <= top <= E:
        raise ValueError("top must be from 1 to the %d experts, not %d" % (E, top))
    i32, f32 = (dict(dtype=d, device=scores.device) for d in (torch.int32, torch.float32))
    r = Routing(torch.empty((T, top), **i32), torch.empty((T, top), **f32), torch.empty((T, top), **i32),
                torch.empty(T * top, **i32), torch.empty(E, **i32), torch.empty(E, **i32), torch.empty((), **f32))
    size = xtc_route_experts_workspace(T, E)
    work = torch.empty(max(size, 0), dtype=torch.uint8, device=scores.device)
    with _on(torch, scores.device):
        _check(xtc_route_experts(T, E, top, scores.data_ptr(), _ld(scores), _ptr(mask), r.expert.data_ptr(),
                                 r.p.data_ptr(), r.row.data_ptr(), r.token.data_ptr(), r.counts.data_ptr(),
                                 r.ends.data_ptr(), r.loss.data_ptr(), work.data_ptr(), size,
                                 _dtype_code(torch, scores), _stream(torch, scores.device)), "xtc_route_experts")
    return r


def route_experts_backward(dp, scores, expert, p, counts, dloss=0.0, dtype=None):
    """The gradient of ``route_experts``'s ``scores`` [T, E] (of their type, or ``dtype``) from that of ``p`` (``dp``
    [T, top] float32, or None) and the balance loss's, the number ``dloss``; ``expert``, ``p`` and ``counts`` are its results."""
    if _fast is not None:
        r = _fast.route_experts_backward(dp, scores, expert, p, counts, dloss, dtype)
        if r is not None:
            return r
    import torch
    _matrix(scores, "scores", (torch.float32, torch.bfloat16))
    T, E = scores.shape
    if expert.dim() != 2:
        raise ValueError("expert must be [T, top]")
    top = expert.shape[1]
    _block(expert, "expert", torch.int32, (T, top), scores.device)
    _block(p, "p", torch.float32, (T, top), scores.device)
    _block(counts, "counts", torch.int32, (E,), scores.device)
    if dp is not None:
        _block(dp, "dp", torch.float32, (T, top), scores.device)
    code = _out_code(torch, scores.dtype if dtype is None else dtype)
    ds = torch.empty((T, E), dtype=torch.bfloat16 if code else torch.float32, device=scores.device)
    with _on(torch, scores.device):
        _check(xtc_route_experts_backward(T, E, top, _ptr(dp), scores.data_ptr(), _ld(scores), expert.data_ptr(),
                                          p.data_ptr(), counts.data_ptr(), dloss, ds.data_ptr(), max(E, 1),
                                          _dtype_code(torch, scores), code, _stream(torch, scores.device)),
               "xtc_route_experts_backward")
    return ds


def combine_experts(rows, row, p=None, residual=None, dtype=None):
    """``out[t] = residual[t] + sum_j p[t, j] * rows[row[t, j]]`` [T, D] (float32 or bfloat16: ``dtype``): the experts'
    rows back at their tokens.  ``rows`` [R, D] and ``residual`` [T, D] are float32 or bfloat16, ``row`` int32 and ``p``
    float32 [T, top] as ``route_experts`` gives them; -1 in ``row`` counts as a row of zeros, no ``p`` as ones (the
    gradient of ``x[token]``)."""
    if _fast is not None:
        r = _fast.combine_experts(rows, row, p, residual, dtype)
        if r is not None:
            return r
    import torch
    either = (torch.float32, torch.bfloat16)
    _matrix(rows, "rows", either)
    R, D = rows.shape
    if row.dim() != 2:
        raise ValueError("row must be [T, top]")
    T, top = row.shape
    _block(row, "row", torch.int32, (T, top), rows.device)
    if p is not None:
        _block(p, "p", torch.float32, (T, top), rows.device)
    if residual is not None:
        _matrix(residual, "residual", either, (T, D), rows.device)
    code = _out_code(torch, dtype)
    out = torch.empty((T, D), dtype=torch.bfloat16 if code else torch.float32, device=rows.device)
    with _on(torch, rows.device):
        _check(xtc_combine_experts(T, top, D, R, rows.data_ptr(), _ld(rows) if R else max(D, 1), row.data_ptr(), _ptr(p),
                                   _ptr(residual), 0 if residual is None else _ld(residual),
                                   XTC_F32 if residual is None else _dtype_code(torch, residual), out.data_ptr(),
                                   max(D, 1), _dtype_code(torch, rows), code, _stream(torch, rows.device)),
               "xtc_combine_experts")
    return out


def combine_experts_backward(dout, rows, row, token, p):
    """``(drows, dp)`` of ``combine_experts`` from its result's gradient ``dout`` [T, D]; ``rows`` [T * top, D], ``row``,
    ``token`` and ``p`` as ``route_experts`` sorts them.  ``drows`` is of the rows' type, zeros where ``token`` is -1;
    ``dp`` [T, top] float32."""
    if _fast is not None:
        r = _fast.combine_experts_backward(dout, rows, row, token, p)
        if r is not None:
            return r
    import torch
    either = (torch.float32, torch.bfloat16)
    _matrix(rows, "rows", either)
    R, D = rows.shape
    if row.dim() != 2:
        raise ValueError("row must be [T, top]")
    T, top = row.shape
    if R != T * top:
        raise ValueError("rows must hold %d rows, not %d" % (T * top, R))
    _block(row, "row", torch.int32, (T, top), rows.device)
    _block(token, "token", torch.int32, (R,), rows.device)
    _block(p, "p", torch.float32, (T, top), rows.device)
    _matrix(dout, "dout", either, (T, D), rows.device)
    drows = torch.empty((R, D), dtype=rows.dtype, device=rows.device)
    dp = torch.empty((T, top), dtype=torch.float32, device=rows.device)
    with _on(torch, rows.device):
        _check(xtc_combine_experts_backward(T, top, D, dout.data_ptr(), _ld(dout), _dtype_code(torch, dout),
                                            rows.data_ptr(), _ld(rows), row.data_ptr(), token.data_ptr(), p.data_ptr(),
                                            drows.data_ptr(), max(D, 1), dp.data_ptr(), _dtype_code(torch, rows),
                                            _stream(torch, rows.device)), "xtc_combine_experts_backward")
    return drows, dp
