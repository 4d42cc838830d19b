"""Thin Python binding of the C ABI in ``include/fireq.h``: argument marshalling only.

Every step of the path runs in the HIP kernels of ``libfireq.so``; torch is used for device
memory and the current stream.  There is no CPU fallback: if the library cannot be loaded or a
tensor is not on the GPU, the call raises.

The calls of a running model, and those that prepare its weights and caches, marshal their arguments in native code
(``_fq_marshal-*.so``, see its source); whatever that does not take -- another kind of tensor, a wrong shape, an argument to
be refused -- comes back as None and goes through the Python form below it, which decides and raises.  Without that
extension every call takes its Python form.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import warnings
from typing import Optional, Tuple

import torch

from . import build as _build

GROUP = 128

_lib = None
_marshal = None

# the C functions the marshalling calls, in the order it expects them
_MARSHALLED = ("fq_quantize_act", "fq_quantize_act_ws", "fq_packed_weight_bytes", "fq_w4a8_gemm_workspace_bytes", "fq_w4a8_gemm_ws",
               "fq_w4a8_gemm_swiglu_ws", "fq_w4a8_gemm_add_ws", "fq_w4a8_gemm_swiglu_quant_ws", "fq_w4a8_linear_workspace_bytes",
               "fq_w4a8_linear_ws", "fq_kv4_packed_bytes", "fq_kv4_scores", "fq_kv4_output_workspace_bytes", "fq_kv4_output_ws",
               "fq_kv4_pack", "fq_pack_weights", "fq_cas_scales_workspace_bytes", "fq_cas_scales_ws", "fq_pts_exponent_workspace_bytes",
               "fq_pts_exponent_ws", "fq_quantize_weights", "fq_rmsnorm", "fq_rmsnorm_quant_ws", "fq_kv4_append", "fq_kv4_read",
               "fq_kv4_attention_workspace_bytes", "fq_kv4_attention_ws", "fq_kv4_attention_prefix_ws")


class FireqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (where, status_string(status), status))


def lib() -> ctypes.CDLL:
    """The loaded shared library (built in-tree on first use if it was never built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB_PATH):
        _build.build_library()
    L = ctypes.CDLL(_build.LIB_PATH)
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    L.fq_w4a8_gemm.restype = ci
    L.fq_w4a8_gemm.argtypes = [vp, vp, vp, vp, cf, vp, ci, ci, ci, vp]
    L.fq_w4a8_gemm_static.restype = ci
    L.fq_w4a8_gemm_static.argtypes = [vp, vp, vp, vp, cf, vp, ci, ci, ci, vp]
    L.fq_w4a8_gemm_static_max_workspace.restype = ctypes.c_size_t
    L.fq_w4a8_gemm_static_max_workspace.argtypes = []
    L.fq_w4a8_gemm_lut.restype = ci
    L.fq_w4a8_gemm_lut.argtypes = [vp, vp, vp, vp, cf, vp, ci, ci, ci, vp]
    L.fq_kv4_packed_bytes.restype = ctypes.c_size_t
    L.fq_kv4_packed_bytes.argtypes = [ci, ci, ci]
    L.fq_kv4_pack.restype = ci
    L.fq_kv4_pack.argtypes = [vp, vp, ci, ci, ci, vp]
    L.fq_kv4_unpack.restype = ci
    L.fq_kv4_unpack.argtypes = [vp, vp, ci, ci, ci, vp]
    L.fq_kv4_scores.restype = ci
    L.fq_kv4_scores.argtypes = [vp, vp, vp, vp, cf, vp, ci, ci, ci, vp]
    L.fq_kv4_output.restype = ci
    L.fq_kv4_output.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, vp]
    L.fq_kv4_output_workspace_bytes.restype = ctypes.c_size_t
    L.fq_kv4_output_workspace_bytes.argtypes = [ci, ci, ci]
    L.fq_kv4_output_ws.restype = ci
    L.fq_kv4_output_ws.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, vp, ctypes.c_size_t, vp]
    c64 = ctypes.c_int64
    L.fq_rmsnorm.restype = ci
    L.fq_rmsnorm.argtypes = [vp, vp, vp, cf, vp, vp, ci, ci, vp]
    L.fq_rmsnorm_quant_ws.restype = ci
    L.fq_rmsnorm_quant_ws.argtypes = [vp, vp, vp, cf, vp, vp, vp, ci, ci, vp, ctypes.c_size_t, vp]
    L.fq_kv4_append.restype = ci
    L.fq_kv4_append.argtypes = [vp, c64, vp, ci, vp, vp, ci, vp, vp, vp, c64, c64, ci, ci, ci, ci, ci, vp]
    L.fq_kv4_read.restype = ci
    L.fq_kv4_read.argtypes = [vp, c64, c64, ci, ci, vp, vp, vp, ci, ci, vp]
    L.fq_kv4_attention_workspace_bytes.restype = ctypes.c_size_t
    L.fq_kv4_attention_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    L.fq_kv4_attention_ws.restype = ci
    L.fq_kv4_attention_ws.argtypes = [vp, vp, vp, c64, c64, ci, ci, vp, ci, vp, cf, vp, ci, ci, ci, ci, vp, ctypes.c_size_t, vp]
    L.fq_kv4_attention_prefix_ws.restype = ci
    L.fq_kv4_attention_prefix_ws.argtypes = [vp, vp, vp, c64, c64, ci, ci, vp, ci, vp, ci, vp, cf, vp, ci, ci, ci, ci, vp, ctypes.c_size_t, vp]
    L.fq_w4a8_gemm_ws.restype = ci
    L.fq_w4a8_gemm_ws.argtypes = [vp, vp, vp, vp, cf, vp, ci, ci, ci, vp, ctypes.c_size_t, ci, vp]
    L.fq_w4a8_gemm_add_ws.restype = ci
    L.fq_w4a8_gemm_add_ws.argtypes = [vp, vp, vp, vp, cf, vp, vp, ci, ci, ci, vp, ctypes.c_size_t, ci, vp]
    L.fq_w4a8_gemm_swiglu_quant_ws.restype = ci
    L.fq_w4a8_gemm_swiglu_quant_ws.argtypes = [vp, vp, vp, vp, cf, vp, vp, vp, ci, ci, ci, vp, ctypes.c_size_t, ci, vp,
                                               ctypes.c_size_t, vp]
    L.fq_w4a8_gemm_swiglu_ws.restype = ci
    L.fq_w4a8_gemm_swiglu_ws.argtypes = [vp, vp, vp, vp, cf, vp, ci, ci, ci, vp, ctypes.c_size_t, ci, vp]
    L.fq_quantize_act_ws.restype = ci
    L.fq_quantize_act_ws.argtypes = [vp, vp, vp, ci, ci, vp, ctypes.c_size_t, vp]
    L.fq_w4a8_gemm_workspace_bytes.restype = ctypes.c_size_t
    L.fq_w4a8_gemm_workspace_bytes.argtypes = [ci, ci, ci]
    L.fq_quantize_act.restype = ci
    L.fq_quantize_act.argtypes = [vp, vp, vp, ci, ci, vp]
    L.fq_packed_weight_bytes.restype = ctypes.c_size_t
    L.fq_packed_weight_bytes.argtypes = [ci, ci]
    L.fq_pack_weights.restype = ci
    L.fq_pack_weights.argtypes = [vp, vp, ci, ci, vp]
    L.fq_unpack_weights.restype = ci
    L.fq_unpack_weights.argtypes = [vp, vp, ci, ci, vp]
    L.fq_w4a8_linear_workspace_bytes.restype = ctypes.c_size_t
    L.fq_w4a8_linear_workspace_bytes.argtypes = [ci, ci, ci]
    L.fq_w4a8_linear_ws.restype = ci
    L.fq_w4a8_linear_ws.argtypes = [vp, vp, vp, cf, vp, ci, ci, ci, vp, ctypes.c_size_t, vp]
    L.fq_cas_scales.restype = ci
    L.fq_cas_scales.argtypes = [vp, cf, vp, ci, ci, vp]
    L.fq_pts_exponent.restype = ci
    L.fq_pts_exponent.argtypes = [vp, vp, vp, ci, ci, vp]
    L.fq_cas_scales_workspace_bytes.restype = ctypes.c_size_t
    L.fq_cas_scales_workspace_bytes.argtypes = [ci, ci]
    L.fq_cas_scales_ws.restype = ci
    L.fq_cas_scales_ws.argtypes = [vp, cf, vp, ci, ci, vp, ctypes.c_size_t, vp]
    L.fq_pts_exponent_workspace_bytes.restype = ctypes.c_size_t
    L.fq_pts_exponent_workspace_bytes.argtypes = [ci, ci]
    L.fq_pts_exponent_ws.restype = ci
    L.fq_pts_exponent_ws.argtypes = [vp, vp, vp, ci, ci, vp, ctypes.c_size_t, vp]
    L.fq_quantize_weights.restype = ci
    L.fq_quantize_weights.argtypes = [vp, vp, ci, ci, vp, vp, ci, ci, vp]
    L.fq_w4a8_gemm_plan.restype = ci
    L.fq_w4a8_gemm_plan.argtypes = [ci, ci, ci, ci, ctypes.POINTER(ctypes.c_int)]
    L.fq_diag_stream_read.restype = ci
    L.fq_diag_stream_read.argtypes = [vp, ctypes.c_size_t, vp, vp]
    L.fq_diag_stream_read_sink_bytes.restype = ctypes.c_size_t
    L.fq_diag_stream_read_sink_bytes.argtypes = []
    L.fq_test_force_kernel.restype = ci
    L.fq_test_force_kernel.argtypes = [ctypes.c_char_p]
    L.fq_layout_version.restype = ci
    L.fq_layout_version.argtypes = []
    L.fq_status_string.restype = ctypes.c_char_p
    L.fq_status_string.argtypes = [ci]
    _lib = L
    return L


class _PythonForms:
    """In the place of the native marshalling where there is none: declines every call."""

    def __getattr__(self, name):
        return _decline


def _decline(*args):
    return None


def marshal():
    """The native marshalling, bound to the loaded library (built in-tree on first use if it was never built from these
    sources for this torch and Python).  Where it can be neither built nor loaded (it needs a C++ compiler and the headers of
    torch and Python, the library itself does not), a warning is given once and every call takes its Python form."""
    global _marshal
    if _marshal is None:
        L = lib()
        try:
            path = _build.marshal_path()
            if not os.path.exists(path):
                _build.build_marshal()
            loader = importlib.machinery.ExtensionFileLoader("_fq_marshal", path)
            m = importlib.util.module_from_spec(importlib.util.spec_from_loader("_fq_marshal", loader))
            loader.exec_module(m)
            m.bind(*(ctypes.cast(getattr(L, name), ctypes.c_void_p).value for name in _MARSHALLED))
        except Exception as e:
            warnings.warn("calls are marshalled in Python (about 6 us more each): " + str(e), RuntimeWarning, stacklevel=3)
            m = _PythonForms()
        _marshal = m
    return _marshal


def status_string(status: int) -> str:
    return lib().fq_status_string(int(status)).decode()


def fq_layout_version() -> int:
    return int(lib().fq_layout_version())


def fq_packed_weight_bytes(N: int, K: int) -> int:
    return int(lib().fq_packed_weight_bytes(int(N), int(K)))


def _dev(t: torch.Tensor, dtype, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a GPU tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t


def _stream() -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def fq_cas_scales(W: torch.Tensor, target: float) -> torch.Tensor:
    """float32 [K]: lambda[k] = target / absmean_n(W[n,k]) of a bf16 weight matrix [N,K]."""
    r = (_marshal or marshal()).cas_scales(W, target)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_cas_scales")
        return r
    W = _dev(W, torch.bfloat16, "W")
    N, K = W.shape
    lam = torch.empty((K,), dtype=torch.float32, device=W.device)
    need = lib().fq_cas_scales_workspace_bytes(N, K)
    ws = torch.empty((need,), dtype=torch.uint8, device=W.device) if need else None
    rc = lib().fq_cas_scales_ws(W.data_ptr(), ctypes.c_float(float(target)), lam.data_ptr(), N, K, ws.data_ptr() if need else 0, need,
                                _stream())
    if rc != 0:
        raise FireqError(rc, "fq_cas_scales")
    return lam


def _lambda_ptr(lam, K):
    if lam is None:
        return 0
    lam = _dev(lam, torch.float32, "lam")
    if lam.numel() != K:
        raise FireqError(-2, "lambda")
    return lam.data_ptr()


def fq_pts_exponent(W: torch.Tensor, lam: Optional[torch.Tensor] = None) -> torch.Tensor:
    """int32 device tensor of 16 ints whose first element is the per-tensor exponent n (delta = 2^n) of the
    bf16 matrix W [N,K] scaled by lam [K]; reading it (``int(t[0])``) synchronises, the call does not."""
    r = (_marshal or marshal()).pts_exponent(W, lam)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_pts_exponent")
        return r
    W = _dev(W, torch.bfloat16, "W")
    N, K = W.shape
    out = torch.empty((16,), dtype=torch.int32, device=W.device)
    need = lib().fq_pts_exponent_workspace_bytes(N, K)
    ws = torch.empty((need,), dtype=torch.uint8, device=W.device) if need else None
    rc = lib().fq_pts_exponent_ws(W.data_ptr(), _lambda_ptr(lam, K), out.data_ptr(), N, K, ws.data_ptr() if need else 0, need, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_pts_exponent")
    return out


def fq_quantize_weights(W: torch.Tensor, lam: Optional[torch.Tensor] = None, n_pts: int = 0,
                        sigma_nearest: bool = False):
    """(int8 [N,K] INT4 codes, uint8 [N,K/128] E4M3 group scales) of W * lam * 2^n_pts."""
    r = (_marshal or marshal()).quantize_weights(W, lam, n_pts, sigma_nearest)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_quantize_weights")
        return r
    W = _dev(W, torch.bfloat16, "W")
    N, K = W.shape
    if K % GROUP:
        raise FireqError(-2, "fq_quantize_weights")
    q = torch.empty((N, K), dtype=torch.int8, device=W.device)
    gs = torch.empty((N, K // GROUP), dtype=torch.uint8, device=W.device)
    rc = lib().fq_quantize_weights(W.data_ptr(), _lambda_ptr(lam, K), int(n_pts), 1 if sigma_nearest else 0,
                                   q.data_ptr(), gs.data_ptr(), N, K, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_quantize_weights")
    return q, gs


def fq_pack_weights(q: torch.Tensor) -> torch.Tensor:
    """int8 [N,K] codes in -8..7 -> packed uint8 buffer of fq_packed_weight_bytes(N,K) bytes."""
    r = (_marshal or marshal()).pack_weights(q)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_pack_weights")
        return r
    q = _dev(q, torch.int8, "q")
    N, K = q.shape
    nbytes = fq_packed_weight_bytes(N, K)
    if nbytes == 0:
        raise FireqError(-2, "fq_pack_weights")
    out = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    rc = lib().fq_pack_weights(q.data_ptr(), out.data_ptr(), N, K, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_pack_weights")
    return out


def fq_unpack_weights(packed: torch.Tensor, N: int, K: int) -> torch.Tensor:
    packed = _dev(packed, torch.uint8, "packed")
    if packed.numel() < fq_packed_weight_bytes(N, K) or fq_packed_weight_bytes(N, K) == 0:
        raise FireqError(-2, "fq_unpack_weights")
    out = torch.empty((N, K), dtype=torch.int8, device=packed.device)
    rc = lib().fq_unpack_weights(packed.data_ptr(), out.data_ptr(), N, K, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_unpack_weights")
    return out


def fq_quantize_act(X: torch.Tensor, workspace: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """bf16 [M,K] -> (uint8 [M,K] E4M3 codes, float32 [M] per-row scales).

    With `workspace` (a device tensor of fq_w4a8_gemm_workspace_bytes(M, N, K) bytes or more) the call is
    fq_quantize_act_ws, which also prepares that workspace for fq_w4a8_gemm(..., workspace_prepared=True)."""
    r = (_marshal or marshal()).quantize_act(X, workspace)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_quantize_act")
        return r
    X = _dev(X, torch.bfloat16, "X")
    M, K = X.shape
    A = torch.empty((M, K), dtype=torch.uint8, device=X.device)
    s = torch.empty((M,), dtype=torch.float32, device=X.device)
    if workspace is None:
        rc = lib().fq_quantize_act(X.data_ptr(), A.data_ptr(), s.data_ptr(), M, K, _stream())
    else:
        rc = lib().fq_quantize_act_ws(X.data_ptr(), A.data_ptr(), s.data_ptr(), M, K, workspace.data_ptr(),
                                      workspace.numel() * workspace.element_size(), _stream())
    if rc != 0:
        raise FireqError(rc, "fq_quantize_act")
    return A, s


def fq_w4a8_gemm(A: torch.Tensor, a_scale: torch.Tensor, Wq_packed: torch.Tensor,
                 w_gscale: torch.Tensor, w_tscale: float, N: int,
                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 workspace_prepared: bool = False) -> torch.Tensor:
    """Y[M,N] (bf16) = W4A8-FP GEMM of E4M3 activations and packed INT4 weights.

    Calls fq_w4a8_gemm_ws; `workspace` (a device tensor of at least
    fq_w4a8_gemm_workspace_bytes(M, N, K) bytes) is allocated here when not given;
    `workspace_prepared` says that fq_quantize_act(X, workspace) has filled it for this A."""
    r = (_marshal or marshal()).gemm(A, a_scale, Wq_packed, w_gscale, w_tscale, N, out, workspace, workspace_prepared)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_w4a8_gemm_ws")
        return r
    A = _dev(A, torch.uint8, "A")
    a_scale = _dev(a_scale, torch.float32, "a_scale")
    Wq_packed = _dev(Wq_packed, torch.uint8, "Wq_packed")
    w_gscale = _dev(w_gscale, torch.uint8, "w_gscale")
    M, K = A.shape
    if a_scale.numel() != M or K % GROUP or w_gscale.numel() != N * (K // GROUP) \
            or Wq_packed.numel() < fq_packed_weight_bytes(N, K):
        raise FireqError(-2, "fq_w4a8_gemm")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    else:
        out = _dev(out, torch.bfloat16, "out")
        if tuple(out.shape) != (M, N):
            raise FireqError(-2, "fq_w4a8_gemm")
    # the workspace comes from torch's caching allocator (stream-ordered, no hipMalloc per call)
    need = lib().fq_w4a8_gemm_workspace_bytes(M, N, K)
    if workspace is None and need > 0:
        workspace = torch.empty((need,), dtype=torch.uint8, device=A.device)
    ws_ptr, ws_bytes = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (0, 0)
    rc = lib().fq_w4a8_gemm_ws(A.data_ptr(), a_scale.data_ptr(), Wq_packed.data_ptr(),
                               w_gscale.data_ptr(), ctypes.c_float(float(w_tscale)), out.data_ptr(),
                               M, N, K, ws_ptr, ws_bytes, 1 if (workspace_prepared and workspace is not None) else 0,
                               _stream())
    if rc != 0:
        raise FireqError(rc, "fq_w4a8_gemm_ws")
    return out


def fq_w4a8_gemm_swiglu(A: torch.Tensor, a_scale: torch.Tensor, Wq_packed: torch.Tensor,
                        w_gscale: torch.Tensor, w_tscale: float, N: int,
                        out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        workspace_prepared: bool = False) -> torch.Tensor:
    """H[M,N/2] (bf16) = SiLU(gate) * up of the W4A8-FP GEMM whose N weight rows interleave gate (even)
    and up (odd) channels.  Calls fq_w4a8_gemm_swiglu_ws; workspace handling as in fq_w4a8_gemm."""
    r = (_marshal or marshal()).gemm_swiglu(A, a_scale, Wq_packed, w_gscale, w_tscale, N, out, workspace, workspace_prepared)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_w4a8_gemm_swiglu_ws")
        return r
    A = _dev(A, torch.uint8, "A")
    a_scale = _dev(a_scale, torch.float32, "a_scale")
    Wq_packed = _dev(Wq_packed, torch.uint8, "Wq_packed")
    w_gscale = _dev(w_gscale, torch.uint8, "w_gscale")
    M, K = A.shape
    if N % 2 or a_scale.numel() != M or K % GROUP or w_gscale.numel() != N * (K // GROUP) \
            or Wq_packed.numel() < fq_packed_weight_bytes(N, K):
        raise FireqError(-2, "fq_w4a8_gemm_swiglu")
    if out is None:
        out = torch.empty((M, N // 2), dtype=torch.bfloat16, device=A.device)
    else:
        out = _dev(out, torch.bfloat16, "out")
        if tuple(out.shape) != (M, N // 2):
            raise FireqError(-2, "fq_w4a8_gemm_swiglu")
    need = lib().fq_w4a8_gemm_workspace_bytes(M, N, K)
    if workspace is None and need > 0:
        workspace = torch.empty((need,), dtype=torch.uint8, device=A.device)
    ws_ptr, ws_bytes = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (0, 0)
    rc = lib().fq_w4a8_gemm_swiglu_ws(A.data_ptr(), a_scale.data_ptr(), Wq_packed.data_ptr(),
                                      w_gscale.data_ptr(), ctypes.c_float(float(w_tscale)), out.data_ptr(),
                                      M, N, K, ws_ptr, ws_bytes,
                                      1 if (workspace_prepared and workspace is not None) else 0, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_w4a8_gemm_swiglu_ws")
    return out


def fq_w4a8_gemm_swiglu_quant(A: torch.Tensor, a_scale: torch.Tensor, Wq_packed: torch.Tensor,
                              w_gscale: torch.Tensor, w_tscale: float, N: int,
                              out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                              workspace_prepared: bool = False, next_workspace: Optional[torch.Tensor] = None
                              ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(H bf16 [M,N/2], H as E4M3 codes [M,N/2], float32 [M] scales): fq_w4a8_gemm_swiglu whose output also leaves
    quantised for the next layer, as fq_quantize_act would give it.  Calls fq_w4a8_gemm_swiglu_quant_ws;
    `next_workspace` (fq_w4a8_gemm_workspace_bytes(M, N', N/2) bytes or more) is prepared for a GEMM on the codes."""
    r = (_marshal or marshal()).gemm_swiglu_quant(A, a_scale, Wq_packed, w_gscale, w_tscale, N, out, workspace, workspace_prepared,
                                                  next_workspace)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_w4a8_gemm_swiglu_quant_ws")
        return r
    A = _dev(A, torch.uint8, "A")
    a_scale = _dev(a_scale, torch.float32, "a_scale")
    Wq_packed = _dev(Wq_packed, torch.uint8, "Wq_packed")
    w_gscale = _dev(w_gscale, torch.uint8, "w_gscale")
    M, K = A.shape
    if N % 2 or a_scale.numel() != M or K % GROUP or w_gscale.numel() != N * (K // GROUP) \
            or Wq_packed.numel() < fq_packed_weight_bytes(N, K):
        raise FireqError(-2, "fq_w4a8_gemm_swiglu_quant")
    if out is None:
        out = torch.empty((M, N // 2), dtype=torch.bfloat16, device=A.device)
    else:
        out = _dev(out, torch.bfloat16, "out")
        if tuple(out.shape) != (M, N // 2):
            raise FireqError(-2, "fq_w4a8_gemm_swiglu_quant")
    codes = torch.empty((M, N // 2), dtype=torch.uint8, device=A.device)
    scales = torch.empty((M,), dtype=torch.float32, device=A.device)
    need = lib().fq_w4a8_gemm_workspace_bytes(M, N, K)
    if workspace is None and need > 0:
        workspace = torch.empty((need,), dtype=torch.uint8, device=A.device)
    ws_ptr, ws_bytes = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (0, 0)
    nws_ptr, nws_bytes = (next_workspace.data_ptr(), next_workspace.numel() * next_workspace.element_size()) \
        if next_workspace is not None else (0, 0)
    rc = lib().fq_w4a8_gemm_swiglu_quant_ws(A.data_ptr(), a_scale.data_ptr(), Wq_packed.data_ptr(),
                                            w_gscale.data_ptr(), ctypes.c_float(float(w_tscale)), out.data_ptr(),
                                            codes.data_ptr(), scales.data_ptr(), M, N, K, ws_ptr, ws_bytes,
                                            1 if (workspace_prepared and workspace is not None) else 0,
                                            nws_ptr, nws_bytes, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_w4a8_gemm_swiglu_quant_ws")
    return out, codes, scales


def fq_w4a8_gemm_add(A: torch.Tensor, a_scale: torch.Tensor, Wq_packed: torch.Tensor,
                     w_gscale: torch.Tensor, w_tscale: float, N: int, residual: torch.Tensor,
                     out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     workspace_prepared: bool = False) -> torch.Tensor:
    """Y[M,N] (bf16) = GEMM + residual, rounded once.  Calls fq_w4a8_gemm_add_ws; `out` may be
    `residual` itself (in-place update); workspace handling as in fq_w4a8_gemm."""
    r = (_marshal or marshal()).gemm_add(A, a_scale, Wq_packed, w_gscale, w_tscale, N, out, workspace, workspace_prepared, residual)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_w4a8_gemm_add_ws")
        return r
    A = _dev(A, torch.uint8, "A")
    a_scale = _dev(a_scale, torch.float32, "a_scale")
    Wq_packed = _dev(Wq_packed, torch.uint8, "Wq_packed")
    w_gscale = _dev(w_gscale, torch.uint8, "w_gscale")
    residual = _dev(residual, torch.bfloat16, "residual")
    M, K = A.shape
    if a_scale.numel() != M or K % GROUP or w_gscale.numel() != N * (K // GROUP) \
            or Wq_packed.numel() < fq_packed_weight_bytes(N, K) or tuple(residual.shape) != (M, N):
        raise FireqError(-2, "fq_w4a8_gemm_add")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    else:
        out = _dev(out, torch.bfloat16, "out")
        if tuple(out.shape) != (M, N):
            raise FireqError(-2, "fq_w4a8_gemm_add")
    need = lib().fq_w4a8_gemm_workspace_bytes(M, N, K)
    if workspace is None and need > 0:
        workspace = torch.empty((need,), dtype=torch.uint8, device=A.device)
    ws_ptr, ws_bytes = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (0, 0)
    rc = lib().fq_w4a8_gemm_add_ws(A.data_ptr(), a_scale.data_ptr(), Wq_packed.data_ptr(),
                                   w_gscale.data_ptr(), ctypes.c_float(float(w_tscale)), residual.data_ptr(),
                                   out.data_ptr(), M, N, K, ws_ptr, ws_bytes,
                                   1 if (workspace_prepared and workspace is not None) else 0, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_w4a8_gemm_add_ws")
    return out


def fq_w4a8_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().fq_w4a8_linear_workspace_bytes(M, N, K))


def fq_w4a8_linear(X: torch.Tensor, Wq_packed: torch.Tensor, w_gscale: torch.Tensor, w_tscale: float, N: int,
                   out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y[M,N] (bf16) of a whole linear layer from bf16 activations X[M,K] (quantiser + GEMM; one kernel
    for a few rows).  Calls fq_w4a8_linear_ws; the workspace is allocated here when not given."""
    r = (_marshal or marshal()).linear(X, Wq_packed, w_gscale, w_tscale, N, out, workspace)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_w4a8_linear_ws")
        return r
    X = _dev(X, torch.bfloat16, "X")
    Wq_packed = _dev(Wq_packed, torch.uint8, "Wq_packed")
    w_gscale = _dev(w_gscale, torch.uint8, "w_gscale")
    M, K = X.shape
    if K % GROUP or w_gscale.numel() != N * (K // GROUP) or Wq_packed.numel() < fq_packed_weight_bytes(N, K):
        raise FireqError(-2, "fq_w4a8_linear")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=X.device)
    else:
        out = _dev(out, torch.bfloat16, "out")
        if tuple(out.shape) != (M, N):
            raise FireqError(-2, "fq_w4a8_linear")
    need = fq_w4a8_linear_workspace_bytes(M, N, K)
    if workspace is None and need > 0:
        workspace = torch.empty((need,), dtype=torch.uint8, device=X.device)
    ws_ptr, ws_bytes = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (0, 0)
    rc = lib().fq_w4a8_linear_ws(X.data_ptr(), Wq_packed.data_ptr(), w_gscale.data_ptr(), ctypes.c_float(float(w_tscale)),
                                 out.data_ptr(), M, N, K, ws_ptr, ws_bytes, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_w4a8_linear_ws")
    return out


def fq_w4a8_gemm_workspace_bytes(M: int, N: int, K: int) -> int:
    r = (_marshal or marshal()).gemm_workspace_bytes(M, N, K)
    return int(lib().fq_w4a8_gemm_workspace_bytes(M, N, K)) if r is None else r


def fq_w4a8_gemm_plan(M: int, N: int, K: int, cus: int = 0) -> dict:
    """How the GEMM entry points would run this shape (see fireq.h); cus = 0 asks the current device."""
    buf = (ctypes.c_int * 8)()
    rc = lib().fq_w4a8_gemm_plan(int(M), int(N), int(K), int(cus), buf)
    if rc != 0:
        raise FireqError(rc, "fq_w4a8_gemm_plan")
    return {"kernel": ("simple", "small16", "smallm", "large", "ksplit256x128", "ksplit128x64", "ksplit64x64",
                       "ksplit128x128")[buf[0]], "whole": buf[1],
            "whole_ragged": buf[2], "half": buf[3], "half_ragged": buf[4], "ksplit_tiles": buf[5], "ksplit_slices": buf[6]}


def fq_test_force_kernel(name: Optional[str]) -> None:
    """Cross-check hook: "simple" | "small" | "large" | "ksplit" forces that GEMM kernel, None or "auto" restores the choice by M."""
    lib().fq_test_force_kernel((name or "").encode() if name != "auto" else b"")


def fq_diag_stream_read(src: torch.Tensor, sink: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Measurement aid: enqueue a kernel that only reads `src` (its bytes must be a multiple of 16)."""
    nbytes = src.numel() * src.element_size()
    if sink is None:
        sink = torch.empty((lib().fq_diag_stream_read_sink_bytes(),), dtype=torch.uint8, device=src.device)
    rc = lib().fq_diag_stream_read(src.data_ptr(), nbytes, sink.data_ptr(), _stream())
    if rc != 0:
        raise FireqError(rc, "fq_diag_stream_read")
    return sink


def fq_w4a8_gemm_lut(A: torch.Tensor, a_scale: torch.Tensor, Wq_packed: torch.Tensor, w_gscale: torch.Tensor,
                     w_tscale: float, N: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y[M,N] (bf16) of the GEMM in the paper's table mode (weights rounded to E4M3(q * sigma)); calls fq_w4a8_gemm_lut."""
    A = _dev(A, torch.uint8, "A")
    a_scale = _dev(a_scale, torch.float32, "a_scale")
    Wq_packed = _dev(Wq_packed, torch.uint8, "Wq_packed")
    w_gscale = _dev(w_gscale, torch.uint8, "w_gscale")
    M, K = A.shape
    if a_scale.numel() != M or K % GROUP or w_gscale.numel() != N * (K // GROUP) \
            or Wq_packed.numel() < fq_packed_weight_bytes(N, K):
        raise FireqError(-2, "fq_w4a8_gemm_lut")
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    else:
        out = _dev(out, torch.bfloat16, "out")
        if tuple(out.shape) != (M, N):
            raise FireqError(-2, "fq_w4a8_gemm_lut")
    rc = lib().fq_w4a8_gemm_lut(A.data_ptr(), a_scale.data_ptr(), Wq_packed.data_ptr(), w_gscale.data_ptr(),
                                ctypes.c_float(float(w_tscale)), out.data_ptr(), M, N, K, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_w4a8_gemm_lut")
    return out


def fq_kv4_pack(codes: torch.Tensor, values: bool) -> torch.Tensor:
    """int8 [H,T,128] INT4 codes of a key (values=False) or value (values=True) cache -> the packed cache."""
    r = (_marshal or marshal()).kv4_pack(codes, values)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_kv4_pack")
        return r
    codes = _dev(codes, torch.int8, "codes")
    H, T, D = codes.shape
    if D != GROUP:
        raise FireqError(-2, "fq_kv4_pack")
    out = torch.empty((lib().fq_kv4_packed_bytes(H, T, 1 if values else 0),), dtype=torch.uint8, device=codes.device)
    rc = lib().fq_kv4_pack(codes.data_ptr(), out.data_ptr(), H, T, 1 if values else 0, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_kv4_pack")
    return out


def fq_kv4_unpack(packed: torch.Tensor, H: int, T: int, values: bool) -> torch.Tensor:
    packed = _dev(packed, torch.uint8, "packed")
    if packed.numel() < lib().fq_kv4_packed_bytes(H, T, 1 if values else 0):
        raise FireqError(-2, "fq_kv4_unpack")
    out = torch.empty((H, T, GROUP), dtype=torch.int8, device=packed.device)
    rc = lib().fq_kv4_unpack(packed.data_ptr(), out.data_ptr(), H, T, 1 if values else 0, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_kv4_unpack")
    return out


def fq_kv4_scores(Q: torch.Tensor, q_scale: torch.Tensor, K_packed: torch.Tensor, k_scale: torch.Tensor,
                  out_scale: float) -> torch.Tensor:
    """S[H,R,T] (bf16): FP8 queries [H,R,128] against a packed INT4 key cache with E4M3 scales [H,T]."""
    r = (_marshal or marshal()).kv4_scores(Q, q_scale, K_packed, k_scale, out_scale)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_kv4_scores")
        return r
    Q = _dev(Q, torch.uint8, "Q"); q_scale = _dev(q_scale, torch.float32, "q_scale")
    K_packed = _dev(K_packed, torch.uint8, "K_packed"); k_scale = _dev(k_scale, torch.uint8, "k_scale")
    H, R, D = Q.shape
    T = k_scale.shape[1]
    if D != GROUP or tuple(q_scale.shape) != (H, R) or k_scale.shape[0] != H \
            or K_packed.numel() < lib().fq_kv4_packed_bytes(H, T, 0):
        raise FireqError(-2, "fq_kv4_scores")
    S = torch.empty((H, R, T), dtype=torch.bfloat16, device=Q.device)
    rc = lib().fq_kv4_scores(Q.data_ptr(), q_scale.data_ptr(), K_packed.data_ptr(), k_scale.data_ptr(),
                             ctypes.c_float(float(out_scale)), S.data_ptr(), H, R, T, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_kv4_scores")
    return S


def fq_kv4_output(P: torch.Tensor, p_scale: torch.Tensor, V_packed: torch.Tensor, v_scale: torch.Tensor) -> torch.Tensor:
    """O[H,R,128] (bf16): FP8 probabilities [H,R,T] against a packed INT4 value cache with E4M3 scales [H,T]."""
    r = (_marshal or marshal()).kv4_output(P, p_scale, V_packed, v_scale)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_kv4_output")
        return r
    P = _dev(P, torch.uint8, "P"); p_scale = _dev(p_scale, torch.float32, "p_scale")
    V_packed = _dev(V_packed, torch.uint8, "V_packed"); v_scale = _dev(v_scale, torch.uint8, "v_scale")
    H, R, ldp = P.shape
    T = v_scale.shape[1]
    if tuple(p_scale.shape) != (H, R) or v_scale.shape[0] != H or ldp < T \
            or V_packed.numel() < lib().fq_kv4_packed_bytes(H, T, 1):
        raise FireqError(-2, "fq_kv4_output")
    O = torch.empty((H, R, GROUP), dtype=torch.bfloat16, device=P.device)
    # scratch from torch's caching allocator (stream-ordered), where the tokens are cut into slices
    need = lib().fq_kv4_output_workspace_bytes(H, R, T)
    ws = torch.empty((need,), dtype=torch.uint8, device=P.device) if need else None
    rc = lib().fq_kv4_output_ws(P.data_ptr(), p_scale.data_ptr(), V_packed.data_ptr(), v_scale.data_ptr(), O.data_ptr(),
                                H, R, T, ldp, ws.data_ptr() if need else 0, need, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_kv4_output")
    return O


def _fits(*sizes):
    """Whether C ints hold them (ctypes would pass the low bits on)."""
    return all(-(1 << 31) <= n < 1 << 31 for n in sizes)


def _norm_arguments(X, weight, residual, out):
    X = _dev(X, torch.bfloat16, "X")
    weight = _dev(weight, torch.bfloat16, "weight")
    if X.dim() != 2 or weight.numel() != X.shape[1]:
        raise FireqError(-2, "fq_rmsnorm")
    if not _fits(*X.shape):
        raise FireqError(-2, "fq_rmsnorm")
    if residual is None:
        if out is not None:
            raise FireqError(-2, "fq_rmsnorm")
        return X, weight, None, None
    residual = _dev(residual, torch.bfloat16, "residual")
    out = torch.empty_like(X) if out is None else _dev(out, torch.bfloat16, "out")
    if residual.shape != X.shape or out.shape != X.shape:
        raise FireqError(-2, "fq_rmsnorm")
    return X, weight, residual, out


def _scratch(t):
    """(pointer, bytes) of a caller's workspace, or of none"""
    if t is None:
        return 0, 0
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("workspace must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return t.data_ptr(), t.numel() * t.element_size()


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def fq_rmsnorm(X: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None):
    """bf16 [M,K] RMS norm of X, or of H = bf16(X + residual): (Y, H) then.  `out` receives H and may be the residual itself
    (the residual stream updated in place)."""
    r = (_marshal or marshal()).rmsnorm(X, weight, eps, residual, out)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_rmsnorm")
        return r
    X, weight, residual, H = _norm_arguments(X, weight, residual, out)
    M, K = X.shape
    Y = torch.empty_like(X)
    rc = lib().fq_rmsnorm(X.data_ptr(), _ptr(residual), weight.data_ptr(), ctypes.c_float(float(eps)), _ptr(H), Y.data_ptr(), M, K, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_rmsnorm")
    return Y if H is None else (Y, H)


def fq_rmsnorm_quant(X: torch.Tensor, weight: torch.Tensor, eps: float, residual: Optional[torch.Tensor] = None,
                     out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
    """(uint8 [M,K] E4M3 codes, float32 [M] row scales) of the RMS norm of X [M,K], the operands of fq_w4a8_gemm; with a
    residual (codes, scales, H = bf16(X + residual)).  `out` receives H and may be the residual itself; `workspace`
    (fq_w4a8_gemm_workspace_bytes(M, N, K) bytes or more) is prepared for fq_w4a8_gemm(..., workspace_prepared=True)."""
    r = (_marshal or marshal()).rmsnorm_quant(X, weight, eps, residual, out, workspace)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_rmsnorm_quant")
        return r
    X, weight, residual, H = _norm_arguments(X, weight, residual, out)
    M, K = X.shape
    A = torch.empty((M, K), dtype=torch.uint8, device=X.device)
    s = torch.empty((M,), dtype=torch.float32, device=X.device)
    ws, nbytes = _scratch(workspace)
    rc = lib().fq_rmsnorm_quant_ws(X.data_ptr(), _ptr(residual), weight.data_ptr(), ctypes.c_float(float(eps)), _ptr(H), A.data_ptr(),
                                   s.data_ptr(), M, K, ws, nbytes, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_rmsnorm_quant")
    return (A, s) if H is None else (A, s, H)


KV4_TILE_TOKENS, KV4_TILE_BYTES = 16, 2080


def fq_kv4_cache(pages: int, heads: int, page: int, device=None) -> torch.Tensor:
    """uint8 [pages, heads, page / 16, 2080]: an empty paged INT4 key/value cache (one layer's) for tokens of `heads` key/value
    heads, `page` (a multiple of 16) to a page.  A slice of a larger tensor of that form serves too, as long as its last two
    dimensions are contiguous."""
    if page <= 0 or page % KV4_TILE_TOKENS:
        raise FireqError(-2, "fq_kv4_cache")
    return torch.zeros((pages, heads, page // KV4_TILE_TOKENS, KV4_TILE_BYTES), dtype=torch.uint8,
                       device=torch.device("cuda", torch.cuda.current_device()) if device is None else device)


def _cache(cache):
    """(pointer, page stride, head stride, pages, tokens of a page), heads"""
    if not isinstance(cache, torch.Tensor) or not cache.is_cuda:
        raise TypeError("cache must be a GPU tensor")
    if cache.dtype != torch.uint8:
        raise TypeError("cache must have dtype %s, got %s" % (torch.uint8, cache.dtype))
    if cache.dim() != 4 or cache.shape[3] != KV4_TILE_BYTES or cache.shape[2] == 0:
        raise FireqError(-2, "cache")
    if cache.stride(3) != 1 or (cache.shape[2] > 1 and cache.stride(2) != KV4_TILE_BYTES):
        raise ValueError("cache must have its pages contiguous")
    pages, heads, tiles, _ = cache.shape
    if not _fits(pages, heads, tiles * KV4_TILE_TOKENS):
        raise FireqError(-2, "cache")
    per = tiles * KV4_TILE_BYTES
    head_stride = cache.stride(1) if heads > 1 else per
    page_stride = cache.stride(0) if pages > 1 else heads * head_stride
    return (cache.data_ptr(), page_stride, head_stride, pages, tiles * KV4_TILE_TOKENS), heads


def fq_kv4_append(QKV: torch.Tensor, cos_sin: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor, cache: torch.Tensor,
                  interleaved: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """(uint8 [T,Hq,128] E4M3 codes, float32 [T,Hq] scales) of the rotated queries of the fused projections' output QKV
    bf16 [T, (Hq + 2 Hkv) * 128] (rows may be strided); rotated keys and values go to `slots` (int64 [T], negative: padding) of
    the paged cache as INT4.  cos_sin: float32 [positions, 64, 2]; positions: int32 [T]."""
    r = (_marshal or marshal()).kv4_append(QKV, cos_sin, positions, slots, cache, interleaved)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_kv4_append")
        return r
    if not isinstance(QKV, torch.Tensor) or not QKV.is_cuda:
        raise TypeError("QKV must be a GPU tensor")
    if QKV.dtype != torch.bfloat16:
        raise TypeError("QKV must have dtype %s, got %s" % (torch.bfloat16, QKV.dtype))
    cos_sin = _dev(cos_sin, torch.float32, "cos_sin")
    positions = _dev(positions, torch.int32, "positions")
    slots = _dev(slots, torch.int64, "slots")
    geometry, Hkv = _cache(cache)
    if QKV.dim() != 2:
        raise FireqError(-2, "fq_kv4_append")
    T, width = QKV.shape
    if (width > 1 and QKV.stride(1) != 1) or (T > 1 and QKV.stride(0) < width):
        raise ValueError("QKV must have contiguous rows")
    if width % 128 or cos_sin.dim() != 3 or tuple(cos_sin.shape[1:]) != (64, 2):
        raise FireqError(-2, "fq_kv4_append")
    Hq = width // 128 - 2 * Hkv
    if Hq <= 0 or positions.numel() != T or slots.numel() != T:
        raise FireqError(-2, "fq_kv4_append")
    if not _fits(T, Hq, cos_sin.shape[0]):
        raise FireqError(-2, "fq_kv4_append")
    Q = torch.empty((T, Hq, 128), dtype=torch.uint8, device=QKV.device)
    s = torch.empty((T, Hq), dtype=torch.float32, device=QKV.device)
    rc = lib().fq_kv4_append(QKV.data_ptr(), QKV.stride(0) if T > 1 else width, cos_sin.data_ptr(), cos_sin.shape[0], positions.data_ptr(),
                             slots.data_ptr(), 1 if interleaved else 0, Q.data_ptr(), s.data_ptr(), *geometry, T, Hq, Hkv, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_kv4_append")
    return Q, s


def fq_kv4_read(cache: torch.Tensor, slots: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """(K, V) bf16 [n,Hkv,128]: the cached tokens in `slots` (int64 [n]; zeros for a negative slot)."""
    r = (_marshal or marshal()).kv4_read(cache, slots)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, "fq_kv4_read")
        return r
    geometry, Hkv = _cache(cache)
    slots = _dev(slots, torch.int64, "slots")
    n = slots.numel()
    if not _fits(n):
        raise FireqError(-2, "fq_kv4_read")
    K = torch.empty((n, Hkv, 128), dtype=torch.bfloat16, device=cache.device)
    V = torch.empty((n, Hkv, 128), dtype=torch.bfloat16, device=cache.device)
    rc = lib().fq_kv4_read(*geometry, slots.data_ptr(), K.data_ptr(), V.data_ptr(), n, Hkv, _stream())
    if rc != 0:
        raise FireqError(rc, "fq_kv4_read")
    return K, V


def fq_kv4_attention_workspace_bytes(B: int, Hq: int, Hkv: int, max_len: int, prefix_len: int = 0) -> int:
    """Bytes of scratch that the attention of these sizes needs; 0 for sizes that it refuses, as the C function answers."""
    sizes = [int(n) for n in (B, Hq, Hkv, max_len, prefix_len)]
    return int(lib().fq_kv4_attention_workspace_bytes(*sizes)) if _fits(*sizes) else 0


def _attention(where, Q, q_scale, cache, prefix_pages, prefix_len, block_table, seq_lens, out_scale, max_len, out, workspace):
    r = (_marshal or marshal()).kv4_attention(Q, q_scale, cache, prefix_pages, prefix_len, block_table, seq_lens, out_scale, max_len, out, workspace)
    if r is not None:
        if type(r) is int:
            raise FireqError(r, where)
        return r
    Q = _dev(Q, torch.uint8, "Q")
    q_scale = _dev(q_scale, torch.float32, "q_scale")
    geometry, Hkv = _cache(cache)
    block_table = _dev(block_table, torch.int32, "block_table")
    seq_lens = _dev(seq_lens, torch.int32, "seq_lens")
    if Q.dim() != 3 or Q.shape[2] != 128 or block_table.dim() != 2:
        raise FireqError(-2, where)
    B, Hq, _ = Q.shape
    width = block_table.shape[1]
    if q_scale.numel() != B * Hq or block_table.shape[0] != B or seq_lens.numel() != B or Hq % Hkv:
        raise FireqError(-2, where)
    if not _fits(B, Hq, width):
        raise FireqError(-2, where)
    max_len = min(width * geometry[4], 1 << 30) if max_len is None else int(max_len)
    shared = 0
    if prefix_pages is not None:
        prefix_pages = _dev(prefix_pages, torch.int32, "prefix_pages")
        prefix_len = int(prefix_len)
        if prefix_len < 0 or prefix_len > 1 << 30 or prefix_pages.numel() * geometry[4] < prefix_len:
            raise FireqError(-2, where)
        shared = prefix_pages.data_ptr()
    if max_len < 0 or max_len > 1 << 30:                  # (a C int would take its low bits)
        raise FireqError(-2, where)
    if out is None:
        out = torch.empty((B, Hq, 128), dtype=torch.bfloat16, device=Q.device)
    else:
        out = _dev(out, torch.bfloat16, "out")
        if tuple(out.shape) not in ((B, Hq, 128), (B, Hq * 128)):
            raise FireqError(-2, where)
    if workspace is None:
        need = fq_kv4_attention_workspace_bytes(B, Hq, Hkv, max_len, prefix_len)
        workspace = torch.empty((need,), dtype=torch.uint8, device=Q.device) if need else None
    ws, nbytes = _scratch(workspace)
    args = (block_table.data_ptr(), width, seq_lens.data_ptr(), ctypes.c_float(float(out_scale)), out.data_ptr(), B, Hq, Hkv, max_len, ws, nbytes,
            _stream())
    if prefix_pages is None:
        rc = lib().fq_kv4_attention_ws(Q.data_ptr(), q_scale.data_ptr(), *geometry, *args)
    else:
        rc = lib().fq_kv4_attention_prefix_ws(Q.data_ptr(), q_scale.data_ptr(), *geometry, shared, prefix_len, *args)
    if rc != 0:
        raise FireqError(rc, where)
    return out


def fq_kv4_attention(Q: torch.Tensor, q_scale: torch.Tensor, cache: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor,
                     out_scale: float, max_len: Optional[int] = None, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """bf16 [B,Hq,128]: attention of one query token per sequence (codes and scales from fq_kv4_append) over its seq_lens[b]
    (int32 [B]) cached tokens, in the pages block_table[b] (int32 [B, pages of a sequence]) of a paged cache.

    `max_len`: an upper bound of seq_lens that the host knows, by default what the table has room for (it decides how the work is
    split: one far above the lengths costs up to several times the time); `workspace` of fq_kv4_attention_workspace_bytes(B, Hq, Hkv, max_len) bytes is allocated here when not given."""
    return _attention("fq_kv4_attention", Q, q_scale, cache, None, 0, block_table, seq_lens, out_scale, max_len, out, workspace)


def fq_kv4_attention_prefix(Q: torch.Tensor, q_scale: torch.Tensor, cache: torch.Tensor, prefix_pages: torch.Tensor, prefix_len: int,
                            block_table: torch.Tensor, seq_lens: torch.Tensor, out_scale: float, max_len: Optional[int] = None,
                            out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """fq_kv4_attention for sequences that share a prefix: each attends to prefix_len tokens in prefix_pages (int32 [pages]) and
    then to its own seq_lens[b] tokens in block_table[b].  The prefix is worked on for many sequences at a time."""
    if prefix_pages is None:
        raise TypeError("prefix_pages must be a GPU tensor")
    return _attention("fq_kv4_attention_prefix", Q, q_scale, cache, prefix_pages, prefix_len, block_table, seq_lens, out_scale, max_len, out,
                      workspace)
