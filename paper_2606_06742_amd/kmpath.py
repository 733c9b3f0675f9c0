"""ctypes binding of libkmpath.so: the same entry points as include/kmpath.h.

Argument marshalling only. Device arrays are torch tensors on the HIP device
(``torch.device("cuda")`` on ROCm); every computation runs in the library.
Loading fails loudly when the built library is missing: there is no
fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import numpy as np

# KMPATH_LIB points the binding at another build of the library (the
# host-sanitized build of the CPU tests); default: the in-tree libkmpath.so
LIB_PATH = os.environ.get("KMPATH_LIB") or os.path.join(
    os.path.dirname(os.path.abspath(__file__)), "libkmpath.so")

KMP_OK, KMP_WMAXITER = 0, 1
KMP_EINVAL, KMP_EFOLD, KMP_EWORKSPACE, KMP_EHIP, KMP_ENONFINITE = -1, -2, -3, -4, -5
KMP_HINGE, KMP_LOGISTIC, KMP_CHECK = 0, 1, 2
KMP_FLAG_RESTART = 1
KMP_FLAG_GLOBAL_SOLVE = 2
KMP_FLAG_REFIT = 4
KMP_FLAG_SHARED_FACTOR = 8
KMP_FLAG_EXACT_HINGE = 16
KMP_FLAG_EAGER = 32
KMP_WNOTEXACT = 2
KMP_F64, KMP_F32, KMP_BF16, KMP_F16, KMP_I8 = 0, 1, 2, 3, 4
KMP_MAX_TOP = 64
KMP_NORM_RMS, KMP_NORM_AFTER = 1, 2
KMP_NKC = 10
KERNEL_CLASSES = ("gram", "panel", "panel_wy", "trail_update", "q_form", "precompute", "gemm_f",
                  "gemm_zhat", "update", "finalize")
ACT_CODES = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
LOSS_CODES = {"hinge": KMP_HINGE, "logistic": KMP_LOGISTIC, "check": KMP_CHECK}


class kmp_path_spec(C.Structure):
    _fields_ = [("loss", C.c_int32), ("delta0", C.c_double), ("eta", C.c_double),
                ("n_stages", C.c_int32), ("tol", C.c_double), ("max_iter", C.c_int32),
                ("poll_every", C.c_int32), ("flags", C.c_int32), ("timing_mask", C.c_int32),
                ("timing_every", C.c_int32)]


class kmp_timings(C.Structure):
    _fields_ = [("gram_ms", C.c_double), ("factor_ms", C.c_double),
                ("precompute_ms", C.c_double), ("path_ms", C.c_double),
                ("finalize_ms", C.c_double), ("total_ms", C.c_double),
                ("iterations", C.c_int64), ("cell_iterations", C.c_int64),
                ("kernel_ms", C.c_double * KMP_NKC), ("kernel_launches", C.c_int64 * KMP_NKC),
                ("kernel_seen", C.c_int64 * KMP_NKC),
                ("kernel_bytes", C.c_double * KMP_NKC), ("kernel_flops", C.c_double * KMP_NKC),
                ("kernel_ms_mb", C.c_double * KMP_NKC), ("kernel_launches_mb", C.c_int64 * KMP_NKC),
                ("kernel_bytes_mb", C.c_double * KMP_NKC), ("kernel_flops_mb", C.c_double * KMP_NKC)]

    def as_dict(self):
        return {k: (list(getattr(self, k)) if k.startswith("kernel_") else getattr(self, k))
                for k, _ in self._fields_}

    def kernels(self):
        """{class: (ms, bracketed launches, all launches, bytes, flops, and
        ms, launches, bytes, flops of the bracketed launches above the ridge
        point)} of the timed classes; ms, bytes and flops cover the bracketed
        launches."""
        return {KERNEL_CLASSES[i]: (self.kernel_ms[i], int(self.kernel_launches[i]),
                                    int(self.kernel_seen[i]), self.kernel_bytes[i],
                                    self.kernel_flops[i], self.kernel_ms_mb[i],
                                    int(self.kernel_launches_mb[i]), self.kernel_bytes_mb[i],
                                    self.kernel_flops_mb[i])
                for i in range(KMP_NKC) if self.kernel_launches[i] > 0}


class KmpError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"kmpath error {code}: {msg}")
        self.code = code


_lib = None
_VP, _DP, _IP = C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int32)


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2606_06742_amd.build`")
        L = C.CDLL(LIB_PATH)
        L.kmp_default_spec.argtypes = [C.POINTER(kmp_path_spec)]
        L.kmp_default_spec.restype = None
        L.kmp_workspace_bytes.argtypes = [C.POINTER(kmp_path_spec), C.c_int64, C.c_int64, C.c_int32,
                                          _IP, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
        L.kmp_workspace_bytes.restype = C.c_size_t
        L.kmp_fit_path.argtypes = [_VP, C.POINTER(kmp_path_spec), _VP, C.c_int64, C.c_int64,
                                   C.c_int64, _VP, _DP, C.c_int32, _DP, C.c_int32, _DP, C.c_int32,
                                   _IP, C.c_int32, _VP, C.c_size_t, _VP, _VP, _VP, _VP, _VP, _VP,
                                   _VP, _IP, _IP, C.POINTER(kmp_timings)]
        L.kmp_fit_path.restype = C.c_int
        L.kmp_make_folds.argtypes = [C.c_int64, C.c_int32, C.c_uint64, _IP]
        L.kmp_make_folds.restype = C.c_int
        L.kmp_rbf_gram.argtypes = [_VP, _VP, C.c_int64, C.c_int64, C.c_int64, _VP, C.c_int64, _VP,
                                   C.c_int64, _DP, C.c_int32, _VP, C.c_int64]
        L.kmp_rbf_gram.restype = C.c_int
        L.kmp_rbf_gram_noalloc.argtypes = L.kmp_rbf_gram.argtypes
        L.kmp_rbf_gram_noalloc.restype = C.c_int
        L.kmp_tridiag.argtypes = [_VP, _VP, C.c_int32, C.c_int32, _VP, _VP, _VP]
        L.kmp_tridiag.restype = C.c_int
        L.kmp_band_reduce.argtypes = [_VP, _VP, C.c_int32, C.c_int32, _VP, _VP]
        L.kmp_band_reduce.restype = C.c_int
        L.kmp_path_step.argtypes = [_VP, C.c_int32, C.c_double, _VP, C.c_int64, _VP, _DP, _DP,
                                    C.c_int32, _VP, _VP, _VP, _VP, _VP]
        L.kmp_path_step.restype = C.c_int
        L.kmp_dgemm_grouped.argtypes = [_VP, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _VP, _VP,
                                        _VP]
        L.kmp_dgemm_grouped.restype = C.c_int
        I32, I64 = C.c_int32, C.c_int64
        L.kmp_layer_norm.argtypes = [_VP, I32, _VP, I64, I64, I64, I32, _VP, _VP, C.c_double, I32,
                                     _VP, I64, _VP, _VP, _VP]
        L.kmp_layer_norm.restype = C.c_int
        L.kmp_layer_norm_workspace_bytes.argtypes = [I32, I64, I64]
        L.kmp_layer_norm_workspace_bytes.restype = C.c_size_t
        L.kmp_layer_norm_backward.argtypes = [_VP, I32, _VP, I64, _VP, I64, I64, I64, I32, _VP, _VP,
                                              _VP, _VP, I64, _VP, _VP, _VP, C.c_size_t]
        L.kmp_layer_norm_backward.restype = C.c_int
        L.kmp_block_norm.argtypes = [_VP, I32, I32, _VP, I64, _VP, I64, I64, I64, I32, _VP, _VP, _VP, I64,
                                     C.c_double, _VP, _VP, C.c_double, _VP, I64, I32, _VP, I64, _VP, _VP]
        L.kmp_block_norm.restype = C.c_int
        L.kmp_block_norm_workspace_bytes.argtypes = [I32, I64, I64]
        L.kmp_block_norm_workspace_bytes.restype = C.c_size_t
        L.kmp_block_norm_backward.argtypes = [_VP, I32, I32, _VP, I64, _VP, I64, _VP, I64, _VP, I64, I64, I64, I32,
                                              _VP, _VP, _VP, I64, C.c_double, _VP, _VP, _VP, I64, _VP, I64, _VP, I64,
                                              _VP, _VP, _VP, _VP, _VP, C.c_size_t]
        L.kmp_block_norm_backward.restype = C.c_int
        L.kmp_quantize_rows.argtypes = [_VP, I32, _VP, I64, I64, I64, _VP, I64, _VP]
        L.kmp_quantize_rows.restype = C.c_int
        L.kmp_quantized_product.argtypes = [_VP, _VP, I64, _VP, I64, _VP, I64, _VP, I64, I64, _VP,
                                            I32, _VP, I64]
        L.kmp_quantized_product.restype = C.c_int
        L.kmp_dense_product.argtypes = [_VP, I32, _VP, I64, I64, _VP, I64, I64, I64, I32, _VP, I32, I32, _VP, I64, _VP,
                                        I64, _VP, I64]
        L.kmp_dense_product.restype = C.c_int
        L.kmp_dense_product_workspace_bytes.argtypes = [I32, I64, I64, I64]
        L.kmp_dense_product_workspace_bytes.restype = C.c_size_t
        L.kmp_dense_product_backward.argtypes = [_VP, I32, _VP, I64, I64, I64, I64, I32, _VP, I64, _VP, I64, _VP, I64,
                                                 _VP, I64, _VP, I64, I32, _VP, _VP, C.c_size_t]
        L.kmp_dense_product_backward.restype = C.c_int
        L.kmp_token_logprobs_workspace_bytes.argtypes = [I64, I64, I32]
        L.kmp_token_logprobs_workspace_bytes.restype = C.c_size_t
        L.kmp_token_logprobs.argtypes = [_VP, I32, _VP, I64, I64, I64, I32, _VP, _VP, _VP, _VP, I32,
                                         _VP, _VP, _VP, C.c_size_t]
        L.kmp_token_logprobs.restype = C.c_int
        L.kmp_token_logprobs_backward.argtypes = [_VP, I32, _VP, I64, I64, I64, I32, _VP, _VP, _VP,
                                                  _VP, _VP, _VP, I64]
        L.kmp_token_logprobs_backward.restype = C.c_int
        L.kmp_sample_tokens_workspace_bytes.argtypes = [I64, I64]
        L.kmp_sample_tokens_workspace_bytes.restype = C.c_size_t
        L.kmp_sample_tokens.argtypes = [_VP, I32, _VP, I64, I64, I64, _VP, _VP, _VP, _VP, _VP, I32, _VP, _VP, _VP,
                                        C.c_size_t]
        L.kmp_sample_tokens.restype = C.c_int
        L.kmp_strerror.argtypes = [C.c_int]
        L.kmp_strerror.restype = C.c_char_p
        L.kmp_version.argtypes = []
        L.kmp_version.restype = C.c_char_p
        L.kmp_kernel_class_name.argtypes = [C.c_int]
        L.kmp_kernel_class_name.restype = C.c_char_p
        _lib = L
    return _lib


EXPORTED = ("kmp_default_spec", "kmp_workspace_bytes", "kmp_fit_path", "kmp_make_folds",
            "kmp_rbf_gram", "kmp_rbf_gram_noalloc", "kmp_tridiag", "kmp_band_reduce",
            "kmp_path_step",
            "kmp_dgemm_grouped", "kmp_layer_norm", "kmp_layer_norm_workspace_bytes",
            "kmp_layer_norm_backward", "kmp_block_norm", "kmp_block_norm_workspace_bytes",
            "kmp_block_norm_backward", "kmp_quantize_rows", "kmp_quantized_product",
            "kmp_dense_product", "kmp_dense_product_workspace_bytes", "kmp_dense_product_backward",
            "kmp_token_logprobs", "kmp_token_logprobs_workspace_bytes",
            "kmp_token_logprobs_backward", "kmp_sample_tokens", "kmp_sample_tokens_workspace_bytes",
            "kmp_strerror", "kmp_version", "kmp_kernel_class_name")
KMP_BAND = 16


def kmp_kernel_class_name(cls: int) -> str:
    return lib().kmp_kernel_class_name(int(cls)).decode()


def kmp_strerror(code: int) -> str:
    return lib().kmp_strerror(int(code)).decode()


def kmp_version() -> str:
    return lib().kmp_version().decode()


def _check(code: int, allow_maxiter: bool = True) -> int:
    if code == KMP_OK or (allow_maxiter and code in (KMP_WMAXITER, KMP_WNOTEXACT)):
        return code
    raise KmpError(code, kmp_strerror(code))


def kmp_default_spec(loss: str = "hinge", **overrides) -> kmp_path_spec:
    s = kmp_path_spec()
    lib().kmp_default_spec(C.byref(s))
    s.loss = LOSS_CODES[loss] if isinstance(loss, str) else int(loss)
    for k, v in overrides.items():
        setattr(s, k, v)
    return s


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _f64(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.float64)


def kmp_make_folds(n: int, V: int, seed: int) -> np.ndarray:
    out = np.empty(n, dtype=np.int32)
    _check(lib().kmp_make_folds(int(n), int(V), C.c_uint64(seed & (2 ** 64 - 1)),
                                out.ctypes.data_as(_IP)))
    return out


def kmp_workspace_bytes(spec, n, d, L, fold_id, V, S, Q, sigma_batch) -> int:
    f = _i32(fold_id)
    return int(lib().kmp_workspace_bytes(C.byref(spec), int(n), int(d), int(L),
                                         f.ctypes.data_as(_IP), int(V), int(S), int(Q),
                                         int(sigma_batch)))


_current = None      # (device, handle of its current stream), once HIP is up


def _stream_ptr(stream) -> int:
    global _current
    if stream is None:
        if _current is not None:
            return _current[1](_current[0]())          # 0.2 us; a stream object takes 2.9
        import torch
        stream = torch.cuda.current_stream()
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            _current = torch._C._cuda_getDevice, raw
    return int(stream.cuda_stream)


def kmp_rbf_gram(X, rows, cols, sigmas, out, stream=None) -> None:
    """a1 on its own (see kmpath.h). X, rows, cols, out are device tensors."""
    sig = _f64(sigmas)
    _check(lib().kmp_rbf_gram(_stream_ptr(stream), X.data_ptr(), X.shape[0], X.shape[1],
                              X.stride(0), rows.data_ptr(), rows.numel(), cols.data_ptr(),
                              cols.numel(), sig.ctypes.data_as(_DP), sig.size, out.data_ptr(),
                              out.stride(-2)))


def kmp_tridiag(A, Q, diag, off, stream=None) -> None:
    """a2 on its own: A (G, N, N) device tensor, destroyed; Q/diag/off outputs."""
    G, N = A.shape[0], A.shape[1]
    _check(lib().kmp_tridiag(_stream_ptr(stream), A.data_ptr(), G, N, Q.data_ptr(),
                             diag.data_ptr(), off.data_ptr()))


def kmp_band_reduce(A, Q, band, stream=None) -> None:
    """a2 on its own, band form: A (G, N, N) device tensor, destroyed; Q
    (G, N, N) and band (G, KMP_BAND+1, N) outputs, band[g, r, j] = B[j+r, j]."""
    G, N = A.shape[0], A.shape[1]
    _check(lib().kmp_band_reduce(_stream_ptr(stream), A.data_ptr(), G, N, Q.data_ptr(),
                                 band.data_ptr()))


def kmp_path_step(loss, delta, K, y, lambdas, alpha_in, beta_in, alpha_out, beta_out,
                  kkt_out=None, taus=None, stream=None) -> None:
    """a4-a7 on their own (see kmpath.h): K (n, n), y (n), alpha (C, n), beta
    (C) device tensors; lambdas (and taus) host arrays of C entries."""
    lam = _f64(lambdas)
    tau = _f64(taus) if taus is not None else None
    code = lib().kmp_path_step(
        _stream_ptr(stream), LOSS_CODES[loss] if isinstance(loss, str) else int(loss),
        float(delta if delta is not None else 1.0), K.data_ptr(), K.shape[0], y.data_ptr(),
        lam.ctypes.data_as(_DP), tau.ctypes.data_as(_DP) if tau is not None else None, lam.size,
        alpha_in.data_ptr(), beta_in.data_ptr(), alpha_out.data_ptr(), beta_out.data_ptr(),
        kkt_out.data_ptr() if kkt_out is not None else None)
    _check(code, allow_maxiter=False)


def kmp_dgemm_grouped(A, B, C, stream=None) -> None:
    """C[g] = A[g] @ B[g] for (G, M, K), (G, K, N), (G, M, N) device tensors."""
    G, M, K = A.shape
    N = B.shape[2]
    _check(lib().kmp_dgemm_grouped(_stream_ptr(stream), G, M, N, K, A.data_ptr(), B.data_ptr(),
                                   C.data_ptr()), allow_maxiter=False)


# ------------------------------------------ operators at a language model's end
# Tensors are on the current device, and so is `stream` (others are refused);
# matrices are 2-D with consecutive elements in a row and any row stride, vectors
# are contiguous. Nothing waits for the device: `stream` (the current stream if
# None) carries the work, and tensors made on another stream are the caller's to
# order.
_TYPES: dict = {}


def _type(dtype, name: str) -> int:
    """KMP_* code of a torch type."""
    code = _TYPES.get(dtype)
    if code is None:
        import torch
        _TYPES.update({torch.float64: KMP_F64, torch.float32: KMP_F32, torch.bfloat16: KMP_BF16,
                       torch.float16: KMP_F16, torch.int8: KMP_I8})
        code = _TYPES.get(dtype)
        if code is None:
            raise KmpError(KMP_EINVAL, f"{name}: type {dtype} is not supported")
    return code


def _refuse(what: str):
    raise KmpError(KMP_EINVAL, what)


def _place(t, name: str, stream):
    """(index of the tensor's device, handle of the stream); both are of the
    current device: a kernel that ran elsewhere would not own the memory."""
    if stream is None and _current is not None:
        now = _current[0]()
        handle = _current[1](now)
    else:
        import torch
        handle, now = _stream_ptr(stream), torch.cuda.current_device()
        if stream is not None and getattr(stream, "device_index", now) != now:
            _refuse(f"the stream is of device {stream.device_index}, the current device is {now}")
    if t.get_device() != now:
        _refuse(f"{name} is on device {t.get_device()}, the current device is {now}")
    return now, handle


def _matrix(t, name: str, rows=None, cols=None, dtype=None, on=None):
    """(pointer, rows, columns, row stride) of a 2-D tensor of device `on` (None:
    of any)."""
    shape = t.shape
    if len(shape) != 2 or (not t.is_cuda if on is None else t.get_device() != on):
        _refuse(f"{name} must be a 2-D device tensor" + ("" if on is None else f" of device {on}"))
    r, c = shape
    sr, sc = t.stride()
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        _refuse(f"{name} has shape {r} x {c}, not {rows} x {cols}")
    if dtype is not None and t.dtype != dtype:
        _refuse(f"{name} has type {t.dtype}, not {dtype}")
    if r <= 1:
        sr = c or 1
    if (sc != 1 and c > 1) or sr < c:
        _refuse(f"{name} must have consecutive elements in a row and rows that do not overlap")
    return t.data_ptr(), r, c, sr or 1


def _vector(t, name: str, n: int, dtype=None, on=None):
    """Pointer of a contiguous tensor of n elements of device `on` (None: of any);
    None stays None."""
    if t is None:
        return None
    if (not t.is_cuda if on is None else t.get_device() != on) or t.numel() != n or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous device tensor of {n} elements" + ("" if on is None else f" of device {on}"))
    if dtype is not None and t.dtype != dtype:
        _refuse(f"{name} has type {t.dtype}, not {dtype}")
    return t.data_ptr()


def _tokens(t, n: int, on=None):
    """(bits, pointer) of the tokens; None stays None."""
    if t is None:
        return 32, None
    import torch
    if t.dtype != torch.int64 and t.dtype != torch.int32:
        _refuse(f"tokens have type {t.dtype}, not int32 or int64")
    return t.dtype.itemsize * 8, _vector(t, "tokens", n, None, on)


def _workspace(t, on):
    if t is None:
        return None, 0
    if t.get_device() != on or not t.is_contiguous():
        _refuse(f"workspace must be a contiguous device tensor of device {on}")
    return t.data_ptr(), t.numel() * t.element_size()


def kmp_layer_norm(x, gamma, beta, eps, y, mean=None, rstd=None, scale=None, stream=None) -> None:
    """Layer norm of the rows of x (rows, d) into y: of x's type, or int8 with
    the rows' scales in `scale`. gamma and beta (d) are of x's type or float32
    (None: ones, zeros); mean and rstd (rows) take what the backward reads."""
    xp, rows, d, ldx = _matrix(x, "x")
    on, sp = _place(x, "x", stream)
    yp, _, _, ldy = _matrix(y, "y", rows, d, None, on)
    xt = _type(x.dtype, "x")
    w = gamma if gamma is not None else beta
    wd = w.dtype if w is not None else x.dtype
    sd = rd = None
    if mean is not None or rstd is not None or scale is not None:
        import torch
        sd, rd = torch.float64 if xt == KMP_F64 else torch.float32, torch.float32
    _check(lib().kmp_layer_norm(
        sp, xt, xp, rows, d, ldx, _type(wd, "gamma"), _vector(gamma, "gamma", d, wd, on),
        _vector(beta, "beta", d, wd, on), float(eps), _type(y.dtype, "y"), yp, ldy,
        _vector(mean, "mean", rows, sd, on), _vector(rstd, "rstd", rows, sd, on),
        _vector(scale, "scale", rows, rd, on)), allow_maxiter=False)


def kmp_layer_norm_workspace_bytes(rows: int, d: int, dtype) -> int:
    return int(lib().kmp_layer_norm_workspace_bytes(_type(dtype, "x"), int(rows), int(d)))


def kmp_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, workspace, stream=None) -> None:
    """Gradients of kmp_layer_norm from dy (rows, d): dx (rows, d) of x's type,
    dgamma and dbeta (d) of gamma's; each may be None. The workspace has
    kmp_layer_norm_workspace_bytes(rows, d, x.dtype) bytes."""
    import torch
    xp, rows, d, ldx = _matrix(x, "x")
    on, sp = _place(x, "x", stream)
    dyp, _, _, lddy = _matrix(dy, "dy", rows, d, x.dtype, on)
    dxp, lddx = None, d
    if dx is not None:
        dxp, _, _, lddx = _matrix(dx, "dx", rows, d, x.dtype, on)
    xt = _type(x.dtype, "x")
    wd = next((t.dtype for t in (gamma, dgamma, dbeta) if t is not None), x.dtype)
    sd = torch.float64 if xt == KMP_F64 else torch.float32
    wsp, wsb = _workspace(workspace, on)
    _check(lib().kmp_layer_norm_backward(
        sp, xt, dyp, lddy, xp, ldx, rows, d, _type(wd, "gamma"), _vector(gamma, "gamma", d, wd, on),
        _vector(mean, "mean", rows, sd, on), _vector(rstd, "rstd", rows, sd, on), dxp, lddx,
        _vector(dgamma, "dgamma", d, wd, on), _vector(dbeta, "dbeta", d, wd, on), wsp, wsb),
        allow_maxiter=False)


def _gate(t, name, rows, d, xdtype, wdtype, on):
    """(pointer, leading dimension) of a gate: (d) of the weights' type, leading
    dimension 0, or (rows, d) of x's type; None stays None."""
    if t is None:
        return None, 0
    if t.dim() == 2:
        p, _, _, ld = _matrix(t, name, rows, d, xdtype, on)
        return p, max(ld, d)
    return _vector(t, name, d, wdtype, on), 0


def _block_weights(x, *weights):
    """The weights' type: the first given vector's, else x's."""
    for t in weights:
        if t is not None and t.dim() == 1:
            return t.dtype
    return x.dtype


def kmp_block_norm(b, res, h, y, eps, gamma_after=None, beta_after=None, gate=None, gamma=None, beta=None,
                   rscale=1.0, after=True, rms=False, stats=None, scale=None, stream=None) -> None:
    """h = rscale res + gate n and y = N(h; gamma, beta), n = N(b; gamma_after,
    beta_after) with `after`, else b; N the layer norm or, with `rms`, the norm by
    the root mean square. b, res, h (rows, d) of one type, y of that type or int8
    with the rows' scales in `scale`; res, h or y may be None; h may be res. The
    weights (d) and a gate (d) are of b's type or float32, a gate (rows, d) of b's;
    stats (rows, 4) float32 takes what the backward reads."""
    bp, rows, d, ldb = _matrix(b, "b")
    on, sp = _place(b, "b", stream)
    rp = hp = yp = None
    ldr = ldh = ldy = d
    if res is not None:
        rp, _, _, ldr = _matrix(res, "res", rows, d, b.dtype, on)
    if h is not None:
        hp, _, _, ldh = _matrix(h, "h", rows, d, b.dtype, on)
    yt = _type(b.dtype, "b")
    if y is not None:
        yp, _, _, ldy = _matrix(y, "y", rows, d, None, on)
        yt = _type(y.dtype, "y")
    wd = _block_weights(b, gamma_after, beta_after, gamma, beta, gate)
    gp, ldg = _gate(gate, "gate", rows, d, b.dtype, wd, on)
    bt = _type(b.dtype, "b")
    st = sc = None
    if stats is not None or scale is not None:
        import torch
        st, sc = _vector(stats, "stats", 4 * rows, torch.float32, on), _vector(scale, "scale", rows, torch.float32, on)
    _check(lib().kmp_block_norm(
        sp, bt, (KMP_NORM_RMS if rms else 0) | (KMP_NORM_AFTER if after else 0), bp, ldb, rp, ldr, rows, d,
        bt if wd is b.dtype else _type(wd, "gamma"),
        None if gamma_after is None else _vector(gamma_after, "gamma_after", d, wd, on),
        None if beta_after is None else _vector(beta_after, "beta_after", d, wd, on), gp, ldg, float(rscale),
        None if gamma is None else _vector(gamma, "gamma", d, wd, on),
        None if beta is None else _vector(beta, "beta", d, wd, on), float(eps), hp, ldh, yt, yp, ldy, st, sc), allow_maxiter=False)


def kmp_block_norm_workspace_bytes(rows: int, d: int, dtype) -> int:
    return int(lib().kmp_block_norm_workspace_bytes(_type(dtype, "b"), int(rows), int(d)))


def kmp_block_norm_backward(dy, dh, b, h, stats, db, dres, gamma_after=None, beta_after=None, gate=None, gamma=None,
                            rscale=1.0, after=True, rms=False, dgate=None, dgamma_after=None, dbeta_after=None,
                            dgamma=None, dbeta=None, workspace=None, stream=None) -> None:
    """Gradients of kmp_block_norm from dy and dh (rows, d), the gradients of y and
    of h (one may be None): db and dres (rows, d) of b's type, dgate of the gate's
    shape, dgamma_after, dbeta_after, dgamma, dbeta (d) of the weights' type; each may
    be None. h and stats are the forward call's (h may be None without dy). The
    workspace has kmp_block_norm_workspace_bytes(rows, d, b.dtype) bytes."""
    import torch
    bp, rows, d, ldb = _matrix(b, "b")
    on, sp = _place(b, "b", stream)

    def matrix(t, name):
        if t is None:
            return None, d
        p, _, _, ld = _matrix(t, name, rows, d, b.dtype, on)
        return p, ld

    (dyp, lddy), (dhp, lddh), (hp, ldh) = matrix(dy, "dy"), matrix(dh, "dh"), matrix(h, "h")
    (dbp, lddb), (drp, lddr) = matrix(db, "db"), matrix(dres, "dres")
    wd = _block_weights(b, gamma_after, beta_after, gamma, gate, dgate, dgamma_after, dbeta_after, dgamma, dbeta)
    gp, ldg = _gate(gate, "gate", rows, d, b.dtype, wd, on)
    if gate is not None and dgate is not None and dgate.dim() != gate.dim():
        _refuse("dgate has the shape of the gate")
    dgp, lddg = _gate(dgate, "dgate", rows, d, b.dtype, wd, on)
    wsp, wsb = _workspace(workspace, on)
    v = lambda t, name: _vector(t, name, d, wd, on)  # noqa: E731
    _check(lib().kmp_block_norm_backward(
        sp, _type(b.dtype, "b"), (KMP_NORM_RMS if rms else 0) | (KMP_NORM_AFTER if after else 0), dyp, lddy, dhp, lddh,
        bp, ldb, hp, ldh, rows, d, _type(wd, "gamma"), v(gamma_after, "gamma_after"), v(beta_after, "beta_after"), gp, ldg,
        float(rscale), v(gamma, "gamma"), _vector(stats, "stats", 4 * rows, torch.float32, on), dbp, lddb, drp, lddr,
        dgp, lddg, v(dgamma_after, "dgamma_after"), v(dbeta_after, "dbeta_after"), v(dgamma, "dgamma"),
        v(dbeta, "dbeta"), wsp, wsb), allow_maxiter=False)


def kmp_quantize_rows(x, q, scale, stream=None) -> None:
    """Rows of x (rows, d) in 8 bits: q (rows, d) int8, scale (rows) float32."""
    import torch
    xp, rows, d, ldx = _matrix(x, "x")
    on, sp = _place(x, "x", stream)
    qp, _, _, ldq = _matrix(q, "q", rows, d, torch.int8, on)
    _check(lib().kmp_quantize_rows(sp, _type(x.dtype, "x"), xp, rows, d, ldx, qp, ldq,
                                   _vector(scale, "scale", rows, torch.float32, on)), allow_maxiter=False)


def kmp_quantized_product(xq, xscale, wq, wscale, out, bias=None, stream=None) -> None:
    """out (M, N) = xscale[m] wscale[n] sum_k xq[m, k] wq[n, k] + bias[n] for
    int8 xq (M, K) and wq (N, K), float32 scales and bias, out of any of the
    floating types up to 32 bits."""
    import torch
    xp, M, K, ldx = _matrix(xq, "xq", dtype=torch.int8)
    on, sp = _place(xq, "xq", stream)
    wp, N, _, ldw = _matrix(wq, "wq", None, K, torch.int8, on)
    op, _, _, ldo = _matrix(out, "out", M, N, None, on)
    f = torch.float32
    _check(lib().kmp_quantized_product(
        sp, xp, ldx, _vector(xscale, "xscale", M, f, on), M, wp, ldw,
        _vector(wscale, "wscale", N, f, on), N, K, _vector(bias, "bias", N, f, on), _type(out.dtype, "out"), op,
        ldo), allow_maxiter=False)


def _act(act) -> int:
    code = ACT_CODES.get(act)
    if code is None:
        _refuse(f"activation {act!r} is not one of {', '.join(ACT_CODES)}")
    return code


def kmp_dense_product(x, w, out, bias=None, act="none", residual=None, z=None, stream=None) -> None:
    """out (M, N) = act(z) + residual, z = x w' + bias, for x (M, K) and w (N, K) of one
    type up to 32 bits; out and residual of that type or float32, bias (N), too; z
    (M, N) of x's type takes what the backward reads. act: none, relu, gelu, gelu_tanh
    or silu. out may be residual."""
    xp, M, K, ldx = _matrix(x, "x")
    on, sp = _place(x, "x", stream)
    wp, N, _, ldw = _matrix(w, "w", None, K, x.dtype, on)
    op, _, _, ldo = _matrix(out, "out", M, N, None, on)
    rp = zp = None
    ldr = ldz = ldo
    if residual is not None:
        rp, _, _, ldr = _matrix(residual, "residual", M, N, out.dtype, on)
    if z is not None:
        zp, _, _, ldz = _matrix(z, "z", M, N, x.dtype, on)
    t = _type(x.dtype, "x")
    bt = t if bias is None else _type(bias.dtype, "bias")
    _check(lib().kmp_dense_product(sp, t, xp, ldx, M, wp, ldw, N, K, bt, _vector(bias, "bias", N, None, on), _act(act),
                                   _type(out.dtype, "out"), rp, ldr, op, ldo, zp, ldz), allow_maxiter=False)


def kmp_dense_product_workspace_bytes(M: int, N: int, K: int, dtype) -> int:
    return int(lib().kmp_dense_product_workspace_bytes(_type(dtype, "x"), int(M), int(N), int(K)))


def kmp_dense_product_backward(dout, x, w, z, dx, dw, dbias, act="none", workspace=None, stream=None) -> None:
    """Gradients of kmp_dense_product from dout (M, N): dx (M, K) and dw (N, K) of
    x's type, dbias (N) of that type or float32; each may be None, and x without dw, w
    without dx. z is what the forward call wrote (None for act "none"). The workspace
    has kmp_dense_product_workspace_bytes(M, N, K, dtype) bytes."""
    dp, M, N, lddo = _matrix(dout, "dout")
    on, sp = _place(dout, "dout", stream)
    code = _act(act)
    t = _type(dout.dtype, "dout")
    K = next((m.shape[-1] for m in (x, w, dx, dw) if m is not None), 0)

    def matrix(m, name, rows, cols):
        if m is None:
            return None, cols
        p, _, _, ld = _matrix(m, name, rows, cols, dout.dtype, on)
        return p, ld

    zp, ldz = matrix(z, "z", M, N)
    xp, ldx = matrix(x, "x", M, K)
    wp, ldw = matrix(w, "w", N, K)
    dxp, lddx = matrix(dx, "dx", M, K)
    dwp, lddw = matrix(dw, "dw", N, K)
    bt = t if dbias is None else _type(dbias.dtype, "dbias")
    wsp, wsb = _workspace(workspace, on)
    _check(lib().kmp_dense_product_backward(sp, t, dp, lddo, M, N, K, code, zp, ldz, xp, ldx, wp, ldw, dxp, lddx, dwp, lddw,
                                            bt, _vector(dbias, "dbias", N, None, on), wsp, wsb), allow_maxiter=False)


def kmp_token_logprobs_workspace_bytes(T: int, V: int, top: int = 0) -> int:
    return int(lib().kmp_token_logprobs_workspace_bytes(int(T), int(V), int(top)))


def kmp_token_logprobs(logits, tokens, logp, entropy=None, stats=None, top_id=None, top_logp=None,
                       workspace=None, stream=None) -> None:
    """Log probabilities of tokens (T; int32 or int64, negative: none) under the
    rows of logits (T, V): logp and entropy (T) float32, stats (T, 2) float32
    (maximum m, log sum exp(x - m); what the backward reads), the most likely
    tokens top_id (T, k) int32 and their top_logp (T, k) float32; each output
    may be None. The workspace has kmp_token_logprobs_workspace_bytes(T, V, k)
    bytes."""
    import torch
    lp, T, V, ldl = _matrix(logits, "logits")
    on, sp = _place(logits, "logits", stream)
    bits, tp = _tokens(tokens, T, on)
    tops = [t.shape[-1] for t in (top_id, top_logp) if t is not None]
    top = tops[0] if tops else 0
    f = torch.float32
    wsp, wsb = _workspace(workspace, on)
    _check(lib().kmp_token_logprobs(
        sp, _type(logits.dtype, "logits"), lp, T, V, ldl, bits, tp,
        _vector(logp, "logp", T, f, on), _vector(entropy, "entropy", T, f, on), _vector(stats, "stats", 2 * T, f, on), top,
        _vector(top_id, "top_id", T * top, torch.int32, on), _vector(top_logp, "top_logp", T * top, f, on),
        wsp, wsb), allow_maxiter=False)


def kmp_token_logprobs_backward(logits, tokens, stats, dlogp, dlogits, entropy=None, dentropy=None,
                                stream=None) -> None:
    """Gradient dlogits (T, V) of sum dlogp logp + dentropy entropy, from the
    forward call's logits, tokens, stats and entropy; dlogp or dentropy may be
    None. dlogits may be logits itself."""
    import torch
    lp, T, V, ldl = _matrix(logits, "logits")
    on, sp = _place(logits, "logits", stream)
    dp, _, _, ldd = _matrix(dlogits, "dlogits", T, V, logits.dtype, on)
    bits, tp = _tokens(tokens, T, on)
    f = torch.float32
    _check(lib().kmp_token_logprobs_backward(
        sp, _type(logits.dtype, "logits"), lp, T, V, ldl, bits, tp,
        _vector(stats, "stats", 2 * T, f, on), _vector(entropy, "entropy", T, f, on), _vector(dlogp, "dlogp", T, f, on),
        _vector(dentropy, "dentropy", T, f, on), dp, ldd), allow_maxiter=False)


def kmp_sample_tokens_workspace_bytes(T: int, V: int) -> int:
    return int(lib().kmp_sample_tokens_workspace_bytes(int(T), int(V)))


def kmp_sample_tokens(logits, u, tokens, temperature=None, top_k=None, top_p=None, min_p=None, logp=None,
                      workspace=None, stream=None) -> None:
    """Tokens (T; int32 or int64) drawn from the rows of logits (T, V) with the
    random numbers u (T) float32 in [0, 1): kept are the first top_k (T) int32 in
    the order of the logits, of these the shortest run that has top_p (T) of their
    weight, of these the tokens with at least min_p (T) of the first one's weight;
    weights at the temperature (T). Each of these may be None; logp (T) float32 takes
    the drawn tokens' log probabilities among the kept ones. The workspace has
    kmp_sample_tokens_workspace_bytes(T, V) bytes."""
    import torch
    lp, T, V, ldl = _matrix(logits, "logits")
    on, sp = _place(logits, "logits", stream)
    bits, tp = _tokens(tokens, T, on)
    f = torch.float32
    wsp, wsb = _workspace(workspace, on)
    _check(lib().kmp_sample_tokens(
        sp, _type(logits.dtype, "logits"), lp, T, V, ldl, _vector(u, "u", T, f, on),
        _vector(temperature, "temperature", T, f, on), _vector(top_k, "top_k", T, torch.int32, on),
        _vector(top_p, "top_p", T, f, on), _vector(min_p, "min_p", T, f, on), bits, tp, _vector(logp, "logp", T, f, on),
        wsp, wsb), allow_maxiter=False)


def kmp_fit_path(stream, spec, X, y, sigmas, taus, lambdas, fold_id, V, workspace, ws_bytes,
                 alpha, beta, objective, cv_sum, cv_err, iters, status, selected, timings,
                 selected_joint=None) -> int:
    """Direct call of the C entry point (device pointers as ints, host arrays as numpy)."""
    sig, tau, lam, fold = _f64(sigmas), _f64(taus), _f64(lambdas), _i32(fold_id)
    return lib().kmp_fit_path(
        stream, C.byref(spec), X.data_ptr(), X.shape[0], X.shape[1], X.stride(0), y.data_ptr(),
        sig.ctypes.data_as(_DP), sig.size, tau.ctypes.data_as(_DP), max(1, tau.size),
        lam.ctypes.data_as(_DP), lam.size, fold.ctypes.data_as(_IP), int(V), workspace,
        int(ws_bytes), alpha.data_ptr(), beta.data_ptr(), objective.data_ptr(), cv_sum.data_ptr(),
        cv_err.data_ptr() if cv_err is not None else None,
        iters.data_ptr() if iters is not None else None,
        status.data_ptr() if status is not None else None,
        selected.ctypes.data_as(_IP) if selected is not None else None,
        selected_joint.ctypes.data_as(_IP) if selected_joint is not None else None,
        C.byref(timings) if timings is not None else None)


class PathRunner:
    """Holds the workspace and output tensors for repeated fits of one problem shape."""

    def __init__(self, X, y, loss, sigmas, lambdas, fold_id, V, taus=None, device="cuda",
                 sigma_batch: Optional[int] = None, kernel_timing=(), refit: bool = False,
                 shared: bool = False, exact_hinge: bool = False, eager: bool = False,
                 **spec_overrides):
        """refit=True: every (sigma, tau, lambda) on all n points (fold_id and V
        are ignored; outputs have V = 1, no CV sums, no selection).
        shared=True: exact CV on one factor of the full K per bandwidth
        (KMP_FLAG_SHARED_FACTOR); V = n with fold_id = 0..n-1 is leave-one-out.
        eager=True: every iteration launched directly, never from a recorded
        HIP graph (KMP_FLAG_EAGER)."""
        import torch
        self.torch = torch
        self.loss = loss
        self.spec = kmp_default_spec(loss, **spec_overrides)
        if refit:
            self.spec.flags |= KMP_FLAG_REFIT
            fold_id, V = np.zeros(np.shape(X)[0], dtype=np.int32), 1
        if shared:
            self.spec.flags |= KMP_FLAG_SHARED_FACTOR
        if exact_hinge:
            self.spec.flags |= KMP_FLAG_EXACT_HINGE
        if eager:
            self.spec.flags |= KMP_FLAG_EAGER
        self.set_kernel_timing(kernel_timing)
        self.X = torch.as_tensor(np.ascontiguousarray(X), dtype=torch.float64, device=device) \
            if not isinstance(X, torch.Tensor) else X
        self.y = torch.as_tensor(np.ascontiguousarray(y), dtype=torch.float64, device=device) \
            if not isinstance(y, torch.Tensor) else y
        self.sigmas = _f64(np.atleast_1d(sigmas))
        self.lambdas = _f64(lambdas)
        self.taus = _f64(taus) if (loss == "check") else np.zeros(1)
        self.fold = _i32(fold_id)
        self.V = int(V)
        n, d = self.X.shape
        S, Q, L = self.sigmas.size, (self.taus.size if loss == "check" else 1), self.lambdas.size
        self.shape = (S, Q, self.V, L)
        sb = S if sigma_batch is None else int(sigma_batch)
        self.ws_bytes = kmp_workspace_bytes(self.spec, n, d, L, self.fold, self.V, S, Q, sb)
        if self.ws_bytes == 0:
            raise KmpError(KMP_EINVAL, "invalid problem for workspace sizing")
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device)
        cells = S * Q * self.V * L
        self.alpha = torch.empty((S, Q, self.V, L, n), dtype=torch.float64, device=device)
        self.beta = torch.empty(self.shape, dtype=torch.float64, device=device)
        self.objective = torch.empty(self.shape, dtype=torch.float64, device=device)
        self.cv_sum = torch.empty(self.shape, dtype=torch.float64, device=device)
        self.cv_err = torch.empty(self.shape, dtype=torch.int32, device=device)
        self.iters = torch.empty(self.shape, dtype=torch.int32, device=device)
        self.status = torch.empty(self.shape, dtype=torch.int32, device=device)
        self.selected = np.zeros((S, Q), dtype=np.int32)
        self.selected_joint = np.zeros((Q, 2), dtype=np.int32)
        self.timings = kmp_timings()
        self.cells = cells

    def set_kernel_timing(self, classes, every: int = 1) -> None:
        """Time the named kernel classes with HIP events on the next runs,
        bracketing one launch in every `every` of each class."""
        mask = 0
        for c in classes:
            mask |= 1 << (KERNEL_CLASSES.index(c) if isinstance(c, str) else int(c))
        self.spec.timing_mask = mask
        self.spec.timing_every = int(every)

    def kernel_times(self) -> dict:
        return self.timings.kernels()

    def run(self, stream=None) -> int:
        code = kmp_fit_path(_stream_ptr(stream), self.spec, self.X, self.y, self.sigmas,
                            self.taus, self.lambdas, self.fold, self.V, self.workspace.data_ptr(),
                            self.ws_bytes, self.alpha, self.beta, self.objective, self.cv_sum,
                            self.cv_err, self.iters, self.status, self.selected, self.timings,
                            self.selected_joint)
        return _check(code)

    def results(self) -> dict:
        out = {k: getattr(self, k).cpu().numpy() for k in
               ("alpha", "beta", "objective", "cv_sum", "cv_err", "iters", "status")}
        out["selected"] = self.selected.copy()
        out["selected_joint"] = self.selected_joint.copy()
        out["timings"] = self.timings.as_dict()
        return out


def fit_path(X, y, loss, sigmas, lambdas, fold_id, V, taus=None, **spec_overrides) -> dict:
    """One call of kmp_fit_path with freshly allocated outputs; returns numpy results."""
    r = PathRunner(X, y, loss, sigmas, lambdas, fold_id, V, taus=taus, **spec_overrides)
    code = r.run()
    out = r.results()
    out["code"] = code
    return out
