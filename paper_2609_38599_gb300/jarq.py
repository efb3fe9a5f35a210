"""Python binding of the JARQ C ABI (``include/jarq.h``).

Argument marshalling only: every step of the refinement runs in the CUDA
library ``libjarq.so``.  Tensors are passed as raw pointers on torch's
current CUDA stream; NumPy arrays are passed as host pointers and staged by
the library.  There is no CPU fallback: importing this module raises if the
library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libjarq.so")

JARQ_OK = 0
JARQ_ERR_ARG = 1
JARQ_ERR_NOT_SPD = 2
JARQ_ERR_NUMERICAL = 3
JARQ_ERR_CUDA = 4
JARQ_ERR_TIMEOUT = 5
JARQ_ERR_NOMEM = 6

# Names declared in include/jarq.h (checked by the test-suite).
EXPORTS = ("jarq_default_options", "jarq_prepare_hessian", "jarq_refine_layer",
           "jarq_objective", "jarq_hessian_din", "jarq_hessian_group_size",
           "jarq_hessian_destroy", "jarq_status_string", "jarq_profile_enable",
           "jarq_profile_reset", "jarq_profile_read", "jarq_launch_count",
           "jarq_objective_noalloc", "jarq_residual_product", "jarq_canonicalize",
           "jarq_dequantize", "jarq_pack_codes", "jarq_accumulate_hessian",
           "jarq_refine_layer_mu", "jarq_fit_scales", "jarq_multicode_probe",
           "jarq_selftest_wait_timeout", "jarq_selftest_stalled_kernel",
           "jarq_async_status", "jarq_quantize_rows", "jarq_integer_codes",
           "jarq_integer_product", "jarq_integer_linear_workspace", "jarq_integer_linear",
           "jarq_token_logprobs", "jarq_token_logprobs_grad", "jarq_rms_norm",
           "jarq_rms_norm_grad_workspace", "jarq_rms_norm_grad", "jarq_cross_entropy_workspace",
           "jarq_cross_entropy", "jarq_cross_entropy_grad_workspace", "jarq_cross_entropy_grad",
           "jarq_adapters_workspace", "jarq_apply_adapters")


class JarqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class Options(ctypes.Structure):
    _fields_ = [("max_iters", ctypes.c_int), ("early_stop", ctypes.c_int),
                ("tau_rel", ctypes.c_float), ("tau_abs", ctypes.c_float),
                ("ridge", ctypes.c_float), ("rcond", ctypes.c_float),
                ("eps", ctypes.c_float), ("ridge_accept", ctypes.c_int),
                ("fixed_grid", ctypes.c_int)]


class Stats(ctypes.Structure):
    _fields_ = [("L_host", ctypes.c_void_p), ("L_final", ctypes.c_void_p),
                ("iters", ctypes.c_void_p), ("accepted", ctypes.c_void_p),
                ("ridge_hits", ctypes.c_void_p), ("row_status", ctypes.c_void_p)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"JARQ CUDA library not built: {LIB_PATH} is missing "
                          "(run __graft_entry__.build())")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.jarq_default_options.restype = Options
    lib.jarq_default_options.argtypes = []
    lib.jarq_prepare_hessian.restype = ci
    lib.jarq_prepare_hessian.argtypes = [vp, ci, ci, cf, ctypes.POINTER(vp), vp]
    lib.jarq_refine_layer.restype = ci
    lib.jarq_refine_layer.argtypes = [vp, vp, vp, vp, vp, ci, ci, ctypes.POINTER(Options),
                                      ctypes.POINTER(Stats), vp]
    lib.jarq_refine_layer_mu.restype = ci
    lib.jarq_refine_layer_mu.argtypes = [vp, vp, vp, vp, vp, ci, ci, vp, vp, cf, cf,
                                         ctypes.POINTER(Options), ctypes.POINTER(Stats), vp]
    lib.jarq_fit_scales.restype = ci
    lib.jarq_fit_scales.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, vp]
    lib.jarq_multicode_probe.restype = ci
    lib.jarq_multicode_probe.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, vp, vp, vp, vp, vp, vp]
    lib.jarq_objective.restype = ci
    lib.jarq_objective.argtypes = [vp, vp, vp, vp, vp, ci, ci, vp, vp]
    lib.jarq_objective_noalloc.restype = ci
    lib.jarq_objective_noalloc.argtypes = [vp, vp, vp, vp, vp, ci, ci, vp, vp]
    lib.jarq_residual_product.restype = ci
    lib.jarq_residual_product.argtypes = [vp, vp, vp, vp, vp, ci, ci, vp, vp]
    lib.jarq_canonicalize.restype = ci
    lib.jarq_canonicalize.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp]
    lib.jarq_dequantize.restype = ci
    lib.jarq_dequantize.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, vp, vp]
    lib.jarq_pack_codes.restype = ci
    lib.jarq_pack_codes.argtypes = [vp, ci, ci, ci, vp, vp]
    lib.jarq_accumulate_hessian.restype = ci
    lib.jarq_accumulate_hessian.argtypes = [vp, ci, ci, cf, vp, vp]
    cl = ctypes.c_int64
    lib.jarq_async_status.restype = ci
    lib.jarq_async_status.argtypes = [vp]
    lib.jarq_quantize_rows.restype = ci
    lib.jarq_quantize_rows.argtypes = [vp, ci, ci, ci, cl, vp, cl, vp, vp]
    lib.jarq_integer_codes.restype = ci
    lib.jarq_integer_codes.argtypes = [vp, vp, ci, ci, ci, ci, vp, cl, vp]
    lib.jarq_integer_product.restype = ci
    lib.jarq_integer_product.argtypes = [vp, cl, vp, vp, cl, vp, ci, vp, ci, ci, ci, ci, vp, cl, vp]
    lib.jarq_integer_linear_workspace.restype = ctypes.c_size_t
    lib.jarq_integer_linear_workspace.argtypes = [ci, ci]
    lib.jarq_integer_linear.restype = ci
    lib.jarq_integer_linear.argtypes = [vp, ci, cl, vp, cl, vp, ci, vp, ci, ci, ci, ci, vp, cl, vp,
                                        ctypes.c_size_t, vp]
    lib.jarq_token_logprobs.restype = ci
    lib.jarq_token_logprobs.argtypes = [vp, ci, ci, ci, cl, vp, ci, ci, vp, vp, vp, vp, vp, vp]
    lib.jarq_token_logprobs_grad.restype = ci
    lib.jarq_token_logprobs_grad.argtypes = [vp, ci, ci, ci, cl, vp, ci, vp, vp, vp, vp, vp, cl, vp]
    cz = ctypes.c_size_t
    lib.jarq_rms_norm.restype = ci
    lib.jarq_rms_norm.argtypes = [vp, ci, ci, ci, cl, vp, cl, vp, cl, vp, ci, cf, vp, cl, vp, cl, vp, vp, vp]
    lib.jarq_rms_norm_grad_workspace.restype = cz
    lib.jarq_rms_norm_grad_workspace.argtypes = [ci, ci]
    lib.jarq_rms_norm_grad.restype = ci
    lib.jarq_rms_norm_grad.argtypes = [vp, ci, ci, ci, cl, vp, ci, vp, vp, cl, vp, cl, vp, cl, vp, vp, cz, vp]
    lib.jarq_cross_entropy_workspace.restype = cz
    lib.jarq_cross_entropy_workspace.argtypes = [ci, ci, ci, ci]
    lib.jarq_cross_entropy.restype = ci
    lib.jarq_cross_entropy.argtypes = [vp, ci, ci, ci, cl, vp, ci, cl, vp, vp, vp, vp, cz, vp]
    lib.jarq_cross_entropy_grad_workspace.restype = cz
    lib.jarq_cross_entropy_grad_workspace.argtypes = [ci, ci, ci, ci, ci, ci]
    lib.jarq_cross_entropy_grad.restype = ci
    lib.jarq_cross_entropy_grad.argtypes = [vp, ci, ci, ci, cl, vp, ci, cl, vp, vp, vp, vp, cl, vp, cl, vp, cz, vp]
    lib.jarq_adapters_workspace.restype = cz
    lib.jarq_adapters_workspace.argtypes = [ci, ci, ci, ci]
    lib.jarq_apply_adapters.restype = ci
    lib.jarq_apply_adapters.argtypes = [vp, ci, cl, vp, vp, vp, ci, ci, vp, ci, ci, ci, vp, cl, vp, cl, ci, vp, cz, vp]
    lib.jarq_hessian_din.restype = ci
    lib.jarq_hessian_din.argtypes = [vp]
    lib.jarq_hessian_group_size.restype = ci
    lib.jarq_hessian_group_size.argtypes = [vp]
    lib.jarq_hessian_destroy.restype = None
    lib.jarq_hessian_destroy.argtypes = [vp]
    lib.jarq_status_string.restype = ctypes.c_char_p
    lib.jarq_status_string.argtypes = [ci]
    lib.jarq_profile_enable.restype = None
    lib.jarq_profile_enable.argtypes = [ci]
    lib.jarq_profile_reset.restype = None
    lib.jarq_profile_reset.argtypes = []
    lib.jarq_profile_read.restype = ci
    lib.jarq_profile_read.argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_longlong),
                                      ctypes.POINTER(ctypes.c_double)]
    lib.jarq_launch_count.restype = ctypes.c_longlong
    lib.jarq_launch_count.argtypes = []
    lib.jarq_selftest_wait_timeout.restype = ci
    lib.jarq_selftest_wait_timeout.argtypes = [vp]
    lib.jarq_selftest_stalled_kernel.restype = ci
    lib.jarq_selftest_stalled_kernel.argtypes = [ctypes.c_char_p, vp]
    return lib


_lib = _load()


def library():
    """The loaded ctypes library (for tests that call the C ABI directly)."""
    return _lib


KERNELS = ("validate", "residual", "init_rows", "hr_full", "grad", "gram", "scale_solve",
           "symmetrize", "group_factor", "slices", "slice_rows", "proj", "whw", "rhs", "htilde",
           "ptilde", "syrk", "mu_combine", "own_rhs", "scale_fit", "probe", "sweep_product",
           "sweep_babai", "quantize_rows", "integer_product", "token_logprobs", "token_grad",
           "rms_norm", "norm_grad", "cross_entropy", "cross_entropy_grad", "adapters")


def profile_enable(on: bool = True):
    """Record CUDA events around each library kernel launch (instrumentation)."""
    _lib.jarq_profile_enable(1 if on else 0)


def profile_reset():
    _lib.jarq_profile_reset()


def profile_read(kernel: str):
    """(launches, total device ms) accumulated for one kernel name."""
    n = ctypes.c_longlong()
    ms = ctypes.c_double()
    if _lib.jarq_profile_read(kernel.encode(), ctypes.byref(n), ctypes.byref(ms)) != 0:
        raise KeyError(kernel)
    return int(n.value), float(ms.value)


def launch_count() -> int:
    """Kernels launched by the library since it was loaded."""
    return int(_lib.jarq_launch_count())


def selftest_wait_timeout() -> int:
    """Status of a device wait that nothing completes (JARQ_ERR_TIMEOUT when
    the bounded-wait path works), on the current torch stream."""
    import torch
    return int(_lib.jarq_selftest_wait_timeout(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)))


def selftest_stalled_kernel(kernel: str) -> int:
    """Status of one tensor-core kernel whose waits run out (JARQ_ERR_TIMEOUT),
    on the current torch stream."""
    import torch
    return int(_lib.jarq_selftest_stalled_kernel(
        kernel.encode(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)))


def status_string(status: int) -> str:
    return _lib.jarq_status_string(int(status)).decode()


def default_options(**overrides) -> Options:
    o = _lib.jarq_default_options()
    for k, v in overrides.items():
        if not hasattr(o, k):
            raise KeyError(f"unknown option {k}")
        setattr(o, k, type(getattr(o, k))(v))
    return o


def _is_torch(x):
    return type(x).__module__.startswith("torch")


def _ptr(x, dtype_np):
    """Raw pointer of a contiguous torch tensor or NumPy array of the given dtype."""
    if x is None:
        return None
    if _is_torch(x):
        import torch
        want = {np.float32: torch.float32, np.uint8: torch.uint8, np.int32: torch.int32,
                np.float64: torch.float64}[dtype_np]
        if x.dtype != want or not x.is_contiguous():
            raise TypeError(f"expected a contiguous {want} tensor, got {x.dtype}")
        return x.data_ptr()
    if not isinstance(x, np.ndarray) or x.dtype != dtype_np or not x.flags.c_contiguous:
        raise TypeError(f"expected a C-contiguous {np.dtype(dtype_np)} array")
    return x.ctypes.data


def _stream(*tensors):
    for t in tensors:
        if _is_torch(t) and t.is_cuda:
            import torch
            return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)
    return ctypes.c_void_p(None)


class Hessian:
    """A prepared Hessian (``jarq_prepare_hessian``); freed on ``close``."""

    def __init__(self, H, group_size: int, nu2: float = 0.0):
        d = int(H.shape[0])
        if tuple(H.shape) != (d, d):
            raise ValueError("H must be square")
        handle = ctypes.c_void_p()
        st = _lib.jarq_prepare_hessian(_ptr(H, np.float32), d, int(group_size), float(nu2),
                                       ctypes.byref(handle), _stream(H))
        if st != JARQ_OK:
            raise JarqError(st, "jarq_prepare_hessian")
        self._h = handle
        self.din = d
        self.group_size = int(group_size)

    @property
    def handle(self):
        return self._h

    def close(self):
        if self._h is not None and self._h.value:
            _lib.jarq_hessian_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def prepare(H, group_size: int, nu2: float = 0.0) -> Hessian:
    return Hessian(H, group_size, nu2)


@dataclass
class RefineStats:
    L_host: object
    L_final: object
    iters: object
    accepted: object
    ridge_hits: object
    row_status: object
    status: int


def _alloc_like(ref, n, dtype_np):
    if _is_torch(ref):
        import torch
        tdt = {np.float64: torch.float64, np.int32: torch.int32}[dtype_np]
        return torch.empty(n, dtype=tdt, device=ref.device)
    return np.empty(n, dtype=dtype_np)


def refine(hess: Hessian, W, S, Q, Z, bits: int, options: Options = None,
           collect_stats: bool = True, raise_on_error: bool = True, **opt):
    """``jarq_refine_layer``: refine S and Q in place; returns RefineStats."""
    o = options if options is not None else default_options(**opt)
    dout = int(W.shape[0])
    st = None
    stats = None
    if collect_stats:
        st = RefineStats(*(_alloc_like(W, dout, t) for t in
                           (np.float64, np.float64, np.int32, np.int32, np.int32, np.int32)),
                         status=0)
        stats = Stats(*(_ptr(x, t) for x, t in zip(
            (st.L_host, st.L_final, st.iters, st.accepted, st.ridge_hits, st.row_status),
            (np.float64, np.float64, np.int32, np.int32, np.int32, np.int32))))
    status = _lib.jarq_refine_layer(hess.handle, _ptr(W, np.float32), _ptr(S, np.float32),
                                    _ptr(Q, np.uint8), _ptr(Z, np.int32), dout, int(bits),
                                    ctypes.byref(o), ctypes.byref(stats) if stats else None,
                                    _stream(W, S, Q, Z))
    if st is not None:
        st.status = status
    if raise_on_error and status not in (JARQ_OK,):
        raise JarqError(status, "jarq_refine_layer")
    return st if st is not None else status


def refine_mu(hess: Hessian, W, S, Q, Z, bits: int, K, XX, mu: float, nu2: float,
              options: Options = None, collect_stats: bool = True, raise_on_error: bool = True,
              **opt):
    """``jarq_refine_layer_mu``: refinement on the propagation-corrected target
    (K = X~^T X, XX = X^T X, normalised like the prepared H = X~^T X~ + nu2 I);
    S and Q in place; returns RefineStats with the mu-objective."""
    o = options if options is not None else default_options(**opt)
    dout = int(W.shape[0])
    st = None
    stats = None
    if collect_stats:
        st = RefineStats(*(_alloc_like(W, dout, t) for t in
                           (np.float64, np.float64, np.int32, np.int32, np.int32, np.int32)),
                         status=0)
        stats = Stats(*(_ptr(x, t) for x, t in zip(
            (st.L_host, st.L_final, st.iters, st.accepted, st.ridge_hits, st.row_status),
            (np.float64, np.float64, np.int32, np.int32, np.int32, np.int32))))
    status = _lib.jarq_refine_layer_mu(hess.handle, _ptr(W, np.float32), _ptr(S, np.float32),
                                       _ptr(Q, np.uint8), _ptr(Z, np.int32), dout, int(bits),
                                       _ptr(K, np.float32), _ptr(XX, np.float32), float(mu),
                                       float(nu2), ctypes.byref(o),
                                       ctypes.byref(stats) if stats else None,
                                       _stream(W, S, Q, Z))
    if st is not None:
        st.status = status
    if raise_on_error and status not in (JARQ_OK,):
        raise JarqError(status, "jarq_refine_layer_mu")
    return st if st is not None else status


JARQ_FIT_JOINT, JARQ_FIT_INDEPENDENT, JARQ_FIT_COORDINATE = 0, 1, 2


def fit_scales(hess: Hessian, W, S, Q, Z, bits: int, method: str = "joint", passes: int = 3):
    """``jarq_fit_scales``: refit S in place for the codes Q with the joint,
    independent or coordinate-descent fit; returns (F_before, F_after)."""
    code = {"joint": JARQ_FIT_JOINT, "independent": JARQ_FIT_INDEPENDENT,
            "coordinate": JARQ_FIT_COORDINATE}[method]
    dout = int(W.shape[0])
    Fb, Fa = _alloc_like(W, dout, np.float64), _alloc_like(W, dout, np.float64)
    status = _lib.jarq_fit_scales(hess.handle, _ptr(W, np.float32), _ptr(S, np.float32),
                                  _ptr(Q, np.uint8), _ptr(Z, np.int32), dout, int(bits), code,
                                  int(passes), _ptr(Fb, np.float64), _ptr(Fa, np.float64),
                                  _stream(W, S, Q, Z))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_fit_scales")
    return Fb, Fa


def multicode_probe(hess: Hessian, W, S, Q, Z, bits: int, group: int):
    """``jarq_multicode_probe``: dict of q_search [dout][g] (uint8), moves,
    accepted, changed (int32) and dF (float64) for one group of every row."""
    dout = int(W.shape[0])
    g = hess.group_size
    if _is_torch(W):
        import torch
        qs = torch.empty(dout, g, dtype=torch.uint8, device=W.device)
    else:
        qs = np.empty((dout, g), dtype=np.uint8)
    out = {"q_search": qs, "moves": _alloc_like(W, dout, np.int32),
           "accepted": _alloc_like(W, dout, np.int32), "changed": _alloc_like(W, dout, np.int32),
           "dF": _alloc_like(W, dout, np.float64)}
    status = _lib.jarq_multicode_probe(
        hess.handle, _ptr(W, np.float32), _ptr(S, np.float32), _ptr(Q, np.uint8),
        _ptr(Z, np.int32), dout, int(bits), int(group), _ptr(qs, np.uint8),
        _ptr(out["moves"], np.int32), _ptr(out["accepted"], np.int32),
        _ptr(out["changed"], np.int32), _ptr(out["dF"], np.float64), _stream(W, S, Q, Z))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_multicode_probe")
    return out


def residual_product(hess: Hessian, W, S, Q, Z, bits: int, out=None):
    """``jarq_residual_product``: H r of every row (float32, dout x din), from
    the split-precision tensor-core kernel behind ``jarq_objective``."""
    dout, din = int(W.shape[0]), int(W.shape[1])
    if out is None:
        if _is_torch(W):
            import torch
            out = torch.empty(dout, din, dtype=torch.float32, device=W.device)
        else:
            out = np.empty((dout, din), dtype=np.float32)
    status = _lib.jarq_residual_product(hess.handle, _ptr(W, np.float32), _ptr(S, np.float32),
                                        _ptr(Q, np.uint8), _ptr(Z, np.int32), dout, int(bits),
                                        _ptr(out, np.float32), _stream(W, S, Q, Z))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_residual_product")
    return out


JARQ_F32, JARQ_F16, JARQ_BF16 = 0, 1, 2


def _dev_stream(*ts):
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream(ts[0].device).cuda_stream)


def canonicalize(S, Q, Z, group_size: int, bits: int):
    """``jarq_canonicalize``: negative scales to the equivalent positive form,
    in place on device tensors (S float32, Q uint8, Z int32)."""
    dout, din = int(Q.shape[0]), int(Q.shape[1])
    status = _lib.jarq_canonicalize(_ptr(S, np.float32), _ptr(Q, np.uint8), _ptr(Z, np.int32),
                                    dout, din, int(group_size), int(bits), _dev_stream(S))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_canonicalize")


def dequantize(S, Q, Z, group_size: int, bits: int, dtype: str = "float16"):
    """``jarq_dequantize``: s (q - z) in float32, float16 or bfloat16 (device tensors)."""
    import torch
    code = {"float32": JARQ_F32, "float16": JARQ_F16, "bfloat16": JARQ_BF16}[dtype]
    tdt = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}[dtype]
    dout, din = int(Q.shape[0]), int(Q.shape[1])
    out = torch.empty(dout, din, dtype=tdt, device=Q.device)
    status = _lib.jarq_dequantize(_ptr(S, np.float32), _ptr(Q, np.uint8), _ptr(Z, np.int32), dout,
                                  din, int(group_size), int(bits), code,
                                  ctypes.c_void_p(out.data_ptr()), _dev_stream(S))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_dequantize")
    return out


def pack_codes(Q, bits: int):
    """``jarq_pack_codes``: b-bit codes packed per row (int32 storage of the
    uint32 words, [dout][ceil(din b / 32)])."""
    import torch
    dout, din = int(Q.shape[0]), int(Q.shape[1])
    nw = (din * int(bits) + 31) // 32
    out = torch.empty(dout, nw, dtype=torch.int32, device=Q.device)
    status = _lib.jarq_pack_codes(_ptr(Q, np.uint8), dout, din, int(bits),
                                  ctypes.c_void_p(out.data_ptr()), _dev_stream(Q))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_pack_codes")
    return out


def accumulate_hessian(X, H=None, scale: float = 1.0):
    """``jarq_accumulate_hessian``: ``H + scale * X^T X`` for a float16 device
    tensor X [tokens][din]; H (float32 [din][din], device) is updated in place
    and returned (a zero matrix when H is None)."""
    import torch
    if not (_is_torch(X) and X.is_cuda and X.dtype == torch.float16 and X.is_contiguous()):
        raise TypeError("X must be a contiguous float16 CUDA tensor [tokens][din]")
    n, d = int(X.shape[0]), int(X.shape[1])
    if H is None:
        H = torch.zeros(d, d, dtype=torch.float32, device=X.device)
    status = _lib.jarq_accumulate_hessian(ctypes.c_void_p(X.data_ptr()), n, d, float(scale),
                                          _ptr(H, np.float32), _dev_stream(X))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_accumulate_hessian")
    return H


def objective(hess: Hessian, W, S, Q, Z, bits: int, out=None):
    """``jarq_objective``: per-row F_j as float64."""
    dout = int(W.shape[0])
    F = out if out is not None else _alloc_like(W, dout, np.float64)
    status = _lib.jarq_objective(hess.handle, _ptr(W, np.float32), _ptr(S, np.float32),
                                 _ptr(Q, np.uint8), _ptr(Z, np.int32), dout, int(bits),
                                 _ptr(F, np.float64), _stream(W, S, Q, Z))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_objective")
    return F


# ---- running and scoring a quantized model: device tensors, enqueued on torch's
# current stream, not waited for.  A call takes a few microseconds on the device,
# so little is done here: every attribute of a tensor is looked at once. ----

class _Torch:
    """What the calls below need of torch, looked up once."""

    def __init__(self):
        import torch
        self.floats = {torch.float32: JARQ_F32, torch.float16: JARQ_F16, torch.bfloat16: JARQ_BF16}
        self.named = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
        self.bytes = {torch.int8: 0}
        self.halves = {torch.float16: JARQ_F16, torch.bfloat16: JARQ_BF16}
        self.empty = torch.empty
        self.f32, self.i32, self.i64, self.i8, self.u8 = (torch.float32, torch.int32, torch.int64, torch.int8,
                                                          torch.uint8)
        # the current stream's handle without an object around it
        self.stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda index: torch.cuda.current_stream(index).cuda_stream)


_torch_cache = None


def _torch() -> _Torch:
    global _torch_cache
    if _torch_cache is None:
        _torch_cache = _Torch()
    return _torch_cache


def _matrix(x, name, types):
    """(pointer, row pitch, rows, columns, type code) of a CUDA matrix whose rows are contiguous."""
    code = types.get(x.dtype)
    shape = x.shape
    if code is None or len(shape) != 2 or not x.is_cuda:
        raise TypeError(f"{name}: expected a CUDA matrix of {' or '.join(str(t) for t in types)}, got {x.dtype} "
                        f"{tuple(shape)} on {x.device}")
    n, d = shape
    pitch, step = x.stride()
    if step != 1 and d > 1:
        raise TypeError(f"{name}: expected contiguous rows, got strides {(pitch, step)}")
    # the pitch of a single row is never used
    return x.data_ptr(), pitch if n > 1 else d, n, d, code


def _flat(x, name, dtype, shape, also=None):
    """Pointer of a contiguous CUDA tensor of the given shape (or the other one)."""
    if x.dtype != dtype or not x.is_cuda or not x.is_contiguous() or (x.shape != shape and x.shape != also):
        raise TypeError(f"{name}: expected a contiguous CUDA tensor of {dtype}, shape {shape}"
                        f"{f' or {also}' if also else ''}, got {x.dtype} {tuple(x.shape)} on {x.device}")
    return x.data_ptr()


def async_status(device=None) -> int:
    """``jarq_async_status`` on torch's current stream: waits for it;
    JARQ_ERR_TIMEOUT if a device wait of an enqueued operator gave up."""
    import torch
    return int(_lib.jarq_async_status(ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)))


def quantize_rows(X):
    """``jarq_quantize_rows``: (codes int8 [n][d], scale float32 [n]) of a
    float32, float16 or bfloat16 matrix, one scale a row.  The rows of the codes
    lie on 16-byte boundaries."""
    T = _torch()
    x, ldx, n, d, code = _matrix(X, "X", T.floats)
    pitch = (d + 15) // 16 * 16
    q = T.empty((n, pitch), dtype=T.i8, device=X.device)
    scale = T.empty((n,), dtype=T.f32, device=X.device)
    status = _lib.jarq_quantize_rows(x, code, n, d, ldx, q.data_ptr(), pitch, scale.data_ptr(),
                                     T.stream(X.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_quantize_rows")
    return q[:, :d], scale


def integer_codes(Q, Z, group_size: int, bits: int):
    """``jarq_integer_codes``: q - z of a refined layer as int8 [dout][din], the
    weights of ``integer_linear`` with the scales S and this group size."""
    T = _torch()
    if len(Q.shape) != 2:
        raise TypeError(f"Q: expected a CUDA matrix of {T.u8}, got {Q.dtype} {tuple(Q.shape)}")
    dout, din = Q.shape
    group_size = int(group_size)
    if group_size <= 0 or din % group_size:
        raise JarqError(JARQ_ERR_ARG, "jarq_integer_codes")
    G = din // group_size
    q = _flat(Q, "Q", T.u8, (dout, din))
    z = _flat(Z, "Z", T.i32, (dout, G), (dout * G,))
    pitch = (din + 15) // 16 * 16
    C = T.empty((dout, pitch), dtype=T.i8, device=Q.device)
    status = _lib.jarq_integer_codes(q, z, dout, din, group_size, int(bits), C.data_ptr(), pitch,
                                     T.stream(Q.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_integer_codes")
    return C[:, :din]


def _integer_layer(T, X, C, ws, group_size, bias, n, din, dtype, out):
    """The arguments that both integer products share, and their output."""
    c, ldc, dout, dc, _ = _matrix(C, "C", T.bytes)
    if dc != din:
        raise ValueError(f"weights have {dc} columns, activations {din}")
    G = din // group_size if group_size else 1
    w = _flat(ws, "ws", T.f32, (dout, G), (dout,) if G == 1 else None)
    b = _flat(bias, "bias", T.f32, (dout,)) if bias is not None else None
    if out is None:
        out = T.empty((n, dout), dtype=dtype, device=X.device)
        return c, ldc, w, b, dout, out, out.data_ptr(), dout
    y, ldy, rows, cols, _ = _matrix(out, "out", {dtype: 0})
    if rows != n or cols != dout:
        raise ValueError(f"out has shape {(rows, cols)}, not {(n, dout)}")
    return c, ldc, w, b, dout, out, y, ldy


def integer_product(X, xs, C, ws, group_size: int = 0, bias=None, dtype: str = "float16", out=None):
    """``jarq_integer_product``: ``xs[t] * sum_i ws[o][i] * (X_i C_i^T) + bias`` for
    int8 codes X [n][din] and C [dout][din], as float32, float16 or bfloat16."""
    T = _torch()
    x, ldx, n, din, _ = _matrix(X, "X", T.bytes)
    ydt = T.named[dtype]
    s = _flat(xs, "xs", T.f32, (n,))
    c, ldc, w, b, dout, out, y, ldy = _integer_layer(T, X, C, ws, group_size, bias, n, din, ydt, out)
    status = _lib.jarq_integer_product(x, ldx, s, c, ldc, w, group_size, b, n, dout, din, T.floats[ydt], y, ldy,
                                       T.stream(X.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_integer_product")
    return out


def integer_linear(X, C, ws, group_size: int = 0, bias=None, dtype: str = None, out=None):
    """``jarq_integer_linear``: the activations X [n][din] (float32, float16 or
    bfloat16) quantized token by token and multiplied with the int8 weights C
    [dout][din]; the result in ``dtype`` (X's own when None)."""
    T = _torch()
    x, ldx, n, din, code = _matrix(X, "X", T.floats)
    ydt = X.dtype if dtype is None else T.named[dtype]
    c, ldc, w, b, dout, out, y, ldy = _integer_layer(T, X, C, ws, group_size, bias, n, din, ydt, out)
    size = _lib.jarq_integer_linear_workspace(n, din)
    work = T.empty((size,), dtype=T.u8, device=X.device)
    status = _lib.jarq_integer_linear(x, code, ldx, c, ldc, w, group_size, b, n, dout, din, T.floats[ydt], y, ldy,
                                      work.data_ptr(), size, T.stream(X.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_integer_linear")
    return out


@dataclass
class TokenScores:
    """Results of ``token_logprobs``, float32 (``top_token`` int32)."""
    logprob: object
    entropy: object
    lse: object
    top_logprob: object
    top_token: object


def token_logprobs(logits, tokens=None, top: int = 0) -> TokenScores:
    """``jarq_token_logprobs``: log probabilities of ``tokens`` (int64 [n] or
    [n][t]) under the rows of ``logits`` [n][vocab], the rows' entropies and log
    sums of exponentials, and their ``top`` most probable tokens."""
    T = _torch()
    x, ld, n, vocab, code = _matrix(logits, "logits", T.floats)
    f32, dev = T.f32, logits.device
    t, tok, logprob, lp = 0, None, None, None
    if tokens is not None:
        shape = tokens.shape
        t = 1 if len(shape) == 1 else shape[-1]
        tok = _flat(tokens, "tokens", T.i64, (n,), (n, t))
        logprob = T.empty(shape, dtype=f32, device=dev)
        lp = logprob.data_ptr()
    entropy, lse = T.empty((n,), dtype=f32, device=dev), T.empty((n,), dtype=f32, device=dev)
    top_logprob, top_token, tl, tt = None, None, None, None
    if top > 0:
        top_logprob, top_token = T.empty((n, top), dtype=f32, device=dev), T.empty((n, top), dtype=T.i32, device=dev)
        tl, tt = top_logprob.data_ptr(), top_token.data_ptr()
    status = _lib.jarq_token_logprobs(x, code, n, vocab, ld, tok, t, top, lp, entropy.data_ptr(), lse.data_ptr(),
                                      tl, tt, T.stream(logits.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_token_logprobs")
    return TokenScores(logprob, entropy, lse, top_logprob, top_token)


def token_logprobs_grad(logits, tokens, lse, g_logprob, entropy=None, g_entropy=None, out=None):
    """``jarq_token_logprobs_grad``: gradient with respect to ``logits`` of
    ``(g_logprob * logprob).sum() + (g_entropy * entropy).sum()``; ``lse`` and
    ``entropy`` are ``token_logprobs``'s.  ``out`` may be ``logits``."""
    T = _torch()
    x, ld, n, vocab, code = _matrix(logits, "logits", T.floats)
    f32, shape = T.f32, tokens.shape
    t = 1 if len(shape) == 1 else shape[-1]
    tok = _flat(tokens, "tokens", T.i64, (n,), (n, t))
    g = _flat(g_logprob, "g_logprob", f32, shape)
    s = _flat(lse, "lse", f32, (n,))
    h = _flat(entropy, "entropy", f32, (n,)) if entropy is not None else None
    gh = _flat(g_entropy, "g_entropy", f32, (n,)) if g_entropy is not None else None
    if out is None:
        out = T.empty((n, vocab), dtype=logits.dtype, device=logits.device)
        dx, ldd = out.data_ptr(), vocab
    else:
        dx, ldd, rows, cols, _ = _matrix(out, "out", {logits.dtype: 0})
        if rows != n or cols != vocab:
            raise ValueError(f"out has shape {(rows, cols)}, not {(n, vocab)}")
    status = _lib.jarq_token_logprobs_grad(x, code, n, vocab, ld, tok, t, s, h, g, gh, dx, ldd,
                                           T.stream(logits.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_token_logprobs_grad")
    return out


@dataclass
class NormedRows:
    """Results of ``rms_norm``; None where not asked for."""
    h: object
    y: object
    codes: object
    scale: object
    rstd: object


def _like(x, name, n, d, dtype):
    """(pointer, row pitch) of a matrix of the shape and type of another one."""
    p, ld, rows, cols, _ = _matrix(x, name, {dtype: 0})
    if rows != n or cols != d:
        raise ValueError(f"{name} has shape {(rows, cols)}, not {(n, d)}")
    return p, ld


def _gain(T, gain, d, dtype, code):
    """(pointer, type code) of the gains of rows of ``dtype``."""
    if gain is None:
        return None, code
    wide = gain.dtype == T.f32
    return _flat(gain, "gain", T.f32 if wide else dtype, (d,)), JARQ_F32 if wide else code


def rms_norm(X, gain=None, eps: float = 1e-6, residual=None, values: bool = True, codes: bool = False,
             h=None) -> NormedRows:
    """``jarq_rms_norm``: the rows ``h = X + residual`` (X itself without one)
    over their root mean square, times ``gain`` [d] (of X's type or float32):
    as ``values`` in X's type and as ``codes`` int8 with a scale a row, the
    arguments of ``integer_product``.  ``h`` receives the sum; it may be
    ``residual``.  The rows of the codes lie on 16-byte boundaries."""
    T = _torch()
    x, ldx, n, d, code = _matrix(X, "X", T.floats)
    dtype, empty = X.dtype, T.empty
    g, gcode = _gain(T, gain, d, dtype, code)
    r = hp = Y = y = Q = q = scale = s = None
    ldr = ldh = ldq = d
    if residual is not None:
        r, ldr = _like(residual, "residual", n, d, dtype)
        if h is None:
            h = empty((n, d), dtype=dtype, device=X.device)
            hp = h.data_ptr()
        else:
            hp, ldh = _like(h, "h", n, d, dtype)
    elif h is not None:
        raise ValueError("h is the sum with a residual: there is none")
    if values:
        Y = empty((n, d), dtype=dtype, device=X.device)
        y = Y.data_ptr()
    if codes:
        ldq = (d + 15) // 16 * 16
        Q = empty((n, ldq), dtype=T.i8, device=X.device)
        scale = empty((n,), dtype=T.f32, device=X.device)
        q, s = Q.data_ptr(), scale.data_ptr()
        if ldq != d:
            Q = Q[:, :d]
    rstd = empty((n,), dtype=T.f32, device=X.device)
    status = _lib.jarq_rms_norm(x, code, n, d, ldx, r, ldr, hp, ldh, g, gcode, eps, y, d, q, ldq, s, rstd.data_ptr(),
                                T.stream(X.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_rms_norm")
    return NormedRows(X if residual is None else h, Y, Q, scale, rstd)


def rms_norm_grad(h, gain, rstd, dy, dh=None, rows: bool = True, gains: bool = True, out=None):
    """``jarq_rms_norm_grad``: (dX, dgain float32 [d]) from the normed rows
    ``h``, the norm's ``rstd`` and the gradient ``dy`` of its values; ``dh`` is
    the gradient that reaches ``h`` by the residual stream.  dX, the gradient of
    X and of the residual alike, goes to ``out``, which may be ``dy`` or ``dh``;
    None in the place of what ``rows`` or ``gains`` does not ask for."""
    T = _torch()
    p, ldh, n, d, code = _matrix(h, "h", T.floats)
    dtype, dev = h.dtype, h.device
    g, gcode = _gain(T, gain, d, dtype, code)
    r = _flat(rstd, "rstd", T.f32, (n,))
    y, ldy = _like(dy, "dy", n, d, dtype)
    s, lds = _like(dh, "dh", n, d, dtype) if dh is not None else (None, d)
    x, ldx, dgain, gp, work, size = None, d, None, None, None, 0
    if rows:
        if out is None:
            out = T.empty((n, d), dtype=dtype, device=dev)
            x = out.data_ptr()
        else:
            x, ldx = _like(out, "out", n, d, dtype)
    elif out is not None:
        raise ValueError("out is dX, which is not asked for")
    if gains:
        dgain = T.empty((d,), dtype=T.f32, device=dev)
        size = _lib.jarq_rms_norm_grad_workspace(n, d)
        if size:
            buffer = T.empty((size,), dtype=T.u8, device=dev)
            work = buffer.data_ptr()
        gp = dgain.data_ptr()
    status = _lib.jarq_rms_norm_grad(p, code, n, d, ldh, g, gcode, r, y, ldy, s, lds, x, ldx, gp, work, size,
                                     T.stream(h.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_rms_norm_grad")
    return out, dgain


def _head(T, X, W, tokens):
    """What the loss of an output head and its gradient share."""
    x, ldx, n, d, code = _matrix(X, "X", T.halves)
    w, ldw, vocab, dw, _ = _matrix(W, "W", {X.dtype: code})
    if dw != d:
        raise ValueError(f"the head has {dw} columns, hidden states {d}")
    tok = _flat(tokens, "tokens", T.i64, (n,))
    aligned = not (x | w) & 15 and (n <= 1 or not ldx & 7) and (vocab <= 1 or not ldw & 7)
    return x, ldx, n, d, code, w, ldw, vocab, tok, 1 if aligned else 0


def cross_entropy(X, W, tokens):
    """``jarq_cross_entropy``: (loss, lse), float32 [n], of ``tokens`` (int64
    [n]; negative ones count for nothing) under the logits ``X W^T`` of hidden
    states X [n][d] and a head W [vocab][d], both float16 or both bfloat16.
    The logits are never in memory."""
    T = _torch()
    x, ldx, n, d, code, w, ldw, vocab, tok, aligned = _head(T, X, W, tokens)
    f32, dev = T.f32, X.device
    loss, lse = T.empty((n,), dtype=f32, device=dev), T.empty((n,), dtype=f32, device=dev)
    size = _lib.jarq_cross_entropy_workspace(n, d, vocab, aligned)
    work = T.empty((size,), dtype=T.u8, device=dev)
    status = _lib.jarq_cross_entropy(x, code, n, d, ldx, w, vocab, ldw, tok, loss.data_ptr(), lse.data_ptr(),
                                     work.data_ptr(), size, T.stream(X.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_cross_entropy")
    return loss, lse


def cross_entropy_grad(X, W, tokens, lse, g_loss, hidden: bool = True, head: bool = True):
    """``jarq_cross_entropy_grad``: (dX, dW), the gradients of ``(g_loss *
    loss).sum()`` with respect to the hidden states and the head, in their type;
    None in the place of one that ``hidden`` or ``head`` does not ask for.
    ``lse`` is ``cross_entropy``'s."""
    T = _torch()
    x, ldx, n, d, code, w, ldw, vocab, tok, aligned = _head(T, X, W, tokens)
    s, g = _flat(lse, "lse", T.f32, (n,)), _flat(g_loss, "g_loss", T.f32, (n,))
    dev, dtype = X.device, X.dtype
    dX = T.empty((n, d), dtype=dtype, device=dev) if hidden else None
    dW = T.empty((vocab, d), dtype=dtype, device=dev) if head else None
    size = _lib.jarq_cross_entropy_grad_workspace(n, d, vocab, aligned, 1 if hidden else 0, 1 if head else 0)
    work = T.empty((size,), dtype=T.u8, device=dev)
    status = _lib.jarq_cross_entropy_grad(x, code, n, d, ldx, w, vocab, ldw, tok, s, g,
                                          dX.data_ptr() if hidden else None, d, dW.data_ptr() if head else None, d,
                                          work.data_ptr(), size, T.stream(X.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_cross_entropy_grad")
    return dX, dW


def apply_adapters(X, A, B, ids, scale=None, base=None, dtype: str = None, out=None):
    """``jarq_apply_adapters``: ``base[t] + scale[i] * B[i] @ (A[i] @ X[t])`` with
    ``i = ids[t]`` (int32 [n]; negative for no adapter), beside a projection
    whose outputs are ``base`` [n][dout].  X [n][din], A [adapters][rank][din]
    and B [adapters][dout][rank] are all float16 or all bfloat16; the result is
    of base's type, X's own or float32 (without one, of ``dtype`` or X's).
    ``out`` may be ``base``."""
    T = _torch()
    x, ldx, n, din, code = _matrix(X, "X", T.halves)
    xdt, dev = X.dtype, X.device
    if len(A.shape) != 3 or len(B.shape) != 3:
        raise TypeError(f"A and B: expected [adapters][rank][din] and [adapters][dout][rank], got {tuple(A.shape)} and "
                        f"{tuple(B.shape)}")
    m, rank, da = A.shape
    dout = B.shape[1]
    if da != din:
        raise ValueError(f"the adapters have {da} columns, activations {din}")
    a, b = _flat(A, "A", xdt, (m, rank, din)), _flat(B, "B", xdt, (m, dout, rank))
    s = _flat(scale, "scale", T.f32, (m,)) if scale is not None else None
    i = _flat(ids, "ids", T.i32, (n,))
    ydt = base.dtype if base is not None else xdt if dtype is None else T.named[dtype]
    if ydt != xdt and ydt != T.f32 or (dtype is not None and ydt != T.named[dtype]):
        raise TypeError(f"expected outputs of {xdt} or {T.f32}, got {ydt}{f' and dtype {dtype}' if dtype else ''}")
    y0, ldy0 = _like(base, "base", n, dout, ydt) if base is not None else (None, dout)
    if out is None:
        out = T.empty((n, dout), dtype=ydt, device=dev)
        y, ldy = out.data_ptr(), dout
    else:
        y, ldy = _like(out, "out", n, dout, ydt)
    size = _lib.jarq_adapters_workspace(n, din, rank, m)
    buffer = T.empty((size,), dtype=T.u8, device=dev) if size else None
    status = _lib.jarq_apply_adapters(x, code, ldx, a, b, s, m, rank, i, n, din, dout, y0, ldy0, y, ldy,
                                      T.floats[ydt], buffer.data_ptr() if size else None, size, T.stream(X.get_device()))
    if status != JARQ_OK:
        raise JarqError(status, "jarq_apply_adapters")
    return out
