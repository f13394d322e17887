"""Python binding of liblogbq (ctypes): argument marshalling only.

Every step of the computation runs in the library: ``fit`` in its host code, ``encode``,
``linear``, ``dequantize`` and a serving step's operators (``batch_tables``, ``tree_tables``,
``linear_adapters``, ``qk_rotate``, ``kv4_append``, ``kv4_append_rotated``, ``kv4_read``, ``kv4_attention``,
``kv4_tree_attention``, ``token_logprobs``) in its gfx950 kernels. PyTorch provides device memory and the
current stream; nothing here computes on the data. If the library is not built, every call
raises ``LogbqUnavailable``: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from contextlib import nullcontext
from ctypes import POINTER, c_double, c_float, c_int32, c_int64, c_uint8, c_uint16, c_void_p
from typing import NamedTuple

import numpy as np

# LOGBQ_LIBRARY selects another build of the library (e.g. a sanitizer build for CPU tests).
LIB_PATH = os.environ.get("LOGBQ_LIBRARY") or \
    os.path.join(os.path.dirname(os.path.abspath(__file__)), "liblogbq.so")

OK, ERR_INVALID_ARG, ERR_NONFINITE, ERR_DEGENERATE, ERR_UNSUPPORTED, ERR_HIP, ERR_HOST_RESOURCE = \
    range(7)


class LogbqUnavailable(RuntimeError):
    pass


class LogbqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_str(status)} (status {status})")


class Params(ctypes.Structure):
    """Mirror of ``logbq_params`` (include/logbq.h)."""
    _fields_ = [
        ("bits", c_int32), ("qmax", c_int32), ("eps", c_double), ("wmin", c_double),
        ("wmax", c_double), ("base", c_double), ("shift", c_int32), ("reserved", c_int32),
        ("wmin_index", c_int64), ("codebook", c_float * 256), ("thresholds", c_float * 128),
    ]

    def codebook_array(self) -> np.ndarray:
        """The 2^bits codebook entries (16 for 4-bit, 256 for 8-bit codes)."""
        return np.ctypeslib.as_array(self.codebook)[: 1 << self.bits].copy()

    def thresholds_array(self) -> np.ndarray:
        """thresholds[0 .. qmax - 1] followed by +inf padding up to 2^(bits-1) entries."""
        return np.ctypeslib.as_array(self.thresholds)[: 1 << (self.bits - 1)].copy()


class Uniform(ctypes.Structure):
    """logbq_uniform: parameters of the asymmetric linear baseline (4-bit)."""
    _fields_ = [("bits", c_int32), ("zero", c_int32), ("wmin", c_double), ("wmax", c_double),
                ("scale", c_double), ("codebook", c_float * 16), ("thresholds", c_float * 15),
                ("reserved", c_float)]

    def codebook_array(self) -> np.ndarray:
        return np.ctypeslib.as_array(self.codebook).copy()

    def thresholds_array(self) -> np.ndarray:
        return np.ctypeslib.as_array(self.thresholds).copy()


class Kv4Struct(ctypes.Structure):
    """Mirror of ``logbq_kv4`` (include/logbq.h)."""
    _fields_ = [("k_codes", c_void_p), ("v_codes", c_void_p), ("k_scales", c_void_p),
                ("v_scales", c_void_p), ("pages", c_int64), ("heads", c_int32), ("page", c_int32),
                ("dim", c_int32), ("reserved", c_int32)]


class RotationStruct(ctypes.Structure):
    """Mirror of ``logbq_rotation`` (include/logbq.h)."""
    _fields_ = [("inv_freq", c_void_p), ("pairs", c_int32), ("interleaved", c_int32), ("factor", c_double)]


_lib = None

SIGNATURES = {
    "logbq_abi_version": (c_int32, []),
    "logbq_status_str": (ctypes.c_char_p, [c_int32]),
    "logbq_fit": (c_int32, [POINTER(c_float), c_int64, c_int32, c_double, POINTER(Params)]),
    "logbq_encode": (c_int32, [c_void_p, c_int64, c_int64, POINTER(Params), c_void_p,
                               POINTER(c_float), c_void_p]),
    "logbq_linear": (c_int32, [c_void_p, c_int64, c_int64, c_void_p, c_int64, POINTER(c_float),
                               c_void_p, c_void_p]),
    "logbq_dequantize": (c_int32, [c_void_p, c_int64, c_int64, POINTER(c_float), c_void_p,
                                   c_void_p]),
    "logbq_linear_multi": (c_int32, [c_void_p, c_int64, c_int64, c_int32, POINTER(c_void_p),
                                     POINTER(c_int64), POINTER(POINTER(c_float)),
                                     POINTER(c_void_p), c_void_p]),
    "logbq_linear8": (c_int32, [c_void_p, c_int64, c_int64, c_void_p, c_int64, POINTER(c_float),
                                c_void_p, c_void_p]),
    "logbq_dequantize8": (c_int32, [c_void_p, c_int64, c_int64, POINTER(c_float), c_void_p,
                                    c_void_p]),
    "logbq_linear_path": (c_int32, [c_int32, c_int64, c_int64, c_int64, POINTER(c_int32)]),
    "logbq_linear_kernel": (c_int32, [c_int32, c_int64, c_int64, c_int64, POINTER(c_float),
                                      ctypes.c_char_p, c_int64]),
    "logbq_fit_uniform": (c_int32, [POINTER(c_float), c_int64, c_int32, POINTER(Uniform)]),
    "logbq_encode_uniform": (c_int32, [c_void_p, c_int64, c_int64, POINTER(Uniform), c_void_p,
                                       c_void_p]),
    "logbq_gptq": (c_int32, [c_void_p, c_int64, c_int64, c_void_p, POINTER(Params),
                             POINTER(Uniform), c_void_p, c_void_p, c_void_p]),
    "logbq_gptq_noalloc": (c_int32, [c_void_p, c_int64, c_int64, c_void_p, POINTER(Params),
                                     POINTER(Uniform), c_void_p, c_void_p]),
    "logbq_fit_device": (c_int32, [c_void_p, c_int64, c_int32, c_double, c_void_p,
                                   POINTER(Params), c_void_p]),
    "logbq_fit_exact": (c_int32, [POINTER(c_float), c_int64, c_int32, c_double, POINTER(Params)]),
    "logbq_batch_tables": (c_int32, [c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                                     c_int64, c_int32, c_int64, c_void_p, c_void_p, c_void_p,
                                     c_void_p, c_void_p, c_void_p]),
    "logbq_kv4_append": (c_int32, [c_void_p, c_int64, c_void_p, c_int64, c_int32, c_int64,
                                   POINTER(Kv4Struct), c_void_p, c_void_p]),
    "logbq_kv4_read": (c_int32, [POINTER(Kv4Struct), c_void_p, c_int64, c_void_p, c_void_p, c_int32,
                                 c_void_p]),
    "logbq_kv4_attention": (c_int32, [c_void_p, c_int64, c_int32, c_int64, c_int32,
                                      POINTER(Kv4Struct), c_void_p, c_int64, c_int64, c_void_p,
                                      c_void_p, c_int64, c_float, c_int32, c_void_p, c_int32,
                                      c_void_p, c_void_p, c_int64, c_void_p]),
    "logbq_tree_tables": (c_int32, [c_void_p, c_int64, c_void_p, c_void_p, c_int64, c_void_p, c_void_p,
                                    c_void_p]),
    "logbq_qk_rotate": (c_int32, [c_void_p, c_int64, c_int32, c_void_p, c_void_p, c_int64, c_int32, c_void_p,
                                  c_int32, c_int64, c_int32, c_double, c_void_p, POINTER(RotationStruct),
                                  c_void_p, c_void_p, c_int32, c_void_p]),
    "logbq_kv4_append_rotated": (c_int32, [c_void_p, c_int64, c_int32, c_void_p, c_void_p, c_int64, c_void_p,
                                           c_void_p, c_int64, c_int32, c_int64, c_double, c_void_p,
                                           POINTER(RotationStruct), POINTER(Kv4Struct), c_void_p, c_void_p,
                                           c_int32, c_void_p]),
    "logbq_kv4_tree_attention": (c_int32, [c_void_p, c_int64, c_int32, c_int64, c_int32,
                                           POINTER(Kv4Struct), c_void_p, c_int64, c_int64, c_void_p,
                                           c_void_p, c_void_p, c_int64, c_float, c_int32, c_void_p, c_int32,
                                           c_void_p, c_void_p, c_int64, c_void_p]),
    "logbq_linear_adapters_workspace": (c_int64, [c_int64, c_int32, c_int32]),
    "logbq_linear_adapters": (c_int32, [c_void_p, c_int64, c_int64, c_int32, POINTER(c_void_p), POINTER(c_void_p),
                                        POINTER(c_int64), c_int32, c_int64, c_int32, c_void_p, c_void_p, c_void_p,
                                        c_void_p, c_int64, c_int64, POINTER(c_void_p), POINTER(c_void_p), c_void_p,
                                        c_int64, c_void_p]),
    "logbq_token_logprobs": (c_int32, [c_void_p, c_int32, c_int64, c_int64, c_int64, c_void_p,
                                       c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                       c_int64, c_void_p]),
}

FIT_WORKSPACE_BYTES = 110600

ABI_VERSION = 2


def lib() -> ctypes.CDLL:
    """The loaded liblogbq.so (raises LogbqUnavailable if it is not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise LogbqUnavailable(
                f"{LIB_PATH} is not built; run __graft_entry__.build() first")
        h = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(h, name)
            fn.restype = res
            fn.argtypes = args
        if h.logbq_abi_version() != ABI_VERSION:
            raise LogbqUnavailable(f"{LIB_PATH} has ABI {h.logbq_abi_version()}, "
                                   f"the binding expects {ABI_VERSION}; rebuild it")
        _lib = h
    return _lib


def status_str(status: int) -> str:
    return lib().logbq_status_str(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise LogbqError(status, where)


_current_stream = None      # set at the first call


def _current_stream_getter():
    """A function that returns the current device's current stream as a number. torch's own raw
    getter takes 0.1 us where building a Stream object takes 2.7 us, as much as a launch."""
    import torch
    raw, device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
    if raw is None or device is None or not torch.cuda.is_initialized():
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


def _stream(stream):
    if stream is None:
        global _current_stream
        if _current_stream is None:
            _current_stream = _current_stream_getter()
        return _current_stream()
    if isinstance(stream, int):
        return c_void_p(stream)
    return c_void_p(stream.cuda_stream)


def _cb_ptr(codebook, entries=16):
    if isinstance(codebook, Params):
        if (1 << codebook.bits) != entries:
            raise ValueError(f"parameters of a {codebook.bits}-bit fit, call needs {entries} entries")
        return codebook.codebook, codebook
    arr = np.ascontiguousarray(np.asarray(codebook, dtype=np.float32))
    if arr.shape != (entries,):
        raise ValueError(f"codebook must hold {entries} float32 values")
    return arr.ctypes.data_as(POINTER(c_float)), arr


def fit(w, bits: int = 4, eps: float = 4e-3) -> Params:
    """logbq_fit on host float32 weights (numpy array or CPU torch tensor)."""
    if hasattr(w, "detach"):
        w = w.detach().cpu().numpy()
    w = np.ascontiguousarray(w, dtype=np.float32)
    p = Params()
    _check(lib().logbq_fit(w.ctypes.data_as(POINTER(c_float)), w.size, bits, eps,
                           ctypes.byref(p)), "logbq_fit")
    return p


def fit_exact(w, bits: int = 4, eps: float = 4e-3) -> Params:
    """logbq_fit_exact on host float32 weights: the device fit's parameters, computed on the host."""
    if hasattr(w, "detach"):
        w = w.detach().cpu().numpy()
    w = np.ascontiguousarray(w, dtype=np.float32)
    p = Params()
    _check(lib().logbq_fit_exact(w.ctypes.data_as(POINTER(c_float)), w.size, bits, eps,
                                 ctypes.byref(p)), "logbq_fit_exact")
    return p


def fit_device(w, bits: int = 4, eps: float = 4e-3, workspace=None, stream=None) -> Params:
    """logbq_fit_device on a contiguous float32 device tensor (Eq. 5 with exact sums). Blocks
    until the fit's passes have run on `stream`."""
    import torch
    if w.dtype != torch.float32 or not w.is_contiguous() or w.device.type != "cuda":
        raise ValueError("w must be a contiguous float32 device tensor")
    if workspace is None:
        workspace = torch.empty(FIT_WORKSPACE_BYTES, dtype=torch.uint8, device=w.device)
    elif workspace.numel() * workspace.element_size() < FIT_WORKSPACE_BYTES:
        raise ValueError(f"workspace must hold {FIT_WORKSPACE_BYTES} bytes")
    p = Params()
    _check(lib().logbq_fit_device(c_void_p(w.data_ptr()), w.numel(), bits, eps,
                                  c_void_p(workspace.data_ptr()), ctypes.byref(p),
                                  _stream(stream)), "logbq_fit_device")
    return p


def encode(w, p: Params, out=None, stream=None):
    """logbq_encode: float32 [N][K] device tensor -> (uint8 codes, float32 codebook).

    Codes are [N][K/2] for a 4-bit fit, [N][K] for an 8-bit one; the codebook has 2^bits
    entries."""
    import torch
    if w.dtype != torch.float32 or w.dim() != 2 or not w.is_contiguous():
        raise ValueError("w must be a contiguous 2-D float32 device tensor")
    n, k = w.shape
    if out is None:
        cols = k // 2 if p.bits == 4 else k
        out = torch.empty((n, cols), dtype=torch.uint8, device=w.device)
    cb = np.zeros(1 << p.bits, dtype=np.float32)
    _check(lib().logbq_encode(c_void_p(w.data_ptr()), n, k, ctypes.byref(p),
                              c_void_p(out.data_ptr()), cb.ctypes.data_as(POINTER(c_float)),
                              _stream(stream)), "logbq_encode")
    return out, cb


def linear(x, codes, codebook, out=None, stream=None):
    """logbq_linear: y[M][N] = x[M][K] . W_hat^T (x float16, y float32) on packed codes."""
    import torch
    if x.dtype != torch.float16 or x.dim() != 2 or not x.is_contiguous():
        raise ValueError("x must be a contiguous 2-D float16 device tensor")
    if codes.dtype != torch.uint8 or codes.dim() != 2 or not codes.is_contiguous():
        raise ValueError("codes must be a contiguous 2-D uint8 device tensor")
    m, k = x.shape
    n = codes.shape[0]
    if codes.shape[1] * 2 != k:
        raise ValueError("codes must be [N][K/2]")
    if out is None:
        out = torch.empty((m, n), dtype=torch.float32, device=x.device)
    cbp, _keep = _cb_ptr(codebook)
    _check(lib().logbq_linear(c_void_p(x.data_ptr()), m, k, c_void_p(codes.data_ptr()), n, cbp,
                              c_void_p(out.data_ptr()), _stream(stream)), "logbq_linear")
    return out


def linear_multi(x, codes_list, codebooks, outs=None, stream=None):
    """logbq_linear_multi: y_i = x . W_hat_i^T for up to 4 linears sharing x (one launch)."""
    import torch
    if x.dtype != torch.float16 or x.dim() != 2 or not x.is_contiguous():
        raise ValueError("x must be a contiguous 2-D float16 device tensor")
    m, k = x.shape
    count = len(codes_list)
    if not 1 <= count <= 4 or len(codebooks) != count:
        raise ValueError("need 1..4 linears with one codebook each")
    for c in codes_list:
        if c.dtype != torch.uint8 or c.dim() != 2 or not c.is_contiguous() or c.shape[1] * 2 != k:
            raise ValueError("codes must be contiguous uint8 [N][K/2] device tensors")
    if outs is None:
        outs = [torch.empty((m, c.shape[0]), dtype=torch.float32, device=x.device)
                for c in codes_list]
    keep = [_cb_ptr(cb) for cb in codebooks]
    cptr = (c_void_p * count)(*[c.data_ptr() for c in codes_list])
    ns = (c_int64 * count)(*[c.shape[0] for c in codes_list])
    cbs = (POINTER(c_float) * count)(*[p for p, _ in keep])
    ys = (c_void_p * count)(*[y.data_ptr() for y in outs])
    _check(lib().logbq_linear_multi(c_void_p(x.data_ptr()), m, k, count, cptr, ns, cbs, ys,
                                    _stream(stream)), "logbq_linear_multi")
    return outs


def dequantize(codes, codebook, out=None, stream=None):
    """logbq_dequantize: uint8 [N][K/2] -> float32 [N][K], bit-exact codebook lookup."""
    import torch
    if codes.dtype != torch.uint8 or codes.dim() != 2 or not codes.is_contiguous():
        raise ValueError("codes must be a contiguous 2-D uint8 device tensor")
    n, h = codes.shape
    k = 2 * h
    if out is None:
        out = torch.empty((n, k), dtype=torch.float32, device=codes.device)
    cbp, _keep = _cb_ptr(codebook)
    _check(lib().logbq_dequantize(c_void_p(codes.data_ptr()), n, k, cbp, c_void_p(out.data_ptr()),
                                  _stream(stream)), "logbq_dequantize")
    return out


def linear8(x, codes, codebook, out=None, stream=None):
    """logbq_linear8: y[M][N] = x[M][K] . W_hat^T on 8-bit codes [N][K] (x float16, y float32)."""
    import torch
    if x.dtype != torch.float16 or x.dim() != 2 or not x.is_contiguous():
        raise ValueError("x must be a contiguous 2-D float16 device tensor")
    if codes.dtype != torch.uint8 or codes.dim() != 2 or not codes.is_contiguous():
        raise ValueError("codes must be a contiguous 2-D uint8 device tensor")
    m, k = x.shape
    n = codes.shape[0]
    if codes.shape[1] != k:
        raise ValueError("8-bit codes must be [N][K]")
    if out is None:
        out = torch.empty((m, n), dtype=torch.float32, device=x.device)
    cbp, _keep = _cb_ptr(codebook, 256)
    _check(lib().logbq_linear8(c_void_p(x.data_ptr()), m, k, c_void_p(codes.data_ptr()), n, cbp,
                               c_void_p(out.data_ptr()), _stream(stream)), "logbq_linear8")
    return out


def dequantize8(codes, codebook, out=None, stream=None):
    """logbq_dequantize8: uint8 [N][K] 8-bit codes -> float32 [N][K], bit-exact lookup."""
    import torch
    if codes.dtype != torch.uint8 or codes.dim() != 2 or not codes.is_contiguous():
        raise ValueError("codes must be a contiguous 2-D uint8 device tensor")
    n, k = codes.shape
    if out is None:
        out = torch.empty((n, k), dtype=torch.float32, device=codes.device)
    cbp, _keep = _cb_ptr(codebook, 256)
    _check(lib().logbq_dequantize8(c_void_p(codes.data_ptr()), n, k, cbp, c_void_p(out.data_ptr()),
                                   _stream(stream)), "logbq_dequantize8")
    return out


PATH_NAMES = {0: "none", 1: "gemv", 2: "mfma", 3: "splitk", 4: "mfma_kq", 5: "mfma_pf"}


def linear_path(bits: int, m: int, k: int, n: int) -> str:
    """logbq_linear_path: name of the kernel ("none", "gemv", "mfma", "splitk", "mfma_kq" or
    "mfma_pf") that linear (bits 4) or linear8 (bits 8) runs for an [m][k] x [n][k] call with a
    fitted codebook. Host only."""
    out = c_int32(0)
    _check(lib().logbq_linear_path(int(bits), int(m), int(k), int(n), ctypes.byref(out)),
           "logbq_linear_path")
    return PATH_NAMES[out.value]


def linear_kernel(bits: int, m: int, k: int, n: int, codebook=None) -> str:
    """logbq_linear_kernel: the kernel instance (e.g. "k_gemv<4, 1, 4, false, 2>") that the first
    launch of a linear / linear8 call of that shape runs; codebook None stands for a fitted
    (sign-symmetric) one. Host only."""
    buf = ctypes.create_string_buffer(96)
    cb = None
    if codebook is not None:
        arr = np.ascontiguousarray(getattr(codebook, "codebook_array", lambda: codebook)(),
                                   dtype=np.float32)
        if arr.size != 1 << bits:
            raise ValueError(f"codebook of {arr.size} entries for {bits}-bit codes")
        cb = arr.ctypes.data_as(POINTER(c_float))
    _check(lib().logbq_linear_kernel(int(bits), int(m), int(k), int(n), cb, buf, len(buf)),
           "logbq_linear_kernel")
    return buf.value.decode()


def fit_uniform(w, bits: int = 4) -> Uniform:
    """logbq_fit_uniform on host float32 weights (numpy array or CPU torch tensor)."""
    if hasattr(w, "detach"):
        w = w.detach().cpu().numpy()
    w = np.ascontiguousarray(w, dtype=np.float32)
    u = Uniform()
    _check(lib().logbq_fit_uniform(w.ctypes.data_as(POINTER(c_float)), w.size, bits,
                                   ctypes.byref(u)), "logbq_fit_uniform")
    return u


def encode_uniform(w, u: Uniform, out=None, stream=None):
    """logbq_encode_uniform: float32 [N][K] device tensor -> packed uint8 [N][K/2] codes."""
    import torch
    if w.dtype != torch.float32 or w.dim() != 2 or not w.is_contiguous():
        raise ValueError("w must be a contiguous 2-D float32 device tensor")
    n, k = w.shape
    if out is None:
        out = torch.empty((n, k // 2), dtype=torch.uint8, device=w.device)
    _check(lib().logbq_encode_uniform(c_void_p(w.data_ptr()), n, k, ctypes.byref(u),
                                      c_void_p(out.data_ptr()), _stream(stream)),
           "logbq_encode_uniform")
    return out


GPTQ_BLOCK = 128


def gptq(w, u, params, out_codes=None, workspace=None, stream=None):
    """logbq_gptq: GPTQ calibration of the float32 [N][K] device tensor `w` (updated in place to
    the error-compensated weights) with the upper factor `u` ([K][K] float32 device tensor of
    the damped inverse Hessian) and a fixed codebook: `params` is a Params (LogbQuant, from
    fit) or a Uniform (the asymmetric linear baseline, from fit_uniform). Returns packed uint8
    [N][K/2] codes."""
    import torch
    if w.dtype != torch.float32 or w.dim() != 2 or not w.is_contiguous():
        raise ValueError("w must be a contiguous 2-D float32 device tensor")
    n, k = w.shape
    if u.dtype != torch.float32 or tuple(u.shape) != (k, k) or not u.is_contiguous():
        raise ValueError("u must be a contiguous [K][K] float32 device tensor")
    if out_codes is None:
        out_codes = torch.empty((n, k // 2), dtype=torch.uint8, device=w.device)
    if workspace is None:
        workspace = torch.empty((n, GPTQ_BLOCK), dtype=torch.float32, device=w.device)
    pp = ctypes.byref(params) if isinstance(params, Params) else None
    up = ctypes.byref(params) if isinstance(params, Uniform) else None
    if pp is None and up is None:
        raise ValueError("params must be a Params or a Uniform")
    _check(lib().logbq_gptq(c_void_p(w.data_ptr()), n, k, c_void_p(u.data_ptr()), pp, up,
                            c_void_p(workspace.data_ptr()), c_void_p(out_codes.data_ptr()),
                            _stream(stream)), "logbq_gptq")
    return out_codes


# ------------------------------------------------------------------ a serving step's operators

KV4_WORKSPACE_BYTES = 1 << 28
LOGPROBS_WORKSPACE_BYTES = 1 << 22
LOGPROBS_MAX_TOP = 32


class Kv4Cache(NamedTuple):
    """The buffers of one layer's 4-bit key/value cache (``logbq_kv4`` in include/logbq.h); any
    4-tuple of such tensors serves as well."""
    k_codes: object       # uint8 [pages][heads][page][dim/2]
    k_scales: object      # bfloat16 [pages][heads][page]
    v_codes: object       # uint8 [pages][heads][page/8][16][8][dim/32]
    v_scales: object      # bfloat16 [pages][heads][page]


def kv4_cache(pages: int, heads: int, dim: int, page: int = 64, device="cuda") -> Kv4Cache:
    """An empty (zeroed) cache of `pages` pages of `page` tokens."""
    import torch
    if dim not in (64, 128, 256) or page not in (16, 32, 64, 128, 256, 512, 1024):
        raise ValueError("dim must be 64, 128 or 256; page a power of two, 16 to 1024")
    u8 = dict(dtype=torch.uint8, device=device)
    bf = dict(dtype=torch.bfloat16, device=device)
    return Kv4Cache(torch.zeros((pages, heads, page, dim // 2), **u8),
                    torch.zeros((pages, heads, page), **bf),
                    torch.zeros((pages, heads, page // 8, 16, 8, dim // 32), **u8),
                    torch.zeros((pages, heads, page), **bf))


_dtype_codes = None


def _dtype_code(dtype) -> int:
    """logbq_dtype of a torch type."""
    global _dtype_codes
    if _dtype_codes is None:
        import torch
        _dtype_codes = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
    try:
        return _dtype_codes[dtype]
    except KeyError:
        raise ValueError(f"{dtype} is none of float32, float16, bfloat16") from None


def _device_array(x, dtype, shape, name):
    """Raises unless x is a contiguous device tensor of a type and shape."""
    if x.dtype != dtype or x.shape != shape or not x.is_contiguous() or not x.is_cuda:
        raise ValueError(f"{name} must be a contiguous {tuple(shape)} {dtype} device tensor, not "
                         f"{tuple(x.shape)} {x.dtype} on {x.device}")


def _device_workspace(x):
    """Raises unless x is a contiguous device tensor; the calls check its size."""
    if not (x.is_cuda and x.is_contiguous()):
        raise ValueError(f"workspace must be a contiguous device tensor, not {tuple(x.shape)} on {x.device}")


def _kv4_struct(cache) -> Kv4Struct:
    import torch
    kc, ks, vc, vs = cache
    if kc.dim() != 4:
        raise ValueError("k_codes must be [pages][heads][page][dim/2]")
    shape = kc.shape
    pages, heads, page, half = shape
    values, scales = (pages, heads, page // 8, 16, 8, half // 16), (pages, heads, page)
    u8, bf16 = torch.uint8, torch.bfloat16
    if not (vc.shape == values and ks.shape == scales and vs.shape == scales and kc.is_cuda and vc.is_cuda
            and ks.is_cuda and vs.is_cuda and kc.dtype == vc.dtype == u8 and ks.dtype == vs.dtype == bf16
            and kc.is_contiguous() and vc.is_contiguous() and ks.is_contiguous()
            and vs.is_contiguous()):
        for x, dtype, s, name in ((kc, u8, shape, "k_codes"), (vc, u8, values, "v_codes"),
                                  (ks, bf16, scales, "k_scales"), (vs, bf16, scales, "v_scales")):
            _device_array(x, dtype, s, name)
    return Kv4Struct(kc.data_ptr(), vc.data_ptr(), ks.data_ptr(), vs.data_ptr(), pages, heads, page,
                     2 * half, 0)


_as_it_is = nullcontext()


def _made_on(stream):
    """A context whose new tensors belong to the stream that a call is given: memory that the
    current stream still uses is not handed out, and what is filled is filled in order."""
    if stream is None:
        return _as_it_is
    import torch
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


def _rows(x, heads, dim, name):
    """Elements between the tokens of x [tokens][heads][dim], whose heads and channels are
    contiguous."""
    shape = x.shape
    if len(shape) != 3 or not x.is_cuda or shape[2] != dim or (heads and shape[1] != heads):
        raise ValueError(f"{name} must be a [tokens][{heads or 'heads'}][{dim}] device tensor")
    stride = x.stride()
    if stride[2] != 1 or (stride[1] != dim and shape[1] != 1):
        raise ValueError(f"the heads and channels of {name} must be contiguous")
    # One token has no distance to the next; its stride may be anything.
    return stride[0] if shape[0] > 1 else shape[1] * dim


def batch_tables(cached, new, free_pages, table, page: int, tokens: int, out=None, stream=None):
    """logbq_batch_tables: slot map, positions and starts of a step, and the block table's new
    entries, from the requests' lengths (int32 device tensors `cached` and `new`). `free_pages`
    (int32) gives new pages from its front; `table` (int32 [requests][width]) is updated in place.
    Returns a dict of slots (int64 [tokens]), positions (int32 [tokens]), q_starts (int32
    [requests + 1]), seq_lens (int32 [requests]) and info (int32 [4]: new tokens, pages taken,
    longest length, 1 pages short + 2 table too narrow + 4 `tokens` too few); `out` may hold the
    tensors to write."""
    import torch
    i32 = torch.int32
    n = cached.numel()
    _device_array(cached, i32, (n,), "cached")
    _device_array(new, i32, (n,), "new")
    _device_array(free_pages, i32, (free_pages.numel(),), "free_pages")
    if table.dim() != 2:
        raise ValueError("table must be [requests][width]")
    width = table.shape[1]
    _device_array(table, i32, (n, width), "table")
    if out is None:
        e = dict(device=cached.device, dtype=i32)
        with _made_on(stream):
            out = dict(slots=torch.empty(tokens, device=cached.device, dtype=torch.int64),
                       positions=torch.empty(tokens, **e), q_starts=torch.empty(n + 1, **e),
                       seq_lens=torch.empty(n, **e), info=torch.empty(4, **e))
    else:
        _device_array(out["slots"], torch.int64, (tokens,), "slots")
        _device_array(out["positions"], i32, (tokens,), "positions")
        _device_array(out["q_starts"], i32, (n + 1,), "q_starts")
        _device_array(out["seq_lens"], i32, (n,), "seq_lens")
        _device_array(out["info"], i32, (4,), "info")
    _check(lib().logbq_batch_tables(
        cached.data_ptr(), new.data_ptr(), n, free_pages.data_ptr(), free_pages.numel(),
        table.data_ptr(), width, page, tokens, out["slots"].data_ptr(), out["positions"].data_ptr(),
        out["q_starts"].data_ptr(), out["seq_lens"].data_ptr(), out["info"].data_ptr(),
        _stream(stream)), "logbq_batch_tables")
    return out


def tree_tables(parents, q_starts, seq_lens, out=None, stream=None):
    """logbq_tree_tables: ancestor masks and positions of drafted trees. `parents` (int32 [tokens]) has each
    node's parent as an index among its request's tokens (negative: the last cached token); `q_starts` (int32
    [requests + 1]) and `seq_lens` (int32 [requests]) are batch_tables' results. Returns a dict of masks (int64
    [tokens], 64 bits each) and positions (int32 [tokens]); `out` may hold the tensors to write."""
    import torch
    i32 = torch.int32
    tokens, n = parents.numel(), seq_lens.numel()
    _device_array(parents, i32, (tokens,), "parents")
    _device_array(q_starts, i32, (n + 1,), "q_starts")
    _device_array(seq_lens, i32, (n,), "seq_lens")
    if out is None:
        with _made_on(stream):
            out = dict(masks=torch.empty(tokens, device=parents.device, dtype=torch.int64),
                       positions=torch.empty(tokens, device=parents.device, dtype=i32))
    else:
        _device_array(out["masks"], torch.int64, (tokens,), "masks")
        _device_array(out["positions"], i32, (tokens,), "positions")
    _check(lib().logbq_tree_tables(parents.data_ptr(), tokens, q_starts.data_ptr(), seq_lens.data_ptr(), n,
                                   out["masks"].data_ptr(), out["positions"].data_ptr(), _stream(stream)),
           "logbq_tree_tables")
    return out


class Rotation(NamedTuple):
    """How queries and keys are turned by their positions (``logbq_rotation`` in include/logbq.h): the first
    2 * len(inv_freq) channels of a head, as halves or as interleaved pairs."""
    inv_freq: object              # float32 device tensor
    interleaved: bool = False
    factor: float = 1.0


def _rotation_struct(rotation, f32) -> RotationStruct:
    inv_freq, interleaved, factor = rotation
    pairs = inv_freq.numel()
    _device_array(inv_freq, f32, (pairs,), "inv_freq")
    return RotationStruct(inv_freq.data_ptr() or None, pairs, 1 if interleaved else 0, factor)


def _weight(x, f32, dim, name):
    if x is None:
        return None
    _device_array(x, f32, (dim,), name)
    return x.data_ptr()


def _rotated_out(x, out, like, stream, name):
    """The tensor that takes x's rotated rows: `out`, checked, or a new one of type `like`; its type."""
    if out is None:
        import torch
        with _made_on(stream):
            return torch.empty_like(x, dtype=like, memory_format=torch.contiguous_format), like
    dtype = out.dtype
    _device_array(out, dtype, x.shape, name)
    return out, dtype


def qk_rotate(q, k, positions, rotation, q_weight=None, k_weight=None, eps: float = 1e-6, q_out=None,
              k_out=None, stream=None):
    """logbq_qk_rotate: queries and keys [tokens][heads][dim] (float32, float16 or bfloat16; the tokens may be
    strided), each head normed with `q_weight` / `k_weight` (float32 [dim]; None: no norm) and turned by
    `positions` (int32 [tokens]) as a Rotation says. `k` may be None. Returns (q_out, k_out), contiguous, of the
    inputs' type unless given; an output may be its own (contiguous) input."""
    import torch
    shape, dtype, f32 = q.shape, q.dtype, torch.float32
    dim = shape[-1] if len(shape) == 3 else 0
    q_stride = _rows(q, 0, dim, "q")
    tokens = shape[0]
    _device_array(positions, torch.int32, (tokens,), "positions")
    q_out, out_dtype = _rotated_out(q, q_out, dtype, stream, "q_out")
    k_stride = k_heads = k_at = k_out_at = 0
    if k is not None:
        k_stride = _rows(k, 0, dim, "k")
        k_tokens, k_heads, _ = k.shape
        if k.dtype != dtype or k_tokens != tokens:
            raise ValueError("q and k must have one type and number of tokens")
        k_out, k_out_dtype = _rotated_out(k, k_out, out_dtype, stream, "k_out")
        if k_out_dtype != out_dtype:
            raise ValueError("q_out and k_out must have one type")
        k_at, k_out_at = k.data_ptr(), k_out.data_ptr()
    r = _rotation_struct(rotation, f32)
    _check(lib().logbq_qk_rotate(
        q.data_ptr(), q_stride, shape[1], _weight(q_weight, f32, dim, "q_weight"), k_at or None, k_stride, k_heads,
        _weight(k_weight, f32, dim, "k_weight"), _dtype_code(dtype), tokens, dim, eps, positions.data_ptr(),
        ctypes.byref(r), q_out.data_ptr(), k_out_at or None, _dtype_code(out_dtype), _stream(stream)),
        "logbq_qk_rotate")
    return q_out, k_out


def kv4_append_rotated(q, k, v, cache, slots, positions, rotation, q_weight=None, k_weight=None,
                       eps: float = 1e-6, q_out=None, stream=None):
    """logbq_kv4_append_rotated: keys normed and turned as in qk_rotate on their way into `slots` (int64 [tokens])
    of a Kv4Cache, with the values, and the queries turned beside them. `q` may be None. Returns q_out
    ([tokens][q_heads][dim], float16 unless given; None without queries)."""
    import torch
    c = _kv4_struct(cache)
    dim, f32, dtype, out_dtype = c.dim, torch.float32, k.dtype, torch.float16
    k_stride, v_stride = _rows(k, c.heads, dim, "k"), _rows(v, c.heads, dim, "v")
    tokens = k.shape[0]
    if v.dtype != dtype or v.shape[0] != tokens:
        raise ValueError("k and v must have one type and number of tokens")
    _device_array(slots, torch.int64, (tokens,), "slots")
    _device_array(positions, torch.int32, (tokens,), "positions")
    q_stride = q_heads = q_at = q_out_at = 0
    if q is not None:
        q_stride = _rows(q, 0, dim, "q")
        q_tokens, q_heads, _ = q.shape
        if q.dtype != dtype or q_tokens != tokens:
            raise ValueError("q and k must have one type and number of tokens")
        q_out, out_dtype = _rotated_out(q, q_out, out_dtype, stream, "q_out")
        q_at, q_out_at = q.data_ptr(), q_out.data_ptr()
    r = _rotation_struct(rotation, f32)
    _check(lib().logbq_kv4_append_rotated(
        q_at or None, q_stride, q_heads, _weight(q_weight, f32, dim, "q_weight"), k.data_ptr(), k_stride,
        _weight(k_weight, f32, dim, "k_weight"), v.data_ptr(), v_stride, _dtype_code(dtype), tokens, eps,
        positions.data_ptr(), ctypes.byref(r), ctypes.byref(c), slots.data_ptr(), q_out_at or None,
        _dtype_code(out_dtype), _stream(stream)), "logbq_kv4_append_rotated")
    return None if q is None else q_out


def kv4_append(k, v, cache, slots, stream=None):
    """logbq_kv4_append: keys and values [tokens][heads][dim] (float32, float16 or bfloat16; the
    tokens may be strided) quantized into `slots` (int64 [tokens]; negative: left out; what a slot
    holds that two tokens name is not specified) of a Kv4Cache."""
    import torch
    c = _kv4_struct(cache)
    k_stride, v_stride = _rows(k, c.heads, c.dim, "k"), _rows(v, c.heads, c.dim, "v")
    if v.dtype != k.dtype or v.shape[0] != k.shape[0]:
        raise ValueError("k and v must have one type and number of tokens")
    _device_array(slots, torch.int64, (k.shape[0],), "slots")
    _check(lib().logbq_kv4_append(k.data_ptr(), k_stride, v.data_ptr(), v_stride,
                                  _dtype_code(k.dtype), k.shape[0], ctypes.byref(c),
                                  slots.data_ptr(), _stream(stream)), "logbq_kv4_append")


def kv4_read(cache, slots, dtype=None, stream=None):
    """logbq_kv4_read: (k, v), each [tokens][heads][dim] of `dtype` (float16 unless given), the
    values that a Kv4Cache holds in `slots` (zeros for a slot outside it)."""
    import torch
    c = _kv4_struct(cache)
    _device_array(slots, torch.int64, (slots.numel(),), "slots")
    shape = (slots.numel(), c.heads, c.dim)
    with _made_on(stream):
        k = slots.new_empty(shape, dtype=dtype or torch.float16)
        v = torch.empty_like(k)
    _check(lib().logbq_kv4_read(ctypes.byref(c), slots.data_ptr(), shape[0], k.data_ptr(),
                                v.data_ptr(), _dtype_code(k.dtype), _stream(stream)),
           "logbq_kv4_read")
    return k, v


def _attention_call(q, cache, table, seq_lens, q_starts, out, lse, workspace, stream):
    """The arguments that the attention calls share, checked: (cache, those before max_new, those after the
    window, out, the workspace, which the caller holds until the call is made)."""
    import torch
    c = _kv4_struct(cache)
    q_stride = _rows(q, 0, c.dim, "q")
    tokens, q_heads = q.shape[0], q.shape[1]
    if table.dim() != 2:
        raise ValueError("table must be [requests][width]")
    n, width = table.shape
    i32 = torch.int32
    _device_array(table, i32, (n, width), "table")
    _device_array(seq_lens, i32, (n,), "seq_lens")
    _device_array(q_starts, i32, (n + 1,), "q_starts")
    if out is None:
        with _made_on(stream):
            out = torch.empty_like(q, dtype=torch.float16, memory_format=torch.contiguous_format)
    else:
        _device_array(out, out.dtype, (tokens, q_heads, c.dim), "out")
    if lse is not None:
        _device_array(lse, torch.float32, (tokens, q_heads), "lse")
    if workspace is None:
        with _made_on(stream):
            workspace = q.new_empty(KV4_WORKSPACE_BYTES, dtype=torch.uint8)
    else:
        _device_workspace(workspace)
    before = (q.data_ptr(), q_stride, _dtype_code(q.dtype), tokens, q_heads, ctypes.byref(c), table.data_ptr(), n,
              width, seq_lens.data_ptr(), q_starts.data_ptr())
    after = (out.data_ptr(), _dtype_code(out.dtype), None if lse is None else lse.data_ptr(), workspace.data_ptr(),
             workspace.numel() * workspace.element_size())
    return c, before, after, out, workspace


def kv4_attention(q, cache, table, seq_lens, q_starts, max_new: int, scale=None, window: int = 0,
                  out=None, lse=None, workspace=None, stream=None):
    """logbq_kv4_attention: attention of q [tokens][q_heads][dim] (float32, float16 or bfloat16;
    the tokens may be strided) over a Kv4Cache. `table` (int32 [requests][width]), `seq_lens`
    (int32 [requests]) and `q_starts` (int32 [requests + 1]) are batch_tables' results; `max_new`
    bounds a request's tokens. `scale` is dim ** -0.5 unless given; `window` 0 sees everything.
    Returns `out` ([tokens][q_heads][dim], float16 unless given); `lse` (float32
    [tokens][q_heads]), if given, receives the log sums of exponentials. `workspace`
    (KV4_WORKSPACE_BYTES bytes serve any call) is allocated if not given."""
    c, before, after, out, _held = _attention_call(q, cache, table, seq_lens, q_starts, out, lse, workspace, stream)
    _check(lib().logbq_kv4_attention(*before, max_new, c.dim ** -0.5 if scale is None else scale, window, *after,
                                     _stream(stream)), "logbq_kv4_attention")
    return out


def kv4_tree_attention(q, cache, table, seq_lens, q_starts, masks, max_new: int, scale=None, window: int = 0,
                       out=None, lse=None, workspace=None, stream=None):
    """logbq_kv4_tree_attention: kv4_attention of a step whose new tokens are the nodes of drafted trees, each of
    which sees its request's cached tokens and the nodes of its mask. `masks` (int64 [tokens]) is tree_tables'
    result; `max_new` is at most 64; `window` is 0 or at least 64."""
    import torch
    _device_array(masks, torch.int64, (q.shape[0],), "masks")
    c, before, after, out, _held = _attention_call(q, cache, table, seq_lens, q_starts, out, lse, workspace, stream)
    _check(lib().logbq_kv4_tree_attention(*before, masks.data_ptr(), max_new,
                                          c.dim ** -0.5 if scale is None else scale, window, *after,
                                          _stream(stream)), "logbq_kv4_tree_attention")
    return out


# ctypes arrays of up to four pointers and sizes; making the types takes longer than filling them.
_ARRAYS = [(c_void_p * n, c_int64 * n) for n in range(5)]


def linear_adapters_workspace_bytes(tokens: int, count: int, rank: int) -> int:
    """logbq_linear_adapters_workspace: bytes of workspace of a linear_adapters call with `tokens` tokens, `count`
    projections and pools of `rank` ranks. Host only."""
    return lib().logbq_linear_adapters_workspace(tokens, count, rank)


def linear_adapters(x, ys, a_list, b_list, q_starts, adapter, max_new: int, scales=None, ranks=None, outs=None,
                    workspace=None, stream=None):
    """logbq_linear_adapters: low-rank adapters of many requests beside up to four projections that share x
    (float16 [tokens][K]): outs[i][t] = ys[i][t] + scales[a] (x[t] A_i[a]^T) B_i[a]^T. `ys` are linear's or
    linear_multi's results (float32 [tokens][N_i]), updated in place unless `outs` is given; `a_list[i]` is a pool
    [adapters][rank][K] and `b_list[i]` [adapters][N_i][rank], float16 or bfloat16. `adapter` (int32 [requests])
    has each request's adapter (negative: none), `q_starts` its first token, `max_new` bounds its tokens. `scales`
    (float32 [adapters]) and `ranks` (int32 [adapters], how many of the pool's ranks an adapter has) may be None.
    `workspace` (linear_adapters_workspace_bytes, one for each stream) is allocated if not given."""
    import torch
    if x.dtype != torch.float16 or x.dim() != 2 or not x.is_contiguous() or not x.is_cuda:
        raise ValueError("x must be a contiguous 2-D float16 device tensor")
    tokens, k = x.shape
    count = len(ys)
    if not 1 <= count <= 4 or len(a_list) != count or len(b_list) != count or \
            (outs is not None and len(outs) != count):
        raise ValueError("need 1..4 projections with a pool of A and one of B each")
    outs = ys if outs is None else outs
    if a_list[0].dim() != 3:
        raise ValueError("a_list must hold [adapters][rank][K] tensors")
    shape, dtype, f32 = a_list[0].shape, a_list[0].dtype, torch.float32
    adapters, rank, _ = shape
    widths = []
    for y, a, b, out in zip(ys, a_list, b_list, outs):
        if y.dim() != 2:
            raise ValueError("ys must hold [tokens][N] tensors")
        n = y.shape[1]
        widths.append(n)
        if not (y.shape[0] == tokens and out.shape == y.shape and a.shape == shape and shape[2] == k and
                b.shape == (adapters, n, rank) and y.dtype == out.dtype == f32 and a.dtype == b.dtype == dtype and
                y.is_cuda and out.is_cuda and a.is_cuda and b.is_cuda and y.is_contiguous() and
                out.is_contiguous() and a.is_contiguous() and b.is_contiguous()):
            _device_array(y, f32, (tokens, n), "ys")
            _device_array(out, f32, (tokens, n), "outs")
            _device_array(a, dtype, (adapters, rank, k), "a_list")
            _device_array(b, dtype, (adapters, n, rank), "b_list")
    requests = adapter.numel()
    _device_array(adapter, torch.int32, (requests,), "adapter")
    _device_array(q_starts, torch.int32, (requests + 1,), "q_starts")
    if scales is not None:
        _device_array(scales, torch.float32, (adapters,), "scales")
    if ranks is not None:
        _device_array(ranks, torch.int32, (adapters,), "ranks")
    if workspace is None:
        with _made_on(stream):
            workspace = x.new_empty(linear_adapters_workspace_bytes(tokens, count, rank), dtype=torch.uint8)
    else:
        _device_workspace(workspace)
    pointers, sizes = _ARRAYS[count]
    _check(lib().logbq_linear_adapters(
        x.data_ptr(), tokens, k, count, pointers(*[a.data_ptr() for a in a_list]),
        pointers(*[b.data_ptr() for b in b_list]), sizes(*widths),
        _dtype_code(dtype), adapters, rank, None if ranks is None else ranks.data_ptr(),
        None if scales is None else scales.data_ptr(), q_starts.data_ptr(), adapter.data_ptr(), requests, max_new,
        pointers(*[y.data_ptr() for y in ys]), pointers(*[o.data_ptr() for o in outs]), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream(stream)), "logbq_linear_adapters")
    return outs


def token_logprobs(logits, targets, top: int = 0, out=None, workspace=None, stream=None):
    """logbq_token_logprobs: of each row of logits [tokens][vocab] (float32, float16 or bfloat16;
    the rows may be strided) the log probability of its target (int64 [tokens]; outside the
    vocabulary: 0), the entropy, and the `top` (up to 32) likeliest tokens. Returns a dict of
    logprob and entropy (float32 [tokens]), top_index (int32) and top_logprob (float32, both
    [tokens][top]); `out` may hold the tensors to write. `workspace` (LOGPROBS_WORKSPACE_BYTES
    bytes, zeroed once by the caller, one for each stream) is allocated and zeroed if not given."""
    import torch
    if logits.dim() != 2 or not logits.is_cuda or (logits.stride(1) != 1 and logits.shape[1] != 1):
        raise ValueError("logits must be a [tokens][vocab] device tensor with contiguous rows")
    tokens, vocab = logits.shape
    _device_array(targets, torch.int64, (tokens,), "targets")
    if out is None:
        f = dict(dtype=torch.float32, device=logits.device)
        with _made_on(stream):
            out = dict(logprob=torch.empty(tokens, **f), entropy=torch.empty(tokens, **f),
                       top_index=torch.empty((tokens, top), dtype=torch.int32, device=logits.device),
                       top_logprob=torch.empty((tokens, top), **f))
    else:
        _device_array(out["logprob"], torch.float32, (tokens,), "logprob")
        _device_array(out["entropy"], torch.float32, (tokens,), "entropy")
        _device_array(out["top_index"], torch.int32, (tokens, top), "top_index")
        _device_array(out["top_logprob"], torch.float32, (tokens, top), "top_logprob")
    if workspace is None:
        with _made_on(stream):
            workspace = torch.zeros(LOGPROBS_WORKSPACE_BYTES, dtype=torch.uint8, device=logits.device)
    else:
        _device_workspace(workspace)
    _check(lib().logbq_token_logprobs(
        logits.data_ptr(), _dtype_code(logits.dtype), tokens, vocab,
        logits.stride(0) if tokens > 1 else vocab, targets.data_ptr(), top,
        out["logprob"].data_ptr(), out["entropy"].data_ptr(), out["top_index"].data_ptr(),
        out["top_logprob"].data_ptr(), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream(stream)), "logbq_token_logprobs")
    return out
