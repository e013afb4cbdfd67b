"""ctypes binding of the C ABI in ``include/bnn.h``; same names, same argument order.

Only marshalling happens here: shapes and strides are read off the tensors,
outputs are allocated with torch on the inputs' device, and the call is
enqueued on torch's current stream.  No arithmetic of the method is done in
Python, and nothing falls back to the CPU.

Calls that bring their output take a native path first (``_calls``, csrc/python_calls.cpp), which reads the tensors
and launches without ctypes; whatever it does not take comes back as -1 and goes through the wrapper below it, whose
checks then say what is wrong.  Where it does not load, a warning says so and all calls go through the wrappers.
"""
from __future__ import annotations

import ctypes
import os
import warnings

import numpy as np
import torch
from torch.autograd.function import once_differentiable

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libbnn_hip.so")

POOL_APART, POOL_IN_CONV, POOL_WINDOWS = range(3)
(KERNEL_AUTO, KERNEL_NAIVE, KERNEL_TILED128, KERNEL_KSPLIT, KERNEL_TILED64, KERNEL_MFMA, KERNEL_MFMA128,
 KERNEL_MFMA_SHORTK, KERNEL_MFMA_PERSIST, KERNEL_MFMA_BIG, KERNEL_MFMA_SPLITK) = range(11)

ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU, ACT_GELU_TANH, ACT_SIGMOID = range(6)
NORM_NONE, NORM_RMS, NORM_LAYER = range(3)
_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}         # bnn_type

_i64 = ctypes.c_int64
_int = ctypes.c_int
_ptr = ctypes.c_void_p
_f32 = ctypes.c_float

_SIGNATURES = {
    "bnn_version": (_int, []),
    "bnn_status_string": (ctypes.c_char_p, [_int]),
    "bnn_words_per_row": (_i64, [_i64]),
    "bnn_pack_sign": (_int, [_ptr, _i64, _i64, _i64, _ptr, _i64, _ptr]),
    "bnn_xnor_gemm": (_int, [_ptr, _i64, _ptr, _i64, _ptr, _i64, _i64, _i64, _i64, _ptr]),
    "bnn_xnor_gemm_kernel": (_int, [_ptr, _i64, _ptr, _i64, _ptr, _i64, _i64, _i64, _i64, _int, _ptr]),
    "bnn_xnor_gemm_bn_sign_pack": (_int, [_ptr, _i64, _ptr, _i64, _i64, _i64, _i64, _ptr, _ptr, _ptr, _i64, _ptr]),
    "bnn_xnor_gemm_bn_sign_pack_kernel": (_int, [_ptr, _i64, _ptr, _i64, _i64, _i64, _i64, _ptr, _ptr, _ptr, _i64,
                                                 _int, _ptr]),
    "bnn_sign_gemm_bn_sign_pack": (_int, [_ptr, _i64, _ptr, _i64, _i64, _i64, _i64, _ptr, _ptr, _ptr, _i64, _ptr, _i64,
                                          _ptr]),
    "bnn_pack_bitplanes": (_int, [_ptr, _i64, _i64, _i64, _ptr, _i64, _ptr]),
    "bnn_bitplane_gemm": (_int, [_ptr, _i64, _ptr, _i64, _ptr, _i64, _i64, _i64, _i64, _ptr]),
    "bnn_bitplane_gemm_bn_sign_pack": (_int, [_ptr, _i64, _ptr, _i64, _i64, _i64, _i64, _ptr, _ptr, _ptr, _i64, _ptr]),
    "bnn_bn_fold": (_int, [_ptr, _ptr, _ptr, _ptr, _f32, _i64, _i64, _ptr, _ptr]),
    "bnn_bn_sign_pack": (_int, [_ptr, _i64, _i64, _i64, _ptr, _ptr, _ptr, _i64, _ptr]),
    "bnn_conv_im2col_pack": (_int, [_ptr, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _ptr, _i64, _ptr]),
    "bnn_conv_xnor": (_int, [_ptr, _i64, _i64, _i64, _i64, _ptr, _i64, _i64, _int, _int, _int, _int, _ptr, _i64, _ptr]),
    "bnn_conv_bn_sign_pack": (_int, [_ptr, _i64, _i64, _i64, _i64, _ptr, _i64, _i64, _int, _int, _int, _int, _ptr,
                                     _ptr, _ptr, _i64, _ptr]),
    "bnn_conv_pool_bn_sign_pack": (_int, [_ptr, _i64, _i64, _i64, _i64, _ptr, _i64, _i64, _int, _int, _int, _int, _int,
                                          _ptr, _ptr, _ptr, _i64, _ptr]),
    "bnn_conv_pool_windows_bn_sign_pack": (_int, [_ptr, _i64, _i64, _i64, _i64, _ptr, _i64, _i64, _int, _int, _int, _int, _int,
                                                  _ptr, _ptr, _ptr, _i64, _ptr]),
    "bnn_conv_pool_form": (_int, [_i64, _i64, _i64, _i64, _i64, _int, _int, _int, _int, _int]),
    "bnn_maxpool_bits": (_int, [_ptr, _i64, _i64, _i64, _i64, _int, _int, _int, _ptr, _ptr, _ptr]),
    "bnn_gemm_i8_mfma": (_int, [_ptr, _i64, _ptr, _i64, _ptr, _i64, _i64, _i64, _i64, _ptr]),
    "bnn_unpack_i8": (_int, [_ptr, _i64, _i64, _i64, _ptr, _i64, _ptr]),
    "bnn_linear_bits": (_int, [_int, _ptr, _i64, _ptr, _i64, _ptr, _ptr, _int, _ptr, _i64, _ptr, _i64, _i64, _i64, _i64, _ptr]),
    "bnn_gated_bits": (_int, [_int, _ptr, _i64, _ptr, _i64, _ptr, _ptr, _int, _ptr, _i64, _i64, _i64, _i64, _ptr]),
    "bnn_linear_bits_backward_workspace": (_i64, [_int, _i64, _i64, _i64, _int]),
    "bnn_linear_bits_backward": (_int, [_int, _ptr, _i64, _ptr, _i64, _ptr, _i64, _ptr, _ptr, _int, _ptr, _i64, _ptr, _i64,
                                        _ptr, _ptr, _i64, _i64, _i64, _ptr, _i64, _ptr]),
    "bnn_gated_bits_backward_workspace": (_i64, [_int, _i64, _i64, _i64, _int]),
    "bnn_gated_bits_backward": (_int, [_int, _ptr, _i64, _ptr, _i64, _ptr, _i64, _ptr, _ptr, _int, _ptr, _i64, _ptr, _i64,
                                       _ptr, _ptr, _i64, _i64, _i64, _ptr, _i64, _ptr]),
    "bnn_norm_residual": (_int, [_int, _ptr, _i64, _ptr, _i64, _ptr, _i64, _i64, _f32, _int, _ptr, _ptr, _int, _ptr, _ptr, _f32,
                                 _ptr, _i64, _ptr, _i64, _i64, _i64, _ptr]),
    "bnn_norm_residual_backward_workspace": (_i64, [_i64, _i64, _i64]),
    "bnn_norm_residual_backward": (_int, [_int, _ptr, _i64, _ptr, _i64, _ptr, _i64, _ptr, _i64, _ptr, _i64, _i64, _f32, _int,
                                          _ptr, _ptr, _int, _ptr, _f32, _ptr, _i64, _ptr, _i64, _ptr, _i64, _ptr, _ptr, _ptr,
                                          _ptr, _i64, _i64, _ptr, _i64, _ptr]),
}

_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

_lib = None
_calls = None            # the native path, bound when the library is loaded


class BnnError(RuntimeError):
    def __init__(self, fn: str, status: int):
        msg = load_library().bnn_status_string(status).decode()
        super().__init__(f"{fn} failed with status {status} ({msg})")
        self.status = status


def lib_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libbnn_hip.so (built in-tree by ``build.build_library``).  Raises if absent."""
    global _lib, _calls
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(
                f"{_LIB_PATH} is not built; run `python -m paper_1602_02830_amd.build` "
                "(there is no CPU fallback)")
        lib = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        if _raw_stream is not None:
            try:
                from . import _calls as calls
                calls.bind({name: ctypes.cast(getattr(lib, name), _ptr).value for name in _SIGNATURES}, _raw_stream)
                _calls = calls
            except ImportError as e:           # absent, or built against another torch: the wrappers below are complete
                warnings.warn(f"calls go through ctypes, the native call path does not load ({e}); "
                              "`python -m paper_1602_02830_amd.build` builds it", RuntimeWarning, stacklevel=2)
        _lib = lib
    return _lib


def exported_symbols():
    return sorted(_SIGNATURES)


def _check(fn: str, status: int):
    if status != 0:
        raise BnnError(fn, status)


def _took(fn: str, status: int) -> bool:
    """Whether the native path took the call (and launched it): False for -1, raises for a status of the library."""
    if status > 0:
        raise BnnError(fn, status)
    return status == 0


def _stream(t: torch.Tensor):
    """torch's current stream on the device of `t`, as the ABI's `void* stream`."""
    if _raw_stream is not None:            # the handle itself, without building a Stream object
        return _raw_stream(t.device.index)
    return torch.cuda.current_stream(t.device).cuda_stream


def _dev(t: torch.Tensor, dtype, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be 2-D with unit stride along its rows")
    return t


def _ld(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _holds(t: torch.Tensor, rows: int, cols: int, name: str):
    """`t` has the [rows][cols] elements a call reads or writes.  The library sees a pointer and a leading dimension:
    one that is too short it refuses itself, but too few rows, or a narrow slice of a wide buffer, only show here."""
    if rows > 0 and 0 < cols <= _ld(t) and (t.shape[0] < rows or t.shape[1] < cols):
        raise ValueError(f"{name} must hold [{rows}][{cols}] elements, got {list(t.shape)}")


def version() -> int:
    return int(load_library().bnn_version())


def words_per_row(K: int) -> int:
    """bnn_words_per_row: 32-bit words of a packed row of K values (the layout rule of the ABI, restated
    here so that the wrappers do not pay a foreign call for it; a host test compares the two)."""
    K = int(K)
    return -1 if K < 0 else (K + 31) // 32


def _alloc_words(rows: int, kw: int, device, ld: int | None = None) -> torch.Tensor:
    ld = kw if ld is None else ld
    if ld < kw:
        raise ValueError("ld smaller than the packed row")
    if ld == kw:
        return torch.empty((rows, kw), dtype=torch.int32, device=device)
    # Words between the packed row and ld are never written by the library: define them.
    return torch.zeros((rows, ld), dtype=torch.int32, device=device)[:, :kw]


def pack_sign(x: torch.Tensor, out: torch.Tensor | None = None, ld_out: int | None = None) -> torch.Tensor:
    """bnn_pack_sign: float32 [rows][cols] -> packed int32 words [rows][ceil(cols/32)]."""
    if out is not None and _calls is not None:
        st = _calls.pack_sign(x, out)
        if st == 0 or _took("bnn_pack_sign", st):
            return out
    lib = load_library()
    _dev(x, torch.float32, "x")
    rows, cols = x.shape
    kw = words_per_row(cols)
    if out is None:
        out = _alloc_words(rows, kw, x.device, ld_out)
    _dev(out, torch.int32, "out")
    _holds(out, rows, kw, "out")
    _check("bnn_pack_sign", lib.bnn_pack_sign(x.data_ptr(), rows, cols, _ld(x), out.data_ptr(), _ld(out),
                                             _stream(out)))
    return out


def xnor_gemm(A: torch.Tensor, B: torch.Tensor, K: int, out: torch.Tensor | None = None,
              kernel: int = KERNEL_AUTO) -> torch.Tensor:
    """bnn_xnor_gemm: packed A [M][Kw], packed B [N][Kw] -> int32 C [M][N]."""
    if out is not None and _calls is not None:
        st = _calls.xnor_gemm(A, B, K, out, kernel)
        if st == 0 or _took("bnn_xnor_gemm", st):
            return out
    lib = load_library()
    _dev(A, torch.int32, "A")
    _dev(B, torch.int32, "B")
    M, N = A.shape[0], B.shape[0]
    kw = words_per_row(K)
    if A.shape[1] < kw or B.shape[1] < kw:
        raise ValueError("packed operands have fewer words per row than K needs")
    if out is None:
        out = torch.empty((M, N), dtype=torch.int32, device=A.device)
    _dev(out, torch.int32, "out")
    _holds(out, M, N, "out")
    if kernel == KERNEL_AUTO:
        st = lib.bnn_xnor_gemm(A.data_ptr(), _ld(A), B.data_ptr(), _ld(B), out.data_ptr(), _ld(out), M, N, K,
                               _stream(out))
    else:
        st = lib.bnn_xnor_gemm_kernel(A.data_ptr(), _ld(A), B.data_ptr(), _ld(B), out.data_ptr(), _ld(out),
                                      M, N, K, kernel, _stream(out))
    _check("bnn_xnor_gemm", st)
    return out


def bn_fold(gamma, beta, mean, var, eps: float, K: int):
    """bnn_bn_fold (host): float32 arrays [N] -> (thr int32 [N], flip_bits uint32 [ceil(N/32)]) numpy."""
    lib = load_library()
    arrs = [np.ascontiguousarray(a, dtype=np.float32) for a in (gamma, beta, mean, var)]
    N = arrs[0].shape[0]
    for a in arrs:
        if a.shape != (N,):
            raise ValueError("BatchNorm parameter arrays must all be [N]")
    thr = np.empty(N, np.int32)
    flip = np.empty((N + 31) // 32, np.uint32)
    st = lib.bnn_bn_fold(*(a.ctypes.data for a in arrs), eps, N, K, thr.ctypes.data, flip.ctypes.data)
    _check("bnn_bn_fold", st)
    return thr, flip


def bn_sign_pack(C: torch.Tensor, thr: torch.Tensor, flip_bits: torch.Tensor,
                 out: torch.Tensor | None = None, ld_out: int | None = None) -> torch.Tensor:
    """bnn_bn_sign_pack: int32 C [M][N] + folded thresholds -> packed bits [M][ceil(N/32)]."""
    if out is not None and _calls is not None:
        st = _calls.bn_sign_pack(C, thr, flip_bits, out)
        if st == 0 or _took("bnn_bn_sign_pack", st):
            return out
    lib = load_library()
    _dev(C, torch.int32, "C")
    M, N = C.shape
    nw = words_per_row(N)
    if thr.dtype != torch.int32 or flip_bits.dtype != torch.int32 or not thr.is_cuda or not flip_bits.is_cuda:
        raise ValueError("thr and flip_bits must be int32 device tensors")
    if thr.numel() != N or flip_bits.numel() != nw or not thr.is_contiguous() or not flip_bits.is_contiguous():
        raise ValueError("thr must be [N] and flip_bits [ceil(N/32)], contiguous")
    if out is None:
        out = _alloc_words(M, nw, C.device, ld_out)
    _dev(out, torch.int32, "out")
    _holds(out, M, nw, "out")
    _check("bnn_bn_sign_pack", lib.bnn_bn_sign_pack(C.data_ptr(), _ld(C), M, N, thr.data_ptr(),
                                                   flip_bits.data_ptr(), out.data_ptr(), _ld(out), _stream(out)))
    return out


def _layer(A: torch.Tensor, B: torch.Tensor, K: int, thr: torch.Tensor, flip_bits: torch.Tensor):
    """Packed rows of at least K bits, and the thresholds and flip bits of B's rows."""
    N, kw = B.shape[0], words_per_row(K)
    if A.shape[1] < kw or B.shape[1] < kw:
        raise ValueError("packed operands have fewer words per row than K needs")
    if thr.dtype != torch.int32 or flip_bits.dtype != torch.int32 or not thr.is_cuda or not flip_bits.is_cuda:
        raise ValueError("thr and flip_bits must be int32 device tensors")
    if thr.numel() != N or flip_bits.numel() != words_per_row(N) or not thr.is_contiguous() or not flip_bits.is_contiguous():
        raise ValueError("thr must be [N] and flip_bits [ceil(N/32)], contiguous")


def xnor_gemm_bn_sign_pack(A: torch.Tensor, B: torch.Tensor, K: int, thr: torch.Tensor, flip_bits: torch.Tensor,
                           out: torch.Tensor | None = None, ld_out: int | None = None,
                           kernel: int = KERNEL_AUTO) -> torch.Tensor:
    """bnn_xnor_gemm_bn_sign_pack: packed A [M][Kw], packed B [N][Kw], thresholds -> packed bits [M][ceil(N/32)]."""
    if out is not None and _calls is not None:
        st = _calls.xnor_gemm_bn_sign_pack(A, B, K, thr, flip_bits, out, kernel)
        if st == 0 or _took("bnn_xnor_gemm_bn_sign_pack", st):
            return out
    lib = load_library()
    _dev(A, torch.int32, "A")
    _dev(B, torch.int32, "B")
    M, N = A.shape[0], B.shape[0]
    nw = words_per_row(N)
    _layer(A, B, K, thr, flip_bits)
    if out is None:
        out = _alloc_words(M, nw, A.device, ld_out)
    _dev(out, torch.int32, "out")
    _holds(out, M, nw, "out")
    if kernel == KERNEL_AUTO:
        st = lib.bnn_xnor_gemm_bn_sign_pack(A.data_ptr(), _ld(A), B.data_ptr(), _ld(B), M, N, K, thr.data_ptr(),
                                            flip_bits.data_ptr(), out.data_ptr(), _ld(out), _stream(out))
    else:
        st = lib.bnn_xnor_gemm_bn_sign_pack_kernel(A.data_ptr(), _ld(A), B.data_ptr(), _ld(B), M, N, K,
                                                   thr.data_ptr(), flip_bits.data_ptr(), out.data_ptr(),
                                                   _ld(out), kernel, _stream(out))
    _check("bnn_xnor_gemm_bn_sign_pack", st)
    return out


def sign_gemm_bn_sign_pack(x: torch.Tensor, B: torch.Tensor, K: int, thr: torch.Tensor, flip_bits: torch.Tensor,
                           a_bits: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
    """pack_sign(x, out=a_bits), then xnor_gemm_bn_sign_pack(a_bits, B, K, thr, flip_bits, out=out): one launch where the
    library has one for these sizes (bnn_sign_gemm_bn_sign_pack)."""
    if _calls is not None:
        st = _calls.sign_gemm_bn_sign_pack(x, B, K, thr, flip_bits, a_bits, out)
        if st == 0 or _took("bnn_sign_gemm_bn_sign_pack", st):
            return out
    if out is None or tuple(x.shape) != (a_bits.shape[0], K):             # other rows than the product's: no one call
        pack_sign(x, out=a_bits)
        return xnor_gemm_bn_sign_pack(a_bits, B, K, thr, flip_bits, out=out)
    lib = load_library()
    for t, dtype, name in ((x, torch.float32, "x"), (B, torch.int32, "B"), (a_bits, torch.int32, "a_bits"), (out, torch.int32, "out")):
        _dev(t, dtype, name)
    M, N = x.shape[0], B.shape[0]
    _layer(a_bits, B, K, thr, flip_bits)
    _holds(out, M, words_per_row(N), "out")
    _check("bnn_sign_gemm_bn_sign_pack",
           lib.bnn_sign_gemm_bn_sign_pack(x.data_ptr(), _ld(x), B.data_ptr(), _ld(B), M, N, K, thr.data_ptr(), flip_bits.data_ptr(),
                                          a_bits.data_ptr(), _ld(a_bits), out.data_ptr(), _ld(out), _stream(out)))
    return out


def pack_bitplanes(x: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_pack_bitplanes: uint8 [rows][cols] -> packed planes int32 [rows][8*ceil(cols/32)] (word 8*w + p)."""
    if out is not None and _calls is not None:
        st = _calls.pack_bitplanes(x, out)
        if st == 0 or _took("bnn_pack_bitplanes", st):
            return out
    lib = load_library()
    _dev(x, torch.uint8, "x")
    rows, cols = x.shape
    kw8 = 8 * words_per_row(cols)
    if out is None:
        out = torch.empty((rows, kw8), dtype=torch.int32, device=x.device)
    _dev(out, torch.int32, "out")
    _holds(out, rows, kw8, "out")
    _check("bnn_pack_bitplanes", lib.bnn_pack_bitplanes(x.data_ptr(), rows, cols, _ld(x), out.data_ptr(), _ld(out),
                                                       _stream(out)))
    return out


def bitplane_gemm(Xp: torch.Tensor, B: torch.Tensor, K: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_bitplane_gemm: bit planes Xp [M][8*Kw], packed +-1 rows B [N][Kw] -> int32 [M][N] = x @ w^T."""
    if out is not None and _calls is not None:
        st = _calls.bitplane_gemm(Xp, B, K, out)
        if st == 0 or _took("bnn_bitplane_gemm", st):
            return out
    lib = load_library()
    _dev(Xp, torch.int32, "Xp")
    _dev(B, torch.int32, "B")
    M, N = Xp.shape[0], B.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.int32, device=Xp.device)
    _dev(out, torch.int32, "out")
    _holds(Xp, M if N else 0, 8 * words_per_row(K), "Xp")
    _holds(B, N if M else 0, words_per_row(K), "B")
    _holds(out, M, N, "out")
    _check("bnn_bitplane_gemm", lib.bnn_bitplane_gemm(Xp.data_ptr(), _ld(Xp), B.data_ptr(), _ld(B), out.data_ptr(),
                                                     _ld(out), M, N, K, _stream(out)))
    return out


def bitplane_gemm_bn_sign_pack(Xp: torch.Tensor, B: torch.Tensor, K: int, thr: torch.Tensor, flip_bits: torch.Tensor,
                               out: torch.Tensor | None = None, ld_out: int | None = None) -> torch.Tensor:
    """bnn_bitplane_gemm_bn_sign_pack: first layer on 8-bit inputs, fused with Sign(BatchNorm)."""
    if out is not None and _calls is not None:
        st = _calls.bitplane_gemm_bn_sign_pack(Xp, B, K, thr, flip_bits, out)
        if st == 0 or _took("bnn_bitplane_gemm_bn_sign_pack", st):
            return out
    lib = load_library()
    _dev(Xp, torch.int32, "Xp")
    _dev(B, torch.int32, "B")
    M, N = Xp.shape[0], B.shape[0]
    nw = words_per_row(N)
    if thr.dtype != torch.int32 or flip_bits.dtype != torch.int32 or not thr.is_cuda or not flip_bits.is_cuda:
        raise ValueError("thr and flip_bits must be int32 device tensors")
    if thr.numel() != N or flip_bits.numel() != nw or not thr.is_contiguous() or not flip_bits.is_contiguous():
        raise ValueError("thr must be [N] and flip_bits [ceil(N/32)], contiguous")
    if out is None:
        out = _alloc_words(M, nw, Xp.device, ld_out)
    _dev(out, torch.int32, "out")
    _holds(Xp, M if N else 0, 8 * words_per_row(K), "Xp")
    _holds(B, N if M else 0, words_per_row(K), "B")
    _holds(out, M, nw, "out")
    _check("bnn_bitplane_gemm_bn_sign_pack",
           lib.bnn_bitplane_gemm_bn_sign_pack(Xp.data_ptr(), _ld(Xp), B.data_ptr(), _ld(B), M, N, K,
                                              thr.data_ptr(), flip_bits.data_ptr(), out.data_ptr(), _ld(out),
                                              _stream(out)))
    return out


def conv_im2col_pack(x_bits: torch.Tensor, Cin: int, kh: int = 3, kw: int = 3, stride: int = 1, pad: int = 1,
                     out: torch.Tensor | None = None, ld_out: int | None = None) -> torch.Tensor:
    """bnn_conv_im2col_pack: packed NHWC int32 [B][H][W][ceil(Cin/32)] -> [B*Ho*Wo][ceil(kh*kw*Cin/32)]."""
    if out is not None and _calls is not None:
        st = _calls.conv_im2col_pack(x_bits, Cin, kh, kw, stride, pad, out)
        if st == 0 or _took("bnn_conv_im2col_pack", st):
            return out
    lib = load_library()
    if not x_bits.is_cuda or x_bits.dtype != torch.int32 or x_bits.dim() != 4 or not x_bits.is_contiguous():
        raise ValueError("x_bits must be a contiguous int32 device tensor [B][H][W][ceil(Cin/32)]")
    B, H, W, Cw = x_bits.shape
    if Cw != words_per_row(Cin):
        raise ValueError("last dimension does not match Cin")
    Ho = (H + 2 * pad - kh) // stride + 1
    Wo = (W + 2 * pad - kw) // stride + 1
    kwords = words_per_row(kh * kw * Cin)
    if out is None:
        out = _alloc_words(B * max(Ho, 0) * max(Wo, 0), kwords, x_bits.device, ld_out)
    _dev(out, torch.int32, "out")
    _holds(out, B * max(Ho, 0) * max(Wo, 0), kwords, "out")
    _check("bnn_conv_im2col_pack",
           lib.bnn_conv_im2col_pack(x_bits.data_ptr(), B, H, W, Cin, kh, kw, stride, pad, out.data_ptr(),
                                    _ld(out), _stream(out)))
    return out


def _check_nhwc_bits(x_bits: torch.Tensor, Cin: int):
    if not x_bits.is_cuda or x_bits.dtype != torch.int32 or x_bits.dim() != 4 or not x_bits.is_contiguous():
        raise ValueError("x_bits must be a contiguous int32 device tensor [B][H][W][ceil(Cin/32)]")
    if x_bits.shape[3] != words_per_row(Cin):
        raise ValueError("last dimension does not match the channel count")


def conv_xnor(x_bits: torch.Tensor, Cin: int, w_bits: torch.Tensor, kh: int = 3, kw: int = 3, stride: int = 1,
              pad: int = 1, out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_conv_xnor: packed NHWC input, packed filters [Cout][kh*kw*Cin/32] -> int32 [B*Ho*Wo][Cout]."""
    if out is not None and _calls is not None:
        st = _calls.conv_xnor(x_bits, Cin, w_bits, kh, kw, stride, pad, out)
        if st == 0 or _took("bnn_conv_xnor", st):
            return out
    lib = load_library()
    _check_nhwc_bits(x_bits, Cin)
    _dev(w_bits, torch.int32, "w_bits")
    B, H, W, _ = x_bits.shape
    Cout = w_bits.shape[0]
    Ho, Wo = (H + 2 * pad - kh) // stride + 1, (W + 2 * pad - kw) // stride + 1
    if out is None:
        out = torch.empty((B * Ho * Wo, Cout), dtype=torch.int32, device=x_bits.device)
    _dev(out, torch.int32, "out")
    M = B * max(Ho, 0) * max(Wo, 0)
    _holds(w_bits, Cout if M else 0, words_per_row(kh * kw * Cin), "w_bits")
    _holds(out, M, Cout, "out")
    _check("bnn_conv_xnor", lib.bnn_conv_xnor(x_bits.data_ptr(), B, H, W, Cin, w_bits.data_ptr(), _ld(w_bits), Cout,
                                             kh, kw, stride, pad, out.data_ptr(), _ld(out), _stream(out)))
    return out


def conv_bn_sign_pack(x_bits: torch.Tensor, Cin: int, w_bits: torch.Tensor, thr: torch.Tensor,
                      flip_bits: torch.Tensor, kh: int = 3, kw: int = 3, stride: int = 1, pad: int = 1,
                      out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_conv_bn_sign_pack: binary conv + Sign(BatchNorm) -> packed bits [B*Ho*Wo][ceil(Cout/32)]."""
    if out is not None and _calls is not None:
        st = _calls.conv_bn_sign_pack(x_bits, Cin, w_bits, kh, kw, stride, pad, thr, flip_bits, out)
        if st == 0 or _took("bnn_conv_bn_sign_pack", st):
            return out
    lib = load_library()
    _check_nhwc_bits(x_bits, Cin)
    _dev(w_bits, torch.int32, "w_bits")
    B, H, W, _ = x_bits.shape
    Cout = w_bits.shape[0]
    Ho, Wo = (H + 2 * pad - kh) // stride + 1, (W + 2 * pad - kw) // stride + 1
    nw = words_per_row(Cout)
    if thr.dtype != torch.int32 or flip_bits.dtype != torch.int32 or not thr.is_cuda or not flip_bits.is_cuda:
        raise ValueError("thr and flip_bits must be int32 device tensors")
    if thr.numel() != Cout or flip_bits.numel() != nw or not thr.is_contiguous() or not flip_bits.is_contiguous():
        raise ValueError("thr must be [Cout] and flip_bits [ceil(Cout/32)], contiguous")
    if out is None:
        out = torch.empty((B * Ho * Wo, nw), dtype=torch.int32, device=x_bits.device)
    _dev(out, torch.int32, "out")
    M = B * max(Ho, 0) * max(Wo, 0)
    _holds(w_bits, Cout if M else 0, words_per_row(kh * kw * Cin), "w_bits")
    _holds(out, M, nw, "out")
    _check("bnn_conv_bn_sign_pack",
           lib.bnn_conv_bn_sign_pack(x_bits.data_ptr(), B, H, W, Cin, w_bits.data_ptr(), _ld(w_bits), Cout, kh, kw,
                                     stride, pad, thr.data_ptr(), flip_bits.data_ptr(), out.data_ptr(), _ld(out),
                                     _stream(out)))
    return out


def conv_pool_bn_sign_pack(x_bits: torch.Tensor, Cin: int, w_bits: torch.Tensor, thr: torch.Tensor,
                           flip_bits: torch.Tensor, kh: int = 3, kw: int = 3, stride: int = 1, pad: int = 1,
                           pool: int = 2, out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_conv_pool_bn_sign_pack: binary conv + max pooling + Sign(BatchNorm) in one launch ->
    packed bits [B*(Ho/pool)*(Wo/pool)][ceil(Cout/32)].  Raises BnnError with status 3 (unsupported)
    for geometries the fused kernel does not take."""
    return _conv_pool("conv_pool_bn_sign_pack", x_bits, Cin, w_bits, thr, flip_bits, kh, kw, stride, pad, pool, out)


def conv_pool_windows_bn_sign_pack(x_bits: torch.Tensor, Cin: int, w_bits: torch.Tensor, thr: torch.Tensor,
                                   flip_bits: torch.Tensor, kh: int = 3, kw: int = 3, stride: int = 1, pad: int = 1,
                                   pool: int = 2, out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_conv_pool_windows_bn_sign_pack: the same on any even map (Cin % 128 == 0)."""
    return _conv_pool("conv_pool_windows_bn_sign_pack", x_bits, Cin, w_bits, thr, flip_bits, kh, kw, stride, pad, pool, out)


def conv_pool_form(B: int, H: int, W: int, Cin: int, Cout: int, kh: int = 3, kw: int = 3, stride: int = 1, pad: int = 1,
                   pool: int = 2) -> int:
    """bnn_conv_pool_form: the fastest form of a pooled layer, POOL_IN_CONV (conv_pool_bn_sign_pack), POOL_WINDOWS
    (conv_pool_windows_bn_sign_pack) or POOL_APART (conv_bn_sign_pack, then maxpool_bits)."""
    return load_library().bnn_conv_pool_form(B, H, W, Cin, Cout, kh, kw, stride, pad, pool)


def _conv_pool(name, x_bits, Cin, w_bits, thr, flip_bits, kh, kw, stride, pad, pool, out):
    if out is not None and _calls is not None:
        st = getattr(_calls, name)(x_bits, Cin, w_bits, kh, kw, stride, pad, thr, flip_bits, out, pool)
        if st == 0 or _took("bnn_" + name, st):
            return out
    lib = load_library()
    _check_nhwc_bits(x_bits, Cin)
    _dev(w_bits, torch.int32, "w_bits")
    B, H, W, _ = x_bits.shape
    Cout = w_bits.shape[0]
    Ho, Wo = (H + 2 * pad - kh) // stride + 1, (W + 2 * pad - kw) // stride + 1
    nw = words_per_row(Cout)
    if thr.dtype != torch.int32 or flip_bits.dtype != torch.int32 or not thr.is_cuda or not flip_bits.is_cuda:
        raise ValueError("thr and flip_bits must be int32 device tensors")
    if thr.numel() != Cout or flip_bits.numel() != nw or not thr.is_contiguous() or not flip_bits.is_contiguous():
        raise ValueError("thr must be [Cout] and flip_bits [ceil(Cout/32)], contiguous")
    if pool < 1:
        raise ValueError("pool must be positive")
    if out is None:
        out = torch.empty((B * (Ho // pool) * (Wo // pool), nw), dtype=torch.int32, device=x_bits.device)
    _dev(out, torch.int32, "out")
    _holds(w_bits, Cout if B * max(Ho, 0) * max(Wo, 0) else 0, words_per_row(kh * kw * Cin), "w_bits")
    if out.shape[0] != B * (Ho // pool) * (Wo // pool) or out.shape[1] != nw:
        raise ValueError("out must be [B*(Ho/pool)*(Wo/pool)][ceil(Cout/32)]")
    _check("bnn_" + name,
           getattr(lib, "bnn_" + name)(x_bits.data_ptr(), B, H, W, Cin, w_bits.data_ptr(), _ld(w_bits), Cout, kh, kw, stride,
                                       pad, pool, thr.data_ptr(), flip_bits.data_ptr(), out.data_ptr(), _ld(out),
                                       _stream(out)))
    return out


def maxpool_bits(x_bits: torch.Tensor, C: int, flip_bits: torch.Tensor | None, ph: int = 2, pw: int = 2,
                 stride: int = 2, out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_maxpool_bits: packed NHWC [B][H][W][Cw] -> [B][Hp][Wp][Cw]; OR where flip = 0, AND where flip = 1."""
    if out is not None and _calls is not None:
        st = _calls.maxpool_bits(x_bits, C, flip_bits, ph, pw, stride, out)
        if st == 0 or _took("bnn_maxpool_bits", st):
            return out
    lib = load_library()
    _check_nhwc_bits(x_bits, C)
    B, H, W, Cw = x_bits.shape
    Hp, Wp = (H - ph) // stride + 1, (W - pw) // stride + 1
    if flip_bits is not None and (flip_bits.dtype != torch.int32 or not flip_bits.is_cuda or
                                  flip_bits.numel() != Cw or not flip_bits.is_contiguous()):
        raise ValueError("flip_bits must be a contiguous int32 device tensor [ceil(C/32)]")
    if out is None:
        out = torch.empty((B, Hp, Wp, Cw), dtype=torch.int32, device=x_bits.device)
    if not out.is_cuda or out.dtype != torch.int32 or not out.is_contiguous() or out.numel() != B * Hp * Wp * Cw:
        raise ValueError("out must be a contiguous int32 device tensor [B][Hp][Wp][Cw]")
    _check("bnn_maxpool_bits", lib.bnn_maxpool_bits(x_bits.data_ptr(), B, H, W, C, ph, pw, stride,
                                                   flip_bits.data_ptr() if flip_bits is not None else None,
                                                   out.data_ptr(), _stream(out)))
    return out


def gemm_i8_mfma(A: torch.Tensor, B: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_gemm_i8_mfma: int8 A [M][K], int8 B [N][K] -> int32 C [M][N]."""
    lib = load_library()
    _dev(A, torch.int8, "A")
    _dev(B, torch.int8, "B")
    M, K = A.shape
    N, K2 = B.shape
    if K != K2:
        raise ValueError("A and B disagree on K")
    if out is None:
        out = torch.empty((M, N), dtype=torch.int32, device=A.device)
    _dev(out, torch.int32, "out")
    _holds(out, M, N, "out")
    _check("bnn_gemm_i8_mfma", lib.bnn_gemm_i8_mfma(A.data_ptr(), _ld(A), B.data_ptr(), _ld(B), out.data_ptr(),
                                                   _ld(out), M, N, K, _stream(out)))
    return out


def unpack_i8(bits: torch.Tensor, K: int, ld_out: int | None = None) -> torch.Tensor:
    """bnn_unpack_i8: packed rows -> int8 +-1 [rows][K] (row stride ld_out, default K rounded up to 16)."""
    lib = load_library()
    _dev(bits, torch.int32, "bits")
    rows = bits.shape[0]
    _holds(bits, rows, words_per_row(K), "bits")
    ld = ld_out if ld_out is not None else (K + 15) // 16 * 16
    buf = torch.empty((rows, ld), dtype=torch.int8, device=bits.device)
    _check("bnn_unpack_i8", lib.bnn_unpack_i8(bits.data_ptr(), _ld(bits), rows, K, buf.data_ptr(), ld, _stream(buf)))
    return buf[:, :K] if ld != K else buf


# ---- real activations, packed weights --------------------------------------------------------------------------

def _real(t: torch.Tensor, name: str, like: torch.Tensor | None = None):
    """A matrix of real activations; of the type and on the device of `like`."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in _TYPES:
        raise ValueError(f"{name} must be bfloat16, float16 or float32, got {t.dtype}")
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be 2-D with unit stride along its rows")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{name} must be {like.dtype} on {like.device}, got {t.dtype} on {t.device}")
    return t


def _sized(t: torch.Tensor, rows: int, cols: int, name: str, like: torch.Tensor):
    _real(t, name, like)
    if tuple(t.shape) != (rows, cols):
        raise ValueError(f"{name} must be [{rows}][{cols}], got {list(t.shape)}")
    return t


def _vector(t: torch.Tensor | None, n: int, name: str, like: torch.Tensor):
    """Address of a float32 vector of n elements, or None."""
    if t is None:
        return None
    if t.dtype != torch.float32 or t.device != like.device or tuple(t.shape) != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 vector of {n} elements on {like.device}")
    return t.data_ptr()


def _weights(x: torch.Tensor, w_bits: torch.Tensor):
    _dev(w_bits, torch.int32, "w_bits")
    if w_bits.device != x.device:
        raise ValueError(f"w_bits must be on {x.device}")
    if w_bits.shape[1] < words_per_row(x.shape[1]):
        raise ValueError("packed weights have fewer words per row than x has columns")


def _count_write(t: torch.Tensor | None):
    """A caller's tensor is written: torch's count of that moves on, so that who kept the tensor can tell."""
    if t is not None and not t.is_inference():
        torch.autograd.graph.increment_version(t)


def _at(t: torch.Tensor | None):
    """Address and leading dimension of a matrix; (None, 0) where there is none."""
    return (None, 0) if t is None else (t.data_ptr(), _ld(t))


def _workspace(workspace: torch.Tensor | None, size: int, like: torch.Tensor, fn: str) -> torch.Tensor:
    if size < 0:
        raise ValueError(f"{fn} takes no such sizes")
    if workspace is None:
        return torch.empty(size, dtype=torch.uint8, device=like.device)
    if workspace.dtype != torch.uint8 or workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {like.device}")
    if workspace.numel() < size:
        raise ValueError(f"workspace holds {workspace.numel()} bytes, {size} are needed")
    return workspace


def _recorded(*inputs) -> bool:
    """Whether torch records what is done with these tensors."""
    return any(t is not None and t.requires_grad for t in inputs) and torch.is_grad_enabled()


class _LinearBits(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_bits, scale, bias, act, residual):
        ctx.save_for_backward(x, w_bits, scale, bias)
        ctx.act = act
        return linear_bits(x, w_bits, scale, bias, act, residual)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        return *_product_gradients(ctx, linear_bits_backward, dy), None, dy if ctx.needs_input_grad[5] else None


class _GatedBits(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_bits, scale, bias, act):
        ctx.save_for_backward(x, w_bits, scale, bias)
        ctx.act = act
        return gated_bits(x, w_bits, scale, bias, act)

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        return *_product_gradients(ctx, gated_bits_backward, dh), None


def _product_gradients(ctx, call, dy):
    """Of x, w_bits (none: it holds bits), scale and bias."""
    need_x, _, need_scale, need_bias = ctx.needs_input_grad[:4]
    if not (need_x or need_scale or need_bias):
        return None, None, None, None
    got = call(dy.contiguous(), *ctx.saved_tensors, ctx.act, need_dx=need_x, need_dw=False)
    return got["dx"], None, got["dscale"] if need_scale else None, got["dbias"] if need_bias else None


class _NormResidual(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, x, gate, res_scale, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, eps, rows_per_gate):
        r, n = norm_residual(y, x, gate, res_scale, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, eps, rows_per_gate)
        ctx.save_for_backward(y, r if pre != NORM_NONE else None, gate, post_gamma, post_beta, pre_gamma, pre_beta)
        ctx.kinds = res_scale, post, pre, eps, rows_per_gate
        ctx.set_materialize_grads(False)
        return r, n

    @staticmethod
    @once_differentiable
    def backward(ctx, dr, dn):
        if dr is None and dn is None:
            return (None,) * 12
        y, r, gate, post_gamma, post_beta, pre_gamma, pre_beta = ctx.saved_tensors
        res_scale, post, pre, eps, rows_per_gate = ctx.kinds
        if pre != NORM_NONE:
            dn = torch.zeros_like(r) if dn is None else dn.contiguous()
        got = norm_residual_backward(None if dr is None else dr.contiguous(), dn, y, r, gate, res_scale, post, post_gamma, post_beta,
                                     pre, pre_gamma, pre_beta, eps, rows_per_gate, need_dx=ctx.needs_input_grad[1])
        grads = (got["dy"], got["dx"], got["dgate"], None, None, got["dpost_gamma"], got["dpost_beta"], None, got["dpre_gamma"],
                 got["dpre_beta"], None, None)
        return tuple(g if need else None for g, need in zip(grads, ctx.needs_input_grad))


def linear_bits(x: torch.Tensor, w_bits: torch.Tensor, scale: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                act: int = ACT_NONE, residual: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_linear_bits: real x [M][K], packed weights [N][ceil(K/32)] -> act(scale * (x w^T) + bias) + residual [M][N].
    `out` may be `residual`.  Without `out`, torch differentiates the result with respect to x, scale, bias and residual (of the
    packed weights linear_bits_backward gives a gradient); what is written to `out` is not recorded."""
    if out is not None and _calls is not None:
        st = _calls.linear_bits(x, w_bits, scale, bias, act, residual, out)
        if st == 0 or _took("bnn_linear_bits", st):
            return out
    if out is None and _recorded(x, scale, bias, residual):
        return _LinearBits.apply(x, w_bits, scale, bias, act, residual)
    lib = load_library()
    _real(x, "x")
    _weights(x, w_bits)
    (M, K), N = x.shape, w_bits.shape[0]
    if residual is not None:
        _sized(residual, M, N, "residual", x)
    given = out
    if out is None:
        out = torch.empty((M, N), dtype=x.dtype, device=x.device)
    _sized(out, M, N, "out", x)
    _check("bnn_linear_bits",
           lib.bnn_linear_bits(_TYPES[x.dtype], *_at(x), *_at(w_bits), _vector(scale, N, "scale", x), _vector(bias, N, "bias", x), act,
                               *_at(residual), *_at(out), M, N, K, _stream(x)))
    _count_write(given)
    return out


def _halves(w_bits: torch.Tensor) -> int:
    if w_bits.shape[0] % 2:
        raise ValueError("gated weights are the gate's rows and as many of the other projection")
    return w_bits.shape[0] // 2


def gated_bits(x: torch.Tensor, w_bits: torch.Tensor, scale: torch.Tensor | None = None, bias: torch.Tensor | None = None,
               act: int = ACT_SILU, out: torch.Tensor | None = None) -> torch.Tensor:
    """bnn_gated_bits: real x [M][K], packed weights [2F][ceil(K/32)] (the gate's rows first) -> act(z_gate) * z_up [M][F]
    with z = scale * (x w^T) + bias.  Differentiated as linear_bits is."""
    if out is not None and _calls is not None:
        st = _calls.gated_bits(x, w_bits, scale, bias, act, out)
        if st == 0 or _took("bnn_gated_bits", st):
            return out
    if out is None and _recorded(x, scale, bias):
        return _GatedBits.apply(x, w_bits, scale, bias, act)
    lib = load_library()
    _real(x, "x")
    _weights(x, w_bits)
    (M, K), F = x.shape, _halves(w_bits)
    given = out
    if out is None:
        out = torch.empty((M, F), dtype=x.dtype, device=x.device)
    _sized(out, M, F, "out", x)
    _check("bnn_gated_bits",
           lib.bnn_gated_bits(_TYPES[x.dtype], *_at(x), *_at(w_bits), _vector(scale, 2 * F, "scale", x),
                              _vector(bias, 2 * F, "bias", x), act, *_at(out), M, F, K, _stream(x)))
    _count_write(given)
    return out


def _real_type(dtype: torch.dtype) -> int:
    if dtype not in _TYPES:
        raise ValueError(f"activations are bfloat16, float16 or float32, not {dtype}")
    return _TYPES[dtype]


def linear_bits_backward_workspace(dtype: torch.dtype, M: int, N: int, K: int, act: int = ACT_NONE) -> int:
    """bnn_linear_bits_backward_workspace: bytes."""
    return load_library().bnn_linear_bits_backward_workspace(_real_type(dtype), M, N, K, act)


def gated_bits_backward_workspace(dtype: torch.dtype, M: int, F: int, K: int, act: int = ACT_SILU) -> int:
    """bnn_gated_bits_backward_workspace: bytes."""
    return load_library().bnn_gated_bits_backward_workspace(_real_type(dtype), M, F, K, act)


def _bits_backward(name, dy, x, w_bits, scale, bias, act, need_dx, need_dw, workspace):
    lib = load_library()
    if _calls is not None:
        got = getattr(_calls, name[4:])(dy, x, w_bits, scale, bias, act, need_dx, need_dw, workspace)
        if got != -1:
            _check(name, got[0])
            return {"dx": got[1], "dw": got[2], "dscale": got[3], "dbias": got[4]}
    cols = _halves(w_bits) if name == "bnn_gated_bits_backward" else w_bits.shape[0]
    _real(x, "x")
    _weights(x, w_bits)
    (M, K), N = x.shape, w_bits.shape[0]
    _sized(dy, M, cols, "the gradient of the result", x)
    size = getattr(lib, name + "_workspace")(_TYPES[x.dtype], M, cols, K, act)
    at_scale, at_bias = _vector(scale, N, "scale", x), _vector(bias, N, "bias", x)
    ws = _workspace(workspace, size, x, name)
    dx = torch.empty((M, K), dtype=x.dtype, device=x.device) if need_dx else None
    dw = torch.empty((N, K), dtype=x.dtype, device=x.device) if need_dw else None
    dscale = torch.empty(N, dtype=torch.float32, device=x.device) if scale is not None else None
    dbias = torch.empty(N, dtype=torch.float32, device=x.device) if bias is not None else None
    _check(name, getattr(lib, name)(_TYPES[x.dtype], *_at(dy), *_at(x), *_at(w_bits), at_scale, at_bias, act, *_at(dx), *_at(dw),
                                    None if dscale is None else dscale.data_ptr(), None if dbias is None else dbias.data_ptr(),
                                    M, cols, K, ws.data_ptr(), ws.numel(), _stream(x)))
    return {"dx": dx, "dw": dw, "dscale": dscale, "dbias": dbias}


def linear_bits_backward(dy: torch.Tensor, x: torch.Tensor, w_bits: torch.Tensor, scale: torch.Tensor | None = None,
                         bias: torch.Tensor | None = None, act: int = ACT_NONE, need_dx: bool = True, need_dw: bool = True,
                         workspace: torch.Tensor | None = None) -> dict:
    """bnn_linear_bits_backward: {"dx" [M][K], "dw" [N][K], "dscale" [N], "dbias" [N]}, None for what was not there or not
    wanted.  dw is the gradient of the weights as real numbers; the residual's gradient is dy."""
    return _bits_backward("bnn_linear_bits_backward", dy, x, w_bits, scale, bias, act, need_dx, need_dw, workspace)


def gated_bits_backward(dh: torch.Tensor, x: torch.Tensor, w_bits: torch.Tensor, scale: torch.Tensor | None = None,
                        bias: torch.Tensor | None = None, act: int = ACT_SILU, need_dx: bool = True, need_dw: bool = True,
                        workspace: torch.Tensor | None = None) -> dict:
    """bnn_gated_bits_backward: as linear_bits_backward, with dw [2F][K], dscale and dbias [2F]."""
    return _bits_backward("bnn_gated_bits_backward", dh, x, w_bits, scale, bias, act, need_dx, need_dw, workspace)


def norm_residual(y: torch.Tensor, x: torch.Tensor | None = None, gate: torch.Tensor | None = None, res_scale: float = 1.0,
                  post: int = NORM_NONE, post_gamma: torch.Tensor | None = None, post_beta: torch.Tensor | None = None,
                  pre: int = NORM_NONE, pre_gamma: torch.Tensor | None = None, pre_beta: torch.Tensor | None = None,
                  eps: float = 1e-5, rows_per_gate: int = 1, out: torch.Tensor | None = None, out_n: torch.Tensor | None = None,
                  need_r: bool = True):
    """bnn_norm_residual: (r, n) with r = x + res_scale * gate * post(y) and n = pre(r); n is None without a `pre` norm, r where
    it is not needed.  Row m has the gate's row m // rows_per_gate.  `out` may be `x`.  Without `out` and `out_n`, torch
    differentiates both results with respect to every tensor; what is written to those two is not recorded."""
    if out is not None and _calls is not None:
        st = _calls.norm_residual(y, x, gate, res_scale, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, eps, rows_per_gate,
                                  out, out_n)
        if st == 0 or _took("bnn_norm_residual", st):
            return out, out_n
    if out is None and out_n is None and _recorded(y, x, gate, post_gamma, post_beta, pre_gamma, pre_beta):
        r, n = _NormResidual.apply(y, x, gate, res_scale, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, eps, rows_per_gate)
        return (r if need_r else None), n
    lib = load_library()
    _real(y, "y")
    M, D = y.shape
    if x is not None:
        _sized(x, M, D, "x", y)
    if gate is not None:
        if rows_per_gate < 1:
            raise ValueError("rows_per_gate must be positive")
        _sized(gate, -(-M // rows_per_gate), D, "gate", y)
    given = out, out_n
    if out is None and need_r:
        out = torch.empty((M, D), dtype=y.dtype, device=y.device)
    if out is not None:
        _sized(out, M, D, "out", y)
    if pre == NORM_NONE:
        if out_n is not None:
            raise ValueError("out_n needs a norm before the next block")
    elif out_n is None:
        out_n = torch.empty((M, D), dtype=y.dtype, device=y.device)
    if out_n is not None:
        _sized(out_n, M, D, "out_n", y)
    _check("bnn_norm_residual",
           lib.bnn_norm_residual(_TYPES[y.dtype], *_at(y), *_at(x), *_at(gate), rows_per_gate, res_scale, post,
                                 _vector(post_gamma, D, "post_gamma", y), _vector(post_beta, D, "post_beta", y), pre,
                                 _vector(pre_gamma, D, "pre_gamma", y), _vector(pre_beta, D, "pre_beta", y), eps,
                                 *_at(out), *_at(out_n), M, D, _stream(y)))
    for t in given:
        _count_write(t)
    return out, out_n


def norm_residual_backward_workspace(M: int, D: int, rows_per_gate: int = 1) -> int:
    """bnn_norm_residual_backward_workspace: bytes."""
    return load_library().bnn_norm_residual_backward_workspace(M, D, rows_per_gate)


def norm_residual_backward(dr: torch.Tensor | None, dn: torch.Tensor | None, y: torch.Tensor, r: torch.Tensor | None,
                           gate: torch.Tensor | None = None, res_scale: float = 1.0, post: int = NORM_NONE,
                           post_gamma: torch.Tensor | None = None, post_beta: torch.Tensor | None = None, pre: int = NORM_NONE,
                           pre_gamma: torch.Tensor | None = None, pre_beta: torch.Tensor | None = None, eps: float = 1e-5,
                           rows_per_gate: int = 1, need_dx: bool = True, workspace: torch.Tensor | None = None) -> dict:
    """bnn_norm_residual_backward: {"dx", "dy", "dgate", "dpost_gamma", "dpost_beta", "dpre_gamma", "dpre_beta"}, None for
    what was not there or not wanted, from the gradients dr of r (by every way but n) and dn of n."""
    lib = load_library()
    if _calls is not None:
        got = _calls.norm_residual_backward(dr, dn, y, r, gate, res_scale, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, eps,
                                            rows_per_gate, need_dx, workspace)
        if got != -1:
            _check("bnn_norm_residual_backward", got[0])
            return {"dx": got[1], "dy": got[2], "dgate": got[3], "dpost_gamma": got[4], "dpost_beta": got[5], "dpre_gamma": got[6],
                    "dpre_beta": got[7]}
    _real(y, "y")
    M, D = y.shape
    for t, name in ((dr, "dr"), (dn, "dn"), (r, "r")):
        if t is not None:
            _sized(t, M, D, name, y)
    if gate is not None:
        if rows_per_gate < 1:
            raise ValueError("rows_per_gate must be positive")
        _sized(gate, -(-M // rows_per_gate), D, "gate", y)
    if pre != NORM_NONE and (dn is None or r is None):
        raise ValueError("a norm before the next block needs dn and r")
    if pre == NORM_NONE and dn is not None:
        raise ValueError("dn needs a norm before the next block")
    vectors = {"post_gamma": post_gamma, "post_beta": post_beta, "pre_gamma": pre_gamma, "pre_beta": pre_beta}
    at = {k: _vector(v, D, k, y) for k, v in vectors.items()}
    ws = _workspace(workspace, lib.bnn_norm_residual_backward_workspace(M, D, rows_per_gate), y, "bnn_norm_residual_backward")
    got = {"dx": torch.empty((M, D), dtype=y.dtype, device=y.device) if need_dx else None,
           "dy": torch.empty((M, D), dtype=y.dtype, device=y.device),
           "dgate": torch.empty(tuple(gate.shape), dtype=y.dtype, device=y.device) if gate is not None else None}
    for k, v in vectors.items():
        got["d" + k] = torch.empty(D, dtype=torch.float32, device=y.device) if v is not None else None
    _check("bnn_norm_residual_backward",
           lib.bnn_norm_residual_backward(_TYPES[y.dtype], *_at(dr), *_at(dn), *_at(y), *_at(r), *_at(gate), rows_per_gate, res_scale,
                                          post, at["post_gamma"], at["post_beta"], pre, at["pre_gamma"], eps, *_at(got["dx"]),
                                          *_at(got["dy"]), *_at(got["dgate"]),
                                          *(None if got["d" + k] is None else got["d" + k].data_ptr() for k in vectors), M, D,
                                          ws.data_ptr(), ws.numel(), _stream(y)))
    return got
