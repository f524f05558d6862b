"""ctypes binding of the few-token operators (``include/exo_decode.h``; argument marshalling only).

The functions have the names of the C entry points and return their status.  ``Q4`` and ``MoePlan`` wrap them and
raise ``ExoGemmError``.  Pointers are device addresses (ints) and streams are stream handles; the caller keeps the
memory behind them alive.  There is no fallback: all compute is in the CUDA library.
"""
from __future__ import annotations

import ctypes

import numpy as np

from . import binding
from .binding import BF16, FP16, FP32, OK, ExoGemmError  # noqa: F401

EXPORTED_SYMBOLS = (
    "exo_q4_quantize", "exo_q4_dequantize", "exo_gemv_q4_run", "exo_moe_validate", "exo_moe_create", "exo_moe_run",
    "exo_moe_workspace_bytes", "exo_moe_destroy", "exo_decode_check", "exo_decode_debug_set",
)

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class Q4Struct(ctypes.Structure):
    """exo_q4_t"""
    _fields_ = [("rows", _i64), ("K", _i64), ("group", _i32), ("dtype", _i32), ("codes", _vp), ("scales", _vp), ("zeros", _vp)]


class MoeDesc(ctypes.Structure):
    """exo_moe_desc_t"""
    _fields_ = [("hidden", _i64), ("inner", _i64), ("experts", _i32), ("shared", _i32), ("top_k", _i32), ("max_tokens", _i32),
                ("dtype", _i32), ("q4_group", _i32), ("renormalize", _i32), ("routed_scale", _f32), ("device", _i32)]

    def __init__(self, hidden, inner, experts, shared, top_k, max_tokens, dtype, q4_group=0, renormalize=1, routed_scale=1.0,
                 device=-1):
        super().__init__(hidden, inner, experts, shared, top_k, max_tokens, dtype, q4_group, renormalize, routed_scale, device)


class MoeMatrix(ctypes.Structure):
    """exo_moe_matrix_t"""
    _fields_ = [("w", _vp), ("ld", _i64), ("expert_rows", _i64), ("scales", _vp), ("zeros", _vp)]


class MoeWeights(ctypes.Structure):
    """exo_moe_weights_t"""
    _fields_ = [("router", _vp), ("ld_router", _i64), ("gate", MoeMatrix), ("up", MoeMatrix), ("down", MoeMatrix)]


_lib = None


def lib():
    """The library of ``binding.lib()`` with this header's prototypes."""
    global _lib
    if _lib is None:
        L = binding.lib()
        q4, desc, weights = ctypes.POINTER(Q4Struct), ctypes.POINTER(MoeDesc), ctypes.POINTER(MoeWeights)
        L.exo_q4_quantize.argtypes = L.exo_q4_dequantize.argtypes = [q4, _vp, _i64, _i32, _vp]
        L.exo_gemv_q4_run.argtypes = [q4, _i64, _vp, _i64, _vp, _i64, _i32, _f32, _f32, _vp]
        L.exo_moe_validate.argtypes = [desc]
        L.exo_moe_create.argtypes = [ctypes.POINTER(_vp), desc]
        L.exo_moe_run.argtypes = [_vp, weights, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp]
        L.exo_moe_workspace_bytes.argtypes = [_vp]
        L.exo_moe_destroy.argtypes = [_vp]
        L.exo_decode_debug_set.argtypes = [_i32, _i32]
        for name in EXPORTED_SYMBOLS:
            getattr(L, name).restype = ctypes.c_int
        L.exo_moe_workspace_bytes.restype = _i64
        _lib = L
    return _lib


# ---- one function per C entry point -------------------------------------------------
def exo_q4_quantize(q, w_ptr: int, ldw: int, w_dtype: int, stream: int = 0) -> int:
    return lib().exo_q4_quantize(q, w_ptr, ldw, w_dtype, stream)


def exo_q4_dequantize(q, w_ptr: int, ldw: int, w_dtype: int, stream: int = 0) -> int:
    return lib().exo_q4_dequantize(q, w_ptr, ldw, w_dtype, stream)


def exo_gemv_q4_run(q, tokens: int, x_ptr: int, ldx: int, y_ptr: int, ldy: int, y_dtype: int, alpha: float = 1.0,
                    beta: float = 0.0, stream: int = 0) -> int:
    return lib().exo_gemv_q4_run(q, tokens, x_ptr, ldx, y_ptr, ldy, y_dtype, alpha, beta, stream)


def exo_moe_validate(desc) -> int:
    return lib().exo_moe_validate(desc)


def exo_moe_create(desc):
    h = _vp()
    st = lib().exo_moe_create(ctypes.byref(h), desc)
    return st, (h if st == OK else None)


def exo_moe_run(handle, weights, tokens: int, x_ptr: int, ldx: int, y_ptr: int, ldy: int, index_ptr: int = 0,
                weight_ptr: int = 0, stream: int = 0) -> int:
    return lib().exo_moe_run(handle, weights, tokens, x_ptr, ldx, y_ptr, ldy, index_ptr, weight_ptr, stream)


def exo_decode_check() -> int:
    return lib().exo_decode_check()


def exo_decode_debug_set(timeout_ms: int, skip_copies: int) -> int:
    return lib().exo_decode_debug_set(timeout_ms, skip_copies)


def exo_moe_workspace_bytes(handle) -> int:
    return lib().exo_moe_workspace_bytes(handle)


def exo_moe_destroy(handle) -> int:
    return lib().exo_moe_destroy(handle)


# ---- thin convenience wrappers --------------------------------------------------------
def padded_k(K: int) -> int:
    """Weights a row of a 4-bit matrix has room for: K rounded up to a multiple of 128."""
    return (K + 127) // 128 * 128


def pack_codes(codes: np.ndarray) -> np.ndarray:
    """rows x K codes 0 .. 15 (host; say of a checkpoint that is 4-bit already) -> rows x padded_k(K) / 2 bytes in the
    layout of exo_q4_t."""
    rows, K = codes.shape
    c = np.zeros((rows, padded_k(K)), np.uint8)
    c[:, :K] = codes
    c = c.reshape(rows, -1, 4, 4, 4, 2).transpose(0, 1, 3, 2, 5, 4)   # block, j, t, i / 2, i % 2 -> block, t, j, i % 2, i / 2
    c = c.reshape(rows, -1, 2)
    return np.ascontiguousarray(c[:, :, 0] | c[:, :, 1] << 4)


class Q4:
    """A 4-bit matrix by its device pointers.  ``codes`` are rows of padded_k(K) / 2 bytes, ``scales`` (of ``dtype``) and
    ``zeros`` (bytes; 0: none, every zero point is 8) rows of padded_k(K) / group values."""

    def __init__(self, rows: int, K: int, group: int, dtype: int, codes: int, scales: int, zeros: int = 0):
        self.struct = Q4Struct(rows, K, group, dtype, codes, scales, zeros)
        # the methods are what a decode loop calls: entry points and the struct's address are looked up once
        L = lib()
        self._calls, self._at = (L.exo_q4_quantize, L.exo_q4_dequantize, L.exo_gemv_q4_run), ctypes.byref(self.struct)

    def quantize(self, w_ptr: int, ldw: int, w_dtype: int, stream: int = 0):
        st = self._calls[0](self._at, w_ptr, ldw, w_dtype, stream)
        if st:
            raise ExoGemmError(st, "exo_q4_quantize")

    def dequantize(self, w_ptr: int, ldw: int, w_dtype: int, stream: int = 0):
        st = self._calls[1](self._at, w_ptr, ldw, w_dtype, stream)
        if st:
            raise ExoGemmError(st, "exo_q4_dequantize")

    def gemv(self, tokens: int, x_ptr: int, ldx: int, y_ptr: int, ldy: int, y_dtype: int, alpha: float = 1.0,
             beta: float = 0.0, stream: int = 0):
        st = self._calls[2](self._at, tokens, x_ptr, ldx, y_ptr, ldy, y_dtype, alpha, beta, stream)
        if st:
            raise ExoGemmError(st, "exo_gemv_q4_run")


class MoePlan:
    """Owns one mixture-of-experts plan."""

    def __init__(self, desc: MoeDesc):
        self.handle = None
        st, h = exo_moe_create(desc)
        if st != OK:
            raise ExoGemmError(st, "exo_moe_create")
        self.handle, self.desc, self._run = h, desc, lib().exo_moe_run

    def run(self, weights: MoeWeights, tokens: int, x_ptr: int, ldx: int, y_ptr: int, ldy: int, index_ptr: int = 0,
            weight_ptr: int = 0, stream: int = 0):
        st = self._run(self.handle, weights, tokens, x_ptr, ldx, y_ptr, ldy, index_ptr, weight_ptr, stream)
        if st:
            raise ExoGemmError(st, "exo_moe_run")

    def workspace_bytes(self) -> int:
        return exo_moe_workspace_bytes(self.handle)

    def close(self):
        if self.handle is not None:
            exo_moe_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
