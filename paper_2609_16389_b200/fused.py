"""ctypes binding of the products with an operator in their epilogue (``include/exo_fused.h``; argument marshalling only).

The functions have the names of the C entry points and return their status.  ``FfnPlan``, ``CePlan`` and ``I8`` wrap them and raise
``ExoGemmError``.  Pointers are device addresses (ints) and streams are stream handles; the caller keeps the memory behind them alive.
There is no fallback: all compute is in the CUDA library.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import BF16, FP16, FP32, OK, ExoGemmError  # noqa: F401

SILU, GELU, GELU_TANH = 0, 1, 2

EXPORTED_SYMBOLS = (
    "exo_ffn_validate", "exo_ffn_create", "exo_ffn_saved_bytes", "exo_ffn_forward", "exo_ffn_backward", "exo_ffn_check",
    "exo_ffn_workspace_bytes", "exo_ffn_destroy", "exo_ce_validate", "exo_ce_create", "exo_ce_saved_bytes", "exo_ce_forward",
    "exo_ce_backward", "exo_ce_check", "exo_ce_workspace_bytes", "exo_ce_destroy", "exo_i8_quantize", "exo_gemm_i8_run",
    "exo_fused_check", "exo_fused_debug_set",
)

_vp, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class FfnDesc(ctypes.Structure):
    """exo_ffn_desc_t; leading dimensions of 0 stand for packed rows."""
    _fields_ = [("tokens", _i64), ("hidden", _i64), ("inner", _i64), ("dtype", _i32), ("activation", _i32), ("training", _i32),
                ("grad_dtype", _i32), ("ldx", _i64), ("ldy", _i64), ("ld_gate_up", _i64), ("ld_down", _i64), ("device", _i32)]

    def __init__(self, tokens, hidden, inner, dtype, activation=SILU, training=0, grad_dtype=FP32, ldx=0, ldy=0, ld_gate_up=0, ld_down=0,
                 device=-1):
        super().__init__(tokens, hidden, inner, dtype, activation, training, grad_dtype, ldx, ldy, ld_gate_up, ld_down, device)


class CeDesc(ctypes.Structure):
    """exo_ce_desc_t; leading dimensions of 0 stand for packed rows."""
    _fields_ = [("tokens", _i64), ("hidden", _i64), ("vocab", _i64), ("dtype", _i32), ("training", _i32), ("grad_dtype", _i32),
                ("label_smoothing", _f32), ("ignore_index", _i64), ("ldx", _i64), ("ldw", _i64), ("keep_bytes", _i64), ("piece", _i64),
                ("device", _i32)]

    def __init__(self, tokens, hidden, vocab, dtype, training=0, grad_dtype=FP32, label_smoothing=0.0, ignore_index=-100, ldx=0, ldw=0,
                 keep_bytes=-1, piece=0, device=-1):
        super().__init__(tokens, hidden, vocab, dtype, training, grad_dtype, label_smoothing, ignore_index, ldx, ldw, keep_bytes, piece,
                         device)


class I8Struct(ctypes.Structure):
    """exo_i8_t"""
    _fields_ = [("rows", _i64), ("K", _i64), ("ld", _i64), ("codes", _vp), ("scales", _vp)]


_lib = None


def lib():
    """The library of ``binding.lib()`` with this header's prototypes."""
    global _lib
    if _lib is None:
        L = binding.lib()
        ffn, ce, i8 = ctypes.POINTER(FfnDesc), ctypes.POINTER(CeDesc), ctypes.POINTER(I8Struct)
        for name in EXPORTED_SYMBOLS:
            getattr(L, name).restype = ctypes.c_int
        for kind, desc in (("ffn", ffn), ("ce", ce)):
            getattr(L, f"exo_{kind}_validate").argtypes = [desc]
            getattr(L, f"exo_{kind}_create").argtypes = [ctypes.POINTER(_vp), desc]
            for name in ("check", "destroy", "saved_bytes", "workspace_bytes"):
                getattr(L, f"exo_{kind}_{name}").argtypes = [_vp]
            getattr(L, f"exo_{kind}_saved_bytes").restype = _i64
            getattr(L, f"exo_{kind}_workspace_bytes").restype = _i64
        L.exo_ffn_forward.argtypes = [_vp] * 7
        L.exo_ffn_backward.argtypes = [_vp] * 9 + [_i32, _vp]
        L.exo_ce_forward.argtypes = [_vp] * 8
        L.exo_ce_backward.argtypes = [_vp] * 9 + [_i32, _vp]
        L.exo_i8_quantize.argtypes = [i8, _vp, _i64, _i32, _vp]
        L.exo_gemm_i8_run.argtypes = [i8, i8, _vp, _i64, _i32, _f32, _f32, _vp]
        L.exo_fused_check.argtypes = []
        L.exo_fused_debug_set.argtypes = [_i32, _i32]
        _lib = L
    return _lib


# ---- one function per C entry point -------------------------------------------------
def exo_ffn_validate(desc) -> int:
    return lib().exo_ffn_validate(desc)


def exo_ffn_create(desc):
    h = _vp()
    st = lib().exo_ffn_create(ctypes.byref(h), desc)
    return st, (h if st == OK else None)


def exo_ffn_saved_bytes(handle) -> int:
    return lib().exo_ffn_saved_bytes(handle)


def exo_ffn_forward(handle, x: int, gate_up: int, down: int, y: int, saved: int = 0, stream: int = 0) -> int:
    return lib().exo_ffn_forward(handle, x, gate_up, down, y, saved, stream)


def exo_ffn_backward(handle, x: int, gate_up: int, down: int, saved: int, dy: int, dx: int = 0, d_gate_up: int = 0, d_down: int = 0,
                     accumulate: int = 0, stream: int = 0) -> int:
    return lib().exo_ffn_backward(handle, x, gate_up, down, saved, dy, dx, d_gate_up, d_down, accumulate, stream)


def exo_ffn_check(handle) -> int:
    return lib().exo_ffn_check(handle)


def exo_ffn_workspace_bytes(handle) -> int:
    return lib().exo_ffn_workspace_bytes(handle)


def exo_ffn_destroy(handle) -> int:
    return lib().exo_ffn_destroy(handle)


def exo_ce_validate(desc) -> int:
    return lib().exo_ce_validate(desc)


def exo_ce_create(desc):
    h = _vp()
    st = lib().exo_ce_create(ctypes.byref(h), desc)
    return st, (h if st == OK else None)


def exo_ce_saved_bytes(handle) -> int:
    return lib().exo_ce_saved_bytes(handle)


def exo_ce_forward(handle, x: int, w: int, target: int, loss: int = 0, lse: int = 0, saved: int = 0, stream: int = 0) -> int:
    return lib().exo_ce_forward(handle, x, w, target, loss, lse, saved, stream)


def exo_ce_backward(handle, x: int, w: int, target: int, lse: int, dloss: int, saved: int = 0, dx: int = 0, dw: int = 0,
                    accumulate: int = 0, stream: int = 0) -> int:
    return lib().exo_ce_backward(handle, x, w, target, lse, dloss, saved, dx, dw, accumulate, stream)


def exo_ce_check(handle) -> int:
    return lib().exo_ce_check(handle)


def exo_ce_workspace_bytes(handle) -> int:
    return lib().exo_ce_workspace_bytes(handle)


def exo_ce_destroy(handle) -> int:
    return lib().exo_ce_destroy(handle)


def exo_i8_quantize(q, x_ptr: int, ldx: int, x_dtype: int, stream: int = 0) -> int:
    return lib().exo_i8_quantize(q, x_ptr, ldx, x_dtype, stream)


def exo_gemm_i8_run(x, w, y_ptr: int, ldy: int, y_dtype: int, alpha: float = 1.0, beta: float = 0.0, stream: int = 0) -> int:
    return lib().exo_gemm_i8_run(x, w, y_ptr, ldy, y_dtype, alpha, beta, stream)


def exo_fused_check() -> int:
    return lib().exo_fused_check()


def exo_fused_debug_set(timeout_ms: int, skip_copies: int) -> int:
    return lib().exo_fused_debug_set(timeout_ms, skip_copies)


# ---- thin convenience wrappers --------------------------------------------------------
def _raise(st: int, where: str):
    if st:
        raise ExoGemmError(st, where)


class _Plan:
    """Owns one plan of `kind`."""
    kind = ""

    def __init__(self, desc):
        self.handle = None
        L = lib()
        h = _vp()
        _raise(getattr(L, f"exo_{self.kind}_create")(ctypes.byref(h), desc), f"exo_{self.kind}_create")
        self.handle, self.desc = h, desc
        # forward and backward are what a loop calls: their entry points are looked up once
        self._forward, self._backward = getattr(L, f"exo_{self.kind}_forward"), getattr(L, f"exo_{self.kind}_backward")

    def saved_bytes(self) -> int:
        return getattr(lib(), f"exo_{self.kind}_saved_bytes")(self.handle)

    def workspace_bytes(self) -> int:
        return getattr(lib(), f"exo_{self.kind}_workspace_bytes")(self.handle)

    def check(self):
        _raise(getattr(lib(), f"exo_{self.kind}_check")(self.handle), f"exo_{self.kind}_check")

    def close(self):
        if self.handle is not None:
            getattr(lib(), f"exo_{self.kind}_destroy")(self.handle)
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


class FfnPlan(_Plan):
    """A gated feed-forward block for a number of tokens."""
    kind = "ffn"

    def forward(self, x: int, gate_up: int, down: int, y: int, saved: int = 0, stream: int = 0):
        _raise(self._forward(self.handle, x, gate_up, down, y, saved, stream), "exo_ffn_forward")

    def backward(self, x: int, gate_up: int, down: int, saved: int, dy: int, dx: int = 0, d_gate_up: int = 0, d_down: int = 0,
                 accumulate: int = 0, stream: int = 0):
        _raise(self._backward(self.handle, x, gate_up, down, saved, dy, dx, d_gate_up, d_down, accumulate, stream), "exo_ffn_backward")


class CePlan(_Plan):
    """The cross entropy of a head over a vocabulary, for a number of tokens."""
    kind = "ce"

    def forward(self, x: int, w: int, target: int, loss: int = 0, lse: int = 0, saved: int = 0, stream: int = 0):
        _raise(self._forward(self.handle, x, w, target, loss, lse, saved, stream), "exo_ce_forward")

    def backward(self, x: int, w: int, target: int, lse: int, dloss: int, saved: int = 0, dx: int = 0, dw: int = 0, accumulate: int = 0,
                 stream: int = 0):
        _raise(self._backward(self.handle, x, w, target, lse, dloss, saved, dx, dw, accumulate, stream), "exo_ce_backward")


class I8:
    """A matrix in 8 bits by its device pointers: rows of ``ld`` codes (a multiple of 16), a scale per row."""

    def __init__(self, rows: int, K: int, ld: int, codes: int, scales: int):
        self.struct = I8Struct(rows, K, ld, codes, scales)
        L = lib()
        self._calls, self._at = (L.exo_i8_quantize, L.exo_gemm_i8_run), ctypes.byref(self.struct)

    def quantize(self, x_ptr: int, ldx: int, x_dtype: int, stream: int = 0):
        _raise(self._calls[0](self._at, x_ptr, ldx, x_dtype, stream), "exo_i8_quantize")

    def gemm(self, x: "I8", y_ptr: int, ldy: int, y_dtype: int, alpha: float = 1.0, beta: float = 0.0, stream: int = 0):
        """Y = alpha * X * W^T + beta * Y, W being this matrix."""
        _raise(self._calls[1](x._at, self._at, y_ptr, ldy, y_dtype, alpha, beta, stream), "exo_gemm_i8_run")
