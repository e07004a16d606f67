"""Thin Python binding of the C ABI in include/pb.h (same names, argument marshalling only).

Every step of the path runs in the HIP kernels of libpbatch.so; torch is used for
device memory and streams.  There is no CPU fallback: if the library is not built the
first call raises.

The calls that launch kernels go through `_binding` (csrc/binding/pb_binding.cpp), which checks the usual
arguments and calls the library natively; the functions below of the same names take what it does not
(keywords, an explicit stream, wrong arguments) and raise the errors.  They serve every call where the extension
is not built, or was built for another torch or Python; a call then takes 6 to 8 us more of host time.
"""
from __future__ import annotations

import contextlib
import ctypes
import importlib
import os
import sys
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# PBATCH_LIB points the binding at another build of the same library (e.g. one compiled with other tuning macros)
LIB_PATH = os.environ.get("PBATCH_LIB") or os.path.join(_HERE, "libpbatch.so")

PB_OK, PB_EINVAL, PB_EALIGN, PB_ESIZE, PB_EHIP = 0, -1, -2, -3, -4
PB_MAX_BITS = 16
PB_MAX_COLS = 32768
PB_MAX_BATCH = 4096
PB_LAYOUT_ROWMAJOR_V1 = 0x50420001   # AND + popcount kernel
PB_LAYOUT_TILE16_V1 = 0x50420002     # matrix-core kernel (what pb_desc_init picks)
PB_LAYOUT_TILE16_GATES_V1 = 0x50420003   # the same with the four gate rows of an LSTM unit in one row tile
PB_LAYOUT_TILE16_PAIRS_V1 = 0x50420004   # the same with two bitlayers per word as base-4 digits (for serving batches)
PB_ACT_NONE, PB_ACT_RELU = 0, 1
PB_GATE_SIGMOID, PB_GATE_SILU, PB_GATE_GELU, PB_GATE_RELU = 0, 1, 2, 3
PB_TYPE_F32, PB_TYPE_BF16, PB_TYPE_F16 = 0, 1, 2
PB_MAX_ADAPTERS = 4096
PB_MAX_RANK = 256
PB_QUANT_SYMMETRIC, PB_QUANT_RANGE, PB_QUANT_SIGN, PB_QUANT_CLIP_SEARCH = 0, 1, 2, 3

EXPORTS = [
    "pb_desc_init", "pb_desc_init_layout", "pb_quantize_pack_desc", "pb_quantize_pack_mode", "pb_packed_bytes", "pb_workspace_bytes", "pb_quantize_pack", "pb_unpack", "pb_matmul",
    "pb_matmul_static", "pb_matmul_bias_act", "pb_matmul_acc", "pb_matmul_acc_pairs", "pb_act_prep", "pb_matmul_prepared", "pb_fixed_point", "pb_lstm_cell", "pb_strerror", "pb_last_hip_error",
    "pb_gated_linear", "pb_grad_workspace_bytes", "pb_matmul_grad", "pb_gated_linear_grad", "pb_adapters_workspace_bytes", "pb_matmul_adapters",
    "pb_matmul_adapters_grad",
]


class pb_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("bits", ctypes.c_int32),
                ("frac_bits", ctypes.c_int32), ("act_bits", ctypes.c_int32), ("layout", ctypes.c_uint32)]


class pb_adapters(ctypes.Structure):
    _fields_ = [("count", ctypes.c_int32), ("rank", ctypes.c_int32), ("type", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("scale", ctypes.c_void_p)]


class PbError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, strerror(status), status))


_lib = None
_P = ctypes.c_void_p
_I = ctypes.c_int
_D = ctypes.POINTER(pb_desc)
_A = ctypes.POINTER(pb_adapters)


def lib():
    """Load libpbatch.so (built by `python -m paper_2003_00822_amd.build`); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "HIP library %s is not built: run `python -m paper_2003_00822_amd.build` (no CPU fallback exists)"
                % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        L.pb_desc_init.argtypes = [_D, _I, _I, _I]
        L.pb_desc_init.restype = _I
        L.pb_desc_init_layout.argtypes = [_D, _I, _I, _I, ctypes.c_uint32]
        L.pb_desc_init_layout.restype = _I
        L.pb_quantize_pack_desc.argtypes = [_P, _D, _P, _P, _P]
        L.pb_quantize_pack_desc.restype = _I
        L.pb_quantize_pack_mode.argtypes = [_P, _D, _I, _P, _P, _P]
        L.pb_quantize_pack_mode.restype = _I
        L.pb_packed_bytes.argtypes = [_D]
        L.pb_packed_bytes.restype = ctypes.c_size_t
        L.pb_workspace_bytes.argtypes = [_D, _I]
        L.pb_workspace_bytes.restype = ctypes.c_size_t
        L.pb_quantize_pack.argtypes = [_P, _I, _I, _I, _P, _P, _P]
        L.pb_quantize_pack.restype = _I
        L.pb_unpack.argtypes = [_P, _D, _P, _P]
        L.pb_unpack.restype = _I
        L.pb_matmul.argtypes = [_P, _P, _D, _I, _P, _I, _P, _P, _P]
        L.pb_matmul.restype = _I
        L.pb_matmul_static.argtypes = [_P, _P, _D, _I, _P, _I, _P, _P]
        L.pb_matmul_static.restype = _I
        L.pb_matmul_bias_act.argtypes = [_P, _P, _D, _I, _P, _I, _P, _I, _P, _P, _P]
        L.pb_matmul_bias_act.restype = _I
        L.pb_matmul_acc.argtypes = [_P, _D, _I, _P, _I, _P, _P, _P]
        L.pb_matmul_acc.restype = _I
        L.pb_matmul_acc_pairs.argtypes = [_P, _D, _I, _P, _I, _P, _P, _P]
        L.pb_matmul_acc_pairs.restype = _I
        L.pb_act_prep.argtypes = [_D, _P, _I, _P, _P]
        L.pb_act_prep.restype = _I
        L.pb_matmul_prepared.argtypes = [_P, _P, _D, _I, _I, _P, _P, _P]
        L.pb_matmul_prepared.restype = _I
        L.pb_fixed_point.argtypes = [_D, _P, _I, _P, _P, _P]
        L.pb_fixed_point.restype = _I
        L.pb_lstm_cell.argtypes = [_P, _P, _D, _I, _P, _I, _P, _P, _P, _P, _P, _I, _P, _P]
        L.pb_lstm_cell.restype = _I
        L.pb_gated_linear.argtypes = [_P, _P, _D, _I, _P, _I, _P, _I, _P, _P, _P, _P]
        L.pb_gated_linear.restype = _I
        L.pb_grad_workspace_bytes.argtypes = [_D, _I]
        L.pb_grad_workspace_bytes.restype = ctypes.c_size_t
        L.pb_matmul_grad.argtypes = [_P, _P, _D, _I, _P, _I, _P, _P, _P]
        L.pb_matmul_grad.restype = _I
        L.pb_gated_linear_grad.argtypes = [_P, _P, _D, _I, _P, _P, _I, _I, _P, _P, _P, _P]
        L.pb_gated_linear_grad.restype = _I
        L.pb_adapters_workspace_bytes.argtypes = [_D, _A, _I]
        L.pb_adapters_workspace_bytes.restype = ctypes.c_size_t
        L.pb_matmul_adapters.argtypes = [_P, _P, _D, _I, _P, _I, _A, _P, _P, _P, _P, _P]
        L.pb_matmul_adapters.restype = _I
        L.pb_matmul_adapters_grad.argtypes = [_P, _P, _D, _I, _P, _P, _I, _A, _P, _P, _P, _P, _P, _P]
        L.pb_matmul_adapters_grad.restype = _I
        L.pb_strerror.argtypes = [_I]
        L.pb_strerror.restype = ctypes.c_char_p
        L.pb_last_hip_error.argtypes = []
        L.pb_last_hip_error.restype = _I
        binding, why_not = _use_binding()   # (once more: it may have been built since this module was imported)
        if binding is not None:
            binding.bind(pb_desc, pb_adapters, PbError,
                         {n: ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in _NATIVE + _NATIVE_OPERATORS + _SIZES})
        else:
            warnings.warn("calls go through ctypes, 6 to 8 us slower each: %s (python -m paper_2003_00822_amd.build)"
                          % why_not, RuntimeWarning, stacklevel=2)
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().pb_strerror(int(status)).decode()


def _check(status, where):
    if status != PB_OK:
        raise PbError(status, where)


def _ptr(t, dtype, name):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA/HIP tensor" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


def pb_desc_init(rows: int, cols: int, bits: int, frac_bits: int = 16, act_bits: int = 32) -> pb_desc:
    d = pb_desc()
    _check(lib().pb_desc_init(ctypes.byref(d), rows, cols, bits), "pb_desc_init")
    d.frac_bits = frac_bits
    d.act_bits = act_bits
    return d


def pb_desc_init_layout(rows: int, cols: int, bits: int, layout: int, frac_bits: int = 16,
                        act_bits: int = 32) -> pb_desc:
    d = pb_desc()
    _check(lib().pb_desc_init_layout(ctypes.byref(d), rows, cols, bits, layout), "pb_desc_init_layout")
    d.frac_bits = frac_bits
    d.act_bits = act_bits
    return d


def pb_packed_bytes(d: pb_desc) -> int:
    return int(lib().pb_packed_bytes(ctypes.byref(d)))


def pb_workspace_bytes(d: pb_desc, batch: int) -> int:
    return int(lib().pb_workspace_bytes(ctypes.byref(d), batch))


def alloc_packed(d: pb_desc, device="cuda") -> torch.Tensor:
    return torch.empty(pb_packed_bytes(d), dtype=torch.uint8, device=device)


def alloc_workspace(d: pb_desc, batch: int, device="cuda") -> torch.Tensor:
    return torch.empty(pb_workspace_bytes(d, batch), dtype=torch.uint8, device=device)


def pb_quantize_pack(W, rows, cols, bits, packed, scales, stream=None):
    _check(lib().pb_quantize_pack(_ptr(W, torch.float32, "W"), rows, cols, bits, _ptr(packed, torch.uint8, "packed"),
                                  _ptr(scales, torch.float32, "scales"), _stream(stream)), "pb_quantize_pack")


def pb_quantize_pack_desc(W, d, packed, scales, stream=None):
    _check(lib().pb_quantize_pack_desc(_ptr(W, torch.float32, "W"), ctypes.byref(d),
                                       _ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"),
                                       _stream(stream)), "pb_quantize_pack_desc")


def pb_quantize_pack_mode(W, d, quantizer, packed, scales, stream=None):
    _check(lib().pb_quantize_pack_mode(_ptr(W, torch.float32, "W"), ctypes.byref(d), quantizer,
                                       _ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"),
                                       _stream(stream)), "pb_quantize_pack_mode")


def pb_unpack(packed, d, q, stream=None):
    _check(lib().pb_unpack(_ptr(packed, torch.uint8, "packed"), ctypes.byref(d), _ptr(q, torch.int32, "q"),
                           _stream(stream)), "pb_unpack")


def pb_matmul(packed, scales, d, bits_used, X, batch, Y, workspace, stream=None):
    _check(lib().pb_matmul(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"),
                           ctypes.byref(d), bits_used, _ptr(X, torch.float32, "X"), batch,
                           _ptr(Y, torch.float32, "Y"), _ptr(workspace, torch.uint8, "workspace"),
                           _stream(stream)), "pb_matmul")


def pb_matmul_static(packed, scales, d, bits_used, X, batch, Y, stream=None):
    _check(lib().pb_matmul_static(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"),
                                  ctypes.byref(d), bits_used, _ptr(X, torch.float32, "X"), batch,
                                  _ptr(Y, torch.float32, "Y"), _stream(stream)), "pb_matmul_static")


def pb_matmul_bias_act(packed, scales, d, bits_used, X, batch, bias, act, Y, workspace, stream=None):
    _check(lib().pb_matmul_bias_act(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"),
                                    ctypes.byref(d), bits_used, _ptr(X, torch.float32, "X"), batch,
                                    _ptr(bias, torch.float32, "bias"), act, _ptr(Y, torch.float32, "Y"),
                                    _ptr(workspace, torch.uint8, "workspace"), _stream(stream)),
           "pb_matmul_bias_act")


def pb_matmul_acc(packed, d, bits_used, X, batch, A, workspace, stream=None):
    _check(lib().pb_matmul_acc(_ptr(packed, torch.uint8, "packed"), ctypes.byref(d), bits_used,
                               _ptr(X, torch.float32, "X"), batch, _ptr(A, torch.int64, "A"),
                               _ptr(workspace, torch.uint8, "workspace"), _stream(stream)), "pb_matmul_acc")


def pb_matmul_acc_pairs(packed, d, bits_used, X, batch, A, workspace, stream=None):
    _check(lib().pb_matmul_acc_pairs(_ptr(packed, torch.uint8, "packed"), ctypes.byref(d), bits_used,
                                     _ptr(X, torch.float32, "X"), batch, _ptr(A, torch.int64, "A"),
                                     _ptr(workspace, torch.uint8, "workspace"), _stream(stream)),
           "pb_matmul_acc_pairs")


def pb_act_prep(d, X, batch, workspace, stream=None):
    _check(lib().pb_act_prep(ctypes.byref(d), _ptr(X, torch.float32, "X"), batch,
                             _ptr(workspace, torch.uint8, "workspace"), _stream(stream)), "pb_act_prep")


def pb_matmul_prepared(packed, scales, d, bits_used, batch, Y, workspace, stream=None):
    _check(lib().pb_matmul_prepared(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"),
                                    ctypes.byref(d), bits_used, batch, _ptr(Y, torch.float32, "Y"),
                                    _ptr(workspace, torch.uint8, "workspace"), _stream(stream)),
           "pb_matmul_prepared")


def pb_fixed_point(d, X, batch, xq, workspace, stream=None):
    _check(lib().pb_fixed_point(ctypes.byref(d), _ptr(X, torch.float32, "X"), batch, _ptr(xq, torch.int32, "xq"),
                                _ptr(workspace, torch.uint8, "workspace"), _stream(stream)), "pb_fixed_point")


def pb_lstm_cell(packed, scales, d, bits_used, x_t, input_size, h_prev, c_prev, bias, h_out, c_out, batch, workspace,
                 stream=None):
    _check(lib().pb_lstm_cell(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"),
                              ctypes.byref(d), bits_used, _ptr(x_t, torch.float32, "x_t"), input_size,
                              _ptr(h_prev, torch.float32, "h_prev"), _ptr(c_prev, torch.float32, "c_prev"),
                              _ptr(bias, torch.float32, "bias"), _ptr(h_out, torch.float32, "h_out"),
                              _ptr(c_out, torch.float32, "c_out"), batch,
                              _ptr(workspace, torch.uint8, "workspace"), _stream(stream)), "pb_lstm_cell")


def pb_grad_workspace_bytes(d: pb_desc, batch: int) -> int:
    return int(lib().pb_grad_workspace_bytes(ctypes.byref(d), batch))


def pb_adapters_workspace_bytes(d: pb_desc, adapters: pb_adapters, batch: int) -> int:
    return int(lib().pb_adapters_workspace_bytes(ctypes.byref(d), ctypes.byref(adapters), batch))


def pb_gated_linear(packed, scales, d, bits_used, X, batch, bias, gate, H, pre, workspace, stream=None):
    _check(lib().pb_gated_linear(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"), ctypes.byref(d), bits_used,
                                 _ptr(X, torch.float32, "X"), batch, _ptr(bias, torch.float32, "bias"), gate,
                                 _ptr(H, torch.float32, "H"), _ptr(pre, torch.float32, "pre"),
                                 _ptr(workspace, torch.uint8, "workspace"), _stream(stream)), "pb_gated_linear")


def pb_matmul_grad(packed, scales, d, bits_used, dY, batch, dX, workspace, stream=None):
    _check(lib().pb_matmul_grad(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"), ctypes.byref(d), bits_used,
                                _ptr(dY, torch.float32, "dY"), batch, _ptr(dX, torch.float32, "dX"),
                                _ptr(workspace, torch.uint8, "workspace"), _stream(stream)), "pb_matmul_grad")


def pb_gated_linear_grad(packed, scales, d, bits_used, pre, dH, batch, gate, dpre, dX, workspace, stream=None):
    _check(lib().pb_gated_linear_grad(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"), ctypes.byref(d), bits_used,
                                      _ptr(pre, torch.float32, "pre"), _ptr(dH, torch.float32, "dH"), batch, gate,
                                      _ptr(dpre, torch.float32, "dpre"), _ptr(dX, torch.float32, "dX"),
                                      _ptr(workspace, torch.uint8, "workspace"), _stream(stream)), "pb_gated_linear_grad")


def pb_matmul_adapters(packed, scales, d, bits_used, X, batch, adapters, index, bias, Y, workspace, stream=None):
    _check(lib().pb_matmul_adapters(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"), ctypes.byref(d), bits_used,
                                    _ptr(X, torch.float32, "X"), batch, ctypes.byref(adapters), _ptr(index, torch.int32, "index"),
                                    _ptr(bias, torch.float32, "bias"), _ptr(Y, torch.float32, "Y"),
                                    _ptr(workspace, torch.uint8, "workspace"), _stream(stream)), "pb_matmul_adapters")


def pb_matmul_adapters_grad(packed, scales, d, bits_used, X, dY, batch, adapters, index, dX, dA, dB, workspace, stream=None):
    _check(lib().pb_matmul_adapters_grad(_ptr(packed, torch.uint8, "packed"), _ptr(scales, torch.float32, "scales"), ctypes.byref(d),
                                         bits_used, _ptr(X, torch.float32, "X"), _ptr(dY, torch.float32, "dY"), batch,
                                         ctypes.byref(adapters), _ptr(index, torch.int32, "index"), _ptr(dX, torch.float32, "dX"),
                                         _ptr(dA, torch.float32, "dA"), _ptr(dB, torch.float32, "dB"),
                                         _ptr(workspace, torch.uint8, "workspace"), _stream(stream)), "pb_matmul_adapters_grad")


_TYPES = {torch.float32: PB_TYPE_F32, torch.bfloat16: PB_TYPE_BF16, torch.float16: PB_TYPE_F16}


class Adapters:
    """Low-rank adapters of one layer, of many requests: adapter k adds scale[k] B[k] A[k] to its matrix.  A [count, rank, cols] and B [count,
    rows, rank] of one type (float32, bfloat16, float16), scale [count] float32 or None for 1."""

    def __init__(self, A: torch.Tensor, B: torch.Tensor, scale: torch.Tensor | None = None):
        if A.dtype not in _TYPES or B.dtype != A.dtype:
            raise TypeError("A and B must both be float32, bfloat16 or float16, got %s and %s" % (A.dtype, B.dtype))
        if A.dim() != 3 or B.dim() != 3 or A.shape[0] != B.shape[0] or A.shape[1] != B.shape[2]:
            raise ValueError("A [count, rank, cols] and B [count, rows, rank], got %s and %s" % (tuple(A.shape), tuple(B.shape)))
        if scale is not None and scale.shape != (A.shape[0],):
            raise ValueError("scale [count], got %s" % (tuple(scale.shape),))
        self.A, self.B, self.scale = A, B, scale
        self.count, self.rank, self.cols = A.shape
        self.rows = B.shape[1]
        self.desc()

    def desc(self) -> pb_adapters:
        """The tensors as they are now (an optimizer may have put others in their place)."""
        A, B = self.A, self.B
        if A.dtype not in _TYPES or A.shape != (self.count, self.rank, self.cols) or B.shape != (self.count, self.rows, self.rank):
            raise ValueError("A or B has another type or shape than it had")
        return pb_adapters(self.count, self.rank, _TYPES[A.dtype], 0, _ptr(A, None, "A"), _ptr(B, A.dtype, "B"),
                           _ptr(self.scale, torch.float32, "scale"))


class PackedLinear:
    """Convenience holder: one quantized, packed weight matrix with its scales and a workspace."""

    def __init__(self, W: torch.Tensor, bits: int, max_batch: int = 1, frac_bits: int = 16, act_bits: int = 32,
                 layout: int | None = None, quantizer: int = PB_QUANT_SYMMETRIC):
        assert W.is_cuda and W.dtype == torch.float32 and W.dim() == 2
        W = W.contiguous()
        self.rows, self.cols = W.shape
        self.bits = bits
        if layout is None:
            self.desc = pb_desc_init(self.rows, self.cols, bits, frac_bits, act_bits)
        else:
            self.desc = pb_desc_init_layout(self.rows, self.cols, bits, layout, frac_bits, act_bits)
        self.packed = alloc_packed(self.desc, W.device)
        self.scales = torch.empty(max(bits, 4), dtype=torch.float32, device=W.device)
        self.max_batch = max_batch
        self.workspace = alloc_workspace(self.desc, max_batch, W.device)
        self.home_stream = torch.cuda.current_stream().cuda_stream   # whose eager calls share `workspace`
        pb_quantize_pack_mode(W, self.desc, quantizer, self.packed, self.scales)

    def __call__(self, X: torch.Tensor, bits_used: int | None = None, out: torch.Tensor | None = None):
        return _linear(self, X, bits_used, out)

    def _call_checked(self, X, bits_used, out):
        X = X.reshape(-1, self.cols)
        batch = X.shape[0]
        assert batch <= self.max_batch
        if out is None:
            out = torch.empty((batch, self.rows), dtype=torch.float32, device=X.device)
        # (a workspace of its own: another thread's call could come between the launches of this one)
        pb_matmul(self.packed, self.scales, self.desc, bits_used or self.bits, X, batch, out, torch.empty_like(self.workspace))
        return out

    def acc(self, X: torch.Tensor, bits_used: int | None = None):
        X = X.reshape(-1, self.cols)
        batch = X.shape[0]
        m = bits_used or self.bits
        A = torch.empty((m, batch, self.rows), dtype=torch.int64, device=X.device)
        pb_matmul_acc(self.packed, self.desc, m, X, batch, A, torch.empty_like(self.workspace))
        return A

    def acc_pairs(self, X: torch.Tensor, bits_used: int | None = None):
        X = X.reshape(-1, self.cols)
        batch = X.shape[0]
        m = bits_used or self.bits
        A = torch.empty(((m + 1) // 2, batch, self.rows), dtype=torch.int64, device=X.device)
        pb_matmul_acc_pairs(self.packed, self.desc, m, X, batch, A, torch.empty_like(self.workspace))
        return A

    # The calls below have workspaces of their own: they take any stream and thread, and a captured graph keeps its own.  Like __call__ they know nothing of
    # autograd: what they return has no history, also where an input requires a gradient; gated_grad, grad and adapted_grad are the backward passes.

    def gated(self, X: torch.Tensor, gate: int = PB_GATE_SILU, bits_used: int | None = None, bias: torch.Tensor | None = None,
              keep: bool = False):
        """H = act(g) u with [g; u] = W x + bias: the block's two projections packed as one matrix, gate rows first.  With `keep` also the
        pre-activations [g; u], for gated_grad.  The results have no autograd history."""
        return _methods["gated"](self, X, gate, bits_used, bias, keep)

    def gated_grad(self, pre: torch.Tensor, dH: torch.Tensor, gate: int = PB_GATE_SILU, bits_used: int | None = None):
        """(dX, dpre) of `gated`, from the pre-activations that it kept."""
        return _methods["gated_grad"](self, pre, dH, gate, bits_used)

    def grad(self, dY: torch.Tensor, bits_used: int | None = None):
        """dX = dY W: the gradient of the layer's activations, through the first `bits_used` bitlayers."""
        return _methods["grad"](self, dY, bits_used)

    def adapted(self, X: torch.Tensor, adapters: Adapters, index: torch.Tensor | None, bits_used: int | None = None,
                bias: torch.Tensor | None = None):
        """W x + bias + scale_k B_k A_k x with k = index[n] (int32; outside [0, count): no adapter; None: adapter 0 for all).  The result has no autograd
        history: the gradients of x, A and B are adapted_grad."""
        return _methods["adapted"](self, X, adapters, index, bits_used, bias)

    def adapted_grad(self, X: torch.Tensor, dY: torch.Tensor, adapters: Adapters, index: torch.Tensor | None, bits_used: int | None = None,
                     inputs: bool = True):
        """(dX, dA, dB) of `adapted`, all fp32; dX is None without `inputs`."""
        return _methods["adapted_grad"](self, X, dY, adapters, index, bits_used, inputs)

    def _gated_checked(self, X, gate, bits_used, bias, keep):
        X = self._vectors(X, self.cols, "X")
        n = X.shape[0]
        self._sized(bias, "bias", (self.rows,))
        with self._here(X, bias):
            H = torch.empty((n, self.rows // 2), dtype=torch.float32, device=X.device)
            pre = torch.empty((n, self.rows), dtype=torch.float32, device=X.device) if keep else None
            pb_gated_linear(self.packed, self.scales, self.desc, self.bits if bits_used is None else bits_used, X, n, bias, gate, H, pre,
                            self._work(pb_workspace_bytes(self.desc, n)))
        return (H, pre) if keep else H

    def _gated_grad_checked(self, pre, dH, gate, bits_used):
        pre, dH = self._vectors(pre, self.rows, "pre"), self._vectors(dH, self.rows // 2, "dH")
        n = pre.shape[0]
        self._sized(dH, "dH", (n, self.rows // 2))
        with self._here(pre, dH):
            dX = torch.empty((n, self.cols), dtype=torch.float32, device=pre.device)
            dpre = torch.empty_like(pre)
            pb_gated_linear_grad(self.packed, self.scales, self.desc, self.bits if bits_used is None else bits_used, pre, dH, n, gate, dpre, dX,
                                 self._work(pb_grad_workspace_bytes(self.desc, n)))
        return dX, dpre

    def _grad_checked(self, dY, bits_used):
        dY = self._vectors(dY, self.rows, "dY")
        n = dY.shape[0]
        with self._here(dY):
            dX = torch.empty((n, self.cols), dtype=torch.float32, device=dY.device)
            pb_matmul_grad(self.packed, self.scales, self.desc, self.bits if bits_used is None else bits_used, dY, n, dX,
                           self._work(pb_grad_workspace_bytes(self.desc, n)))
        return dX

    def _adapted_checked(self, X, adapters, index, bits_used, bias):
        X = self._vectors(X, self.cols, "X")
        n = X.shape[0]
        self._sized(index, "index", (n,))
        self._sized(bias, "bias", (self.rows,))
        with self._here(X, index, bias, adapters.A, adapters.B, adapters.scale):
            desc = self._desc_of(adapters)
            Y = torch.empty((n, self.rows), dtype=torch.float32, device=X.device)
            pb_matmul_adapters(self.packed, self.scales, self.desc, self.bits if bits_used is None else bits_used, X, n, desc, index, bias, Y,
                               self._work(pb_adapters_workspace_bytes(self.desc, desc, n)))
        return Y

    def _adapted_grad_checked(self, X, dY, adapters, index, bits_used, inputs):
        X, dY = self._vectors(X, self.cols, "X"), self._vectors(dY, self.rows, "dY")
        n = X.shape[0]
        self._sized(dY, "dY", (n, self.rows))
        self._sized(index, "index", (n,))
        with self._here(X, dY, index, adapters.A, adapters.B, adapters.scale):
            desc = self._desc_of(adapters)
            dX = torch.empty((n, self.cols), dtype=torch.float32, device=X.device) if inputs else None
            dA = torch.empty(adapters.A.shape, dtype=torch.float32, device=X.device)
            dB = torch.empty(adapters.B.shape, dtype=torch.float32, device=X.device)
            pb_matmul_adapters_grad(self.packed, self.scales, self.desc, self.bits if bits_used is None else bits_used, X, dY, n, desc, index,
                                    dX, dA, dB, self._work(pb_adapters_workspace_bytes(self.desc, desc, n)))
        return dX, dA, dB

    def _vectors(self, t, length, name):
        if t.dim() < 1 or t.shape[-1] != length:
            raise ValueError("%s must have vectors of %d values, got %s" % (name, length, tuple(t.shape)))
        return t if t.dim() == 2 else t.reshape(-1, length)

    @staticmethod
    def _sized(t, name, shape):
        if t is not None and t.shape != shape:
            raise ValueError("%s must have the shape %s, got %s" % (name, shape, tuple(t.shape)))

    def _desc_of(self, adapters):
        if (adapters.rows, adapters.cols) != (self.rows, self.cols):
            raise ValueError("adapters of a layer %d x %d, the layer is %d x %d" % (adapters.rows, adapters.cols, self.rows, self.cols))
        return adapters.desc()

    def _here(self, *tensors):
        """The layer's device as the current one; all tensors are on it."""
        device = self.packed.device
        for t in tensors:
            if t is not None and t.device != device:
                raise ValueError("a tensor is on %s, the layer on %s" % (t.device, device))
        return contextlib.nullcontext() if device.index == torch.cuda.current_device() else torch.cuda.device(device)

    def _work(self, size):
        # (a size of 0: the call is refused, and says why)
        return torch.empty(max(size, 16), dtype=torch.uint8, device=self.packed.device)

    def unpack(self):
        q = torch.empty((self.rows, self.cols), dtype=torch.int32, device=self.packed.device)
        pb_unpack(self.packed, self.desc, q)
        return q


# The functions above stay behind the native ones (same arguments and results); `_linear` is PackedLinear's call.
_NATIVE = ["pb_quantize_pack", "pb_quantize_pack_desc", "pb_quantize_pack_mode", "pb_unpack", "pb_matmul",
           "pb_matmul_static", "pb_matmul_bias_act", "pb_matmul_acc", "pb_matmul_acc_pairs", "pb_act_prep",
           "pb_matmul_prepared", "pb_fixed_point", "pb_lstm_cell"]
_NATIVE_OPERATORS = ["pb_gated_linear", "pb_matmul_grad", "pb_gated_linear_grad", "pb_matmul_adapters", "pb_matmul_adapters_grad"]
_SIZES = ["pb_workspace_bytes", "pb_grad_workspace_bytes", "pb_adapters_workspace_bytes"]
_linear = PackedLinear._call_checked
# PackedLinear's operators, by their names
_methods = {n: getattr(PackedLinear, "_%s_checked" % n) for n in ("gated", "gated_grad", "grad", "adapted", "adapted_grad")}
_PYTHON = {**{n: globals()[n] for n in _NATIVE + _NATIVE_OPERATORS}, "linear": _linear, **_methods}


def _use_binding():
    """Put the native functions in front of the Python ones: (the extension, None), or (None, why it is not used)."""
    importlib.invalidate_caches()
    try:
        binding = importlib.import_module(__package__ + "._binding")
    except ImportError as e:
        return None, "no native binding (%s)" % e
    here = "%s %s" % (torch.__version__, sys.implementation.cache_tag)
    if getattr(binding, "BUILT_FOR", None) != here:   # (it takes tensors apart by torch's headers)
        return None, "the native binding is built for %s, not for %s" % (getattr(binding, "BUILT_FOR", "?"), here)
    if not all(hasattr(binding, n) for n in [*_NATIVE, *_NATIVE_OPERATORS, *_methods]):
        return None, "the native binding is built from other sources"
    binding.set_slow(_PYTHON)
    globals().update({n: getattr(binding, n) for n in _NATIVE + _NATIVE_OPERATORS})
    globals()["_linear"] = binding.linear
    globals()["_methods"] = {n: getattr(binding, n) for n in _methods}
    return binding, None


_use_binding()
