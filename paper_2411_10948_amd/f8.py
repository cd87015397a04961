"""Dense linear layers in 8-bit floating point with a scale for each block of 128,
trained or served (include/shiftquant.h has the formats, formulas and layouts).

As in the ``mx`` module, ``sq_*`` marshal torch tensors to the C entry points one
to one, and ``LinearPlan`` keeps the buffers of a fixed shape: its calls only
enqueue work.
"""
from __future__ import annotations

import ctypes as ct
import dataclasses
import functools
from typing import Optional, Tuple

import torch

from .mx import TYPE_F32, _TYPES, _checked, _gpu_of, _of_layer, _on, _rows, _shape, _sized, _type, _workspace
from .norm import _fixed
from .shiftquant import _I64, _P, _SZ, _check, _ptr, _stream, _ws_ptr, load


@dataclasses.dataclass
class F8Matrix:
    """A matrix [rows, cols] in 8-bit codes with a scale for each block of 128"""
    codes: torch.Tensor
    scales: torch.Tensor
    rows: int
    cols: int

    def __post_init__(self):
        for t, size, name in zip((self.codes, self.scales), sq_f8_size(self.rows, self.cols), ("codes", "scales")):
            if t.dtype != torch.uint8 or not t.is_contiguous() or t.numel() < size:
                raise ValueError(f"{name}: expected at least {size} contiguous uint8 values")
        if self.codes.device != self.scales.device:
            raise ValueError("codes and scales are on different devices")

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "F8Matrix":
        nc, ns = sq_f8_size(rows, cols)
        return cls(torch.empty(nc, dtype=torch.uint8, device=device), torch.empty(ns, dtype=torch.uint8, device=device), rows, cols)

    def values(self, dtype=torch.float32, stream=None) -> torch.Tensor:
        """The values that the codes stand for."""
        out = torch.empty((self.rows, self.cols), dtype=dtype, device=self.codes.device)
        sq_f8_dequantize(self.codes, self.scales, self.rows, self.cols, out, stream)
        return out


# ---------------------------------------------------------------------------
# one-to-one wrappers of the C entry points
# ---------------------------------------------------------------------------
def sq_f8_size(rows: int, cols: int) -> Tuple[int, int]:
    """(bytes of the codes, bytes of the scales)"""
    a, b = _SZ(0), _SZ(0)
    _check("sq_f8_size", load().sq_f8_size(rows, cols, ct.byref(a), ct.byref(b)))
    return a.value, b.value


_f8_size = functools.lru_cache(maxsize=1024)(sq_f8_size)     # of the arguments alone


def _f8(codes, scales, rows: int, cols: int, name: str):
    return _sized(codes, scales, _f8_size(rows, cols), name)


def sq_f8_quantize(X, square, codes, scales, codes_t, scales_t, stream=None) -> None:
    rows, cols = X.shape
    _check("sq_f8_quantize", load().sq_f8_quantize(
        _ptr(X), _type(X), rows, cols, _rows(X, "X"), int(square), *_f8(codes, scales, rows, cols, "codes"),
        *_f8(codes_t, scales_t, cols, rows, "codes_t"), _stream(stream)))


def sq_f8_dequantize(codes, scales, rows, cols, out, stream=None) -> None:
    _shape(out, (rows, cols), "out")
    _check("sq_f8_dequantize", load().sq_f8_dequantize(
        *_f8(codes, scales, rows, cols, "codes"), rows, cols, _ptr(out), _type(out), _rows(out, "out"), _stream(stream)))


def sq_f8_gemm_workspace_size(M: int, N: int, K: int) -> int:
    nb = _SZ(0)
    _check("sq_f8_gemm_workspace_size", load().sq_f8_gemm_workspace_size(M, N, K, ct.byref(nb)))
    return nb.value


def sq_f8_gemm(A, A_scales, B, B_scales, K, C, workspace=None, stream=None) -> None:
    M, N = C.shape
    ws, nws = _ws_ptr(workspace)
    _check("sq_f8_gemm", load().sq_f8_gemm(
        *_f8(A, A_scales, M, K, "A"), *_f8(B, B_scales, N, K, "B"), M, N, K, _ptr(C), _type(C), _rows(C, "C"), ws, nws,
        _stream(stream)))


def sq_f8_linear_workspace_size(M: int, K: int, N: int) -> int:
    nb = _SZ(0)
    _check("sq_f8_linear_workspace_size", load().sq_f8_linear_workspace_size(M, K, N, ct.byref(nb)))
    return nb.value


def sq_f8_linear(X, W, W_scales, Y, workspace=None, stream=None) -> None:
    (M, K), N = X.shape, Y.shape[1]
    _shape(Y, (M, N), "Y")
    ws, nws = _ws_ptr(workspace)
    _check("sq_f8_linear", load().sq_f8_linear(
        _ptr(X), _type(X), M, K, _rows(X, "X"), *_f8(W, W_scales, N, K, "W"), N, _ptr(Y), _type(Y), _rows(Y, "Y"), ws, nws,
        _stream(stream)))


class Layer(ct.Structure):
    """sq_f8_layer"""
    _fields_ = ([(n, _I64) for n in ("rows", "c_in", "c_out")] + [("type", ct.c_int32), ("reserved", ct.c_int32)]
                + [(m + s, ct.c_void_p) for m in ("w", "w_t", "x", "x_t", "dy", "dy_t") for s in ("", "_scales")]
                + [("workspace", ct.c_void_p), ("workspace_bytes", _SZ)])


def sq_f8_layer_workspace_size(layer: Layer) -> int:
    nb = _SZ(0)
    _check("sq_f8_layer_workspace_size", load().sq_f8_layer_workspace_size(ct.addressof(layer), ct.byref(nb)))
    return nb.value


def sq_f8_layer_weight(layer: Layer, W, stream=None) -> None:
    _check("sq_f8_layer_weight", load().sq_f8_layer_weight(
        ct.addressof(layer), _of_layer(layer, W, (layer.c_out, layer.c_in), "W"), _rows(W, "W"), _stream(stream)))


def sq_f8_layer_forward(layer: Layer, X, Y, stream=None) -> None:
    _check("sq_f8_layer_forward", load().sq_f8_layer_forward(
        ct.addressof(layer), _of_layer(layer, X, (layer.rows, layer.c_in), "X"), _rows(X, "X"),
        _of_layer(layer, Y, (layer.rows, layer.c_out), "Y"), _rows(Y, "Y"), _stream(stream)))


def sq_f8_layer_backward(layer: Layer, dY, dX, dW, stream=None) -> None:
    _check("sq_f8_layer_backward", load().sq_f8_layer_backward(
        ct.addressof(layer), _of_layer(layer, dY, (layer.rows, layer.c_out), "dY"), _rows(dY, "dY"),
        _of_layer(layer, dX, (layer.rows, layer.c_in), "dX"), _rows(dX, "dX"),
        _of_layer(layer, dW, (layer.c_out, layer.c_in), "dW", TYPE_F32), _rows(dW, "dW"), _stream(stream)))


# ---------------------------------------------------------------------------
# layers
# ---------------------------------------------------------------------------
def quantize(X: torch.Tensor, square: bool = False, rows: bool = True, cols: bool = False,
             stream=None) -> Tuple[Optional[F8Matrix], Optional[F8Matrix]]:
    """Codes of X [rows, cols] with blocks along its columns (``rows``: the operand X) and
    along its rows (``cols``: the operand X^T), in one read; ``square``: in blocks of 128 x 128,
    as a layer's weights are held."""
    M, C = X.shape
    a = F8Matrix.empty(M, C, X.device) if rows else None
    t = F8Matrix.empty(C, M, X.device) if cols else None
    sq_f8_quantize(X, square, a and a.codes, a and a.scales, t and t.codes, t and t.scales, stream)
    return a, t


class LinearPlan:
    """A linear layer Y = X W^T on M rows with 8-bit operands, all of its buffers allocated
    once.

    Serving: ``forward(x, w)`` with W's codes (``quantize(W, square=True)[0]``).  Training
    (``train=True``): ``quantize_weight(W)``, ``forward(x)``, then ``backward(dy)``, which gives dX in
    the layer's type and dW in float32.  Results are the plan's buffers, overwritten by its next
    call of the same kind."""

    def __init__(self, M: int, C_in: int, C_out: int, dtype=torch.bfloat16, train: bool = False, device="cuda"):
        if dtype not in _TYPES:
            raise TypeError(f"dtype: expected float32 or bfloat16, got {dtype}")
        dev = torch.device(device)
        nbytes = sq_f8_linear_workspace_size(M, C_in, C_out)    # refuses sizes that the calls refuse
        self.M, self.C_in, self.C_out, self.dtype, self.train = M, C_in, C_out, dtype, train
        self._x_shape, self._y_shape, self._w_shape = torch.Size((M, C_in)), torch.Size((M, C_out)), torch.Size((C_out, C_in))
        self.Y = torch.empty(self._y_shape, dtype=dtype, device=dev)
        self._lib, self._gpu = load(), _gpu_of(self.Y)
        y, ld = (_P, self.Y.data_ptr()), (_I64, max(C_out, 1))
        self._has_weight = self._has_input = False
        if not train:
            self.ws = _workspace(nbytes, dev)
            kind, (ws, nws) = (ct.c_int32, _TYPES[dtype]), _ws_ptr(self.ws)
            self._size = _fixed(kind, (_I64, M), (_I64, C_in))
            self._to = _fixed((_I64, C_out), y, kind, ld, (_P, ws), (_SZ, nws))
            self._held = [self.Y, self.ws]      # the pointers kept stay valid as long as the plan
            return
        self.w, self.w_t = F8Matrix.empty(C_out, C_in, dev), F8Matrix.empty(C_in, C_out, dev)
        self.x, self.x_t = F8Matrix.empty(M, C_in, dev), F8Matrix.empty(C_in, M, dev)
        self.dy, self.dy_t = F8Matrix.empty(M, C_out, dev), F8Matrix.empty(C_out, M, dev)
        self.dX = torch.empty(self._x_shape, dtype=dtype, device=dev)
        self.dW = torch.empty(self._w_shape, dtype=torch.float32, device=dev)
        self.layer = Layer(M, C_in, C_out, _TYPES[dtype], 0)
        self._held = [self.Y, self.dX, self.dW]     # the layer's pointers stay valid as long as the plan
        for name in ("w", "w_t", "x", "x_t", "dy", "dy_t"):
            m = getattr(self, name)
            self._held += [m.codes, m.scales]
            setattr(self.layer, name, m.codes.data_ptr())
            setattr(self.layer, name + "_scales", m.scales.data_ptr())
        self._layer_ptr, = _fixed((_P, ct.addressof(self.layer)))
        ld_in = _I64, max(C_in, 1)
        self._to, self._to_back = _fixed(y, ld), _fixed((_P, self.dX.data_ptr()), ld_in, (_P, self.dW.data_ptr()), ld_in)
        self.ws = _workspace(sq_f8_layer_workspace_size(self.layer), dev)
        if self.ws is not None:
            self._held.append(self.ws)
            self.layer.workspace, self.layer.workspace_bytes = self.ws.data_ptr(), self.ws.nbytes

    def quantize_weight(self, W: torch.Tensor, stream=None) -> None:
        """W [C_out, C_in], in the layer's type: after every update of the weights"""
        if not self.train:
            raise ValueError("quantize_weight needs a plan with train=True")
        ld = _checked(W, self._w_shape, self.dtype, self._gpu, "W")
        st = self._lib.sq_f8_layer_weight(self._layer_ptr, W.data_ptr(), ld, _on(self._gpu, stream))
        if st:
            _check("sq_f8_layer_weight", st)
        self._has_weight = True

    def forward(self, x: torch.Tensor, w: Optional[F8Matrix] = None, stream=None) -> torch.Tensor:
        ld = _checked(x, self._x_shape, self.dtype, self._gpu, "x")
        if self.train:
            if w is not None:
                raise ValueError("w: a training plan has its own codes (quantize_weight)")
            if not self._has_weight:
                raise ValueError("forward needs a quantize_weight before it")
            st = self._lib.sq_f8_layer_forward(self._layer_ptr, x.data_ptr(), ld, *self._to, _on(self._gpu, stream))
            if st:
                _check("sq_f8_layer_forward", st)
            self._has_input = True
            return self.Y
        if w is None or w.rows != self.C_out or w.cols != self.C_in:
            raise ValueError(f"w: expected codes of [{self.C_out}, {self.C_in}]")
        codes = w.codes
        if codes.get_device() != self._gpu:
            raise ValueError("w: expected codes on the plan's GPU")
        st = self._lib.sq_f8_linear(
            x.data_ptr(), *self._size, ld, codes.data_ptr(), w.scales.data_ptr(), *self._to, _on(self._gpu, stream))
        if st:
            _check("sq_f8_linear", st)
        return self.Y

    def backward(self, dy: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(dX, dW) of the last forward"""
        if not self.train:
            raise ValueError("backward needs a plan with train=True")
        ld = _checked(dy, self._y_shape, self.dtype, self._gpu, "dy")
        if not self._has_input:
            raise ValueError("backward needs a forward before it")
        st = self._lib.sq_f8_layer_backward(self._layer_ptr, dy.data_ptr(), ld, *self._to_back, _on(self._gpu, stream))
        if st:
            _check("sq_f8_layer_backward", st)
        return self.dX, self.dW
