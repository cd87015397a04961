"""Microscaled 4-bit linear layers, dense or by expert, and activations whose
backward pass reads an 8-bit copy of their input (include/shiftquant.h has the
formats, formulas and layouts).

As in the ``shiftquant`` module, the functions named ``sq_*`` marshal torch
tensors to the C entry points one to one, and the layer above them keeps the
buffers: ``LinearPlan`` and ``ActPlan`` allocate everything a layer needs once,
for a fixed shape, and their calls only enqueue work.
"""
from __future__ import annotations

import ctypes as ct
import dataclasses
import functools
from typing import Optional, Tuple

import torch

from .shiftquant import _I64, _SZ, _check, _ptr, _stream, _ws_ptr, load

TYPE_F32 = 0
TYPE_BF16 = 1
ACT_SILU = 0
ACT_GELU = 1
ACT_KINDS = {"silu": ACT_SILU, "gelu": ACT_GELU}

_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda gpu: torch.cuda.current_stream(gpu).cuda_stream)
_TYPES = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16}


def _type(t: torch.Tensor) -> int:
    """SQ_TYPE_* of a tensor of values on the GPU."""
    if not t.is_cuda:
        raise ValueError("expected a tensor on the GPU")
    try:
        return _TYPES[t.dtype]
    except KeyError:
        raise TypeError(f"expected float32 or bfloat16, got {t.dtype}") from None


def _rows(t: torch.Tensor, name: str) -> int:
    """Row stride of a 2-D tensor with unit column stride."""
    st = t.stride()
    if len(st) != 2 or (st[1] != 1 and t.shape[1] > 1):
        raise ValueError(f"{name}: expected a 2-D tensor with unit column stride")
    return st[0] if t.shape[0] > 1 else max(st[0], t.shape[1])


def _shape(t: torch.Tensor, shape, name: str) -> None:
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")


def _like(t: torch.Tensor, shape, other: torch.Tensor, name: str) -> None:
    """Shape as given, type and place of ``other``."""
    _shape(t, shape, name)
    if t.dtype != other.dtype or t.device != other.device:
        raise ValueError(f"{name}: expected {other.dtype} on {other.device}, got {t.dtype} on {t.device}")


def _sized(codes: Optional[torch.Tensor], scales: Optional[torch.Tensor], sizes, name: str) -> Tuple[Optional[int], Optional[int]]:
    """The pointers of codes and scales, which hold at least ``sizes`` bytes."""
    for t, n in zip((codes, scales), sizes):
        if t is not None and (not t.is_cuda or t.element_size() != 1 or not t.is_contiguous() or t.numel() < n):
            raise ValueError(f"{name}: expected {n} contiguous bytes on the GPU")
    return _ptr(codes), _ptr(scales)


def _mx(codes, scales, rows: int, cols: int, name: str, stack: int = 1):
    nc, ns = _mx_size(rows, cols)
    return _sized(codes, scales, (nc * stack, ns * stack), name)


def _offsets(offsets: Optional[torch.Tensor], experts: int, gpu: Optional[int] = None) -> Optional[int]:
    if offsets is None:
        if experts:
            raise ValueError("offsets: missing")
        return None
    if (offsets.dtype != torch.int32 or offsets.shape != (experts + 1,) or not offsets.is_contiguous()
            or (not offsets.is_cuda if gpu is None else offsets.get_device() != gpu)):
        raise ValueError(f"offsets: expected {experts + 1} contiguous int32 values on the GPU")
    return offsets.data_ptr()


@dataclasses.dataclass
class MxMatrix:
    """A matrix [rows, cols] in microscaled 4-bit codes, or a stack of them
    (codes and scales are then [stack, bytes of a matrix])."""
    codes: torch.Tensor
    scales: torch.Tensor
    rows: int
    cols: int
    stack: int = 0      # 0: one matrix, or as many as codes has rows

    def __post_init__(self):
        nc, ns = sq_mx_size(self.rows, self.cols)
        if self.stack == 0 and self.codes.dim() == 2 and self.codes.shape[0] > 1:
            self.stack = self.codes.shape[0]
        n = max(self.stack, 1)
        for t, size, name in ((self.codes, nc, "codes"), (self.scales, ns, "scales")):
            if t.dtype != torch.uint8 or not t.is_contiguous() or t.numel() < n * size:
                raise ValueError(f"{name}: expected at least {n * size} contiguous uint8 values")
        if self.codes.device != self.scales.device:
            raise ValueError("codes and scales are on different devices")

    @classmethod
    def empty(cls, rows: int, cols: int, stack: int = 0, device="cuda") -> "MxMatrix":
        nc, ns = sq_mx_size(rows, cols)
        n = max(stack, 1)
        return cls(torch.empty((n, nc), dtype=torch.uint8, device=device),
                   torch.empty((n, ns), dtype=torch.uint8, device=device), rows, cols, stack)

    def values(self, dtype=torch.float32, stream=None) -> torch.Tensor:
        """The values that the codes stand for (exact in float32 and bfloat16)."""
        nc, ns = sq_mx_size(self.rows, self.cols)
        out = torch.empty((max(self.stack, 1), self.rows, self.cols), dtype=dtype, device=self.codes.device)
        codes, scales = self.codes.view(-1), self.scales.view(-1)
        for i in range(out.shape[0]):
            sq_mx_dequantize(codes[i * nc:], scales[i * ns:], self.rows, self.cols, out[i], stream)
        return out if self.stack else out[0]


# ---------------------------------------------------------------------------
# one-to-one wrappers of the C entry points
# ---------------------------------------------------------------------------
def sq_mx_size(rows: int, cols: int) -> Tuple[int, int]:
    """(bytes of the codes, bytes of the scales)"""
    a, b = _SZ(0), _SZ(0)
    _check("sq_mx_size", load().sq_mx_size(rows, cols, ct.byref(a), ct.byref(b)))
    return a.value, b.value


_mx_size = functools.lru_cache(maxsize=1024)(sq_mx_size)     # of the arguments alone


def sq_mx_segment_cols(rows: int, experts: int) -> int:
    n = _I64(0)
    _check("sq_mx_segment_cols", load().sq_mx_segment_cols(rows, experts, ct.byref(n)))
    return n.value


def sq_mx_quantize(X, codes, scales, codes_t, scales_t, offsets=None, experts=0, stream=None) -> None:
    """X [rows, cols] or [batch, rows, cols]"""
    if X.dim() == 3:
        batch, (rows, cols) = X.shape[0], X.shape[1:]
        if cols > 1 and X.stride(2) != 1:
            raise ValueError("X: expected unit column stride")
        ld, stride = (X.stride(1) if rows > 1 else max(X.stride(1), cols)), X.stride(0)
    else:
        (rows, cols), batch, ld, stride = X.shape, 1, _rows(X, "X"), 0
    _check("sq_mx_quantize", load().sq_mx_quantize(
        _ptr(X), _type(X), batch, rows, cols, ld, stride, _offsets(offsets, experts), experts,
        *_mx(codes, scales, rows, cols, "codes", batch),
        *_mx(codes_t, scales_t, cols, sq_mx_segment_cols(rows, experts) if experts else rows, "codes_t", batch),
        _stream(stream)))


def sq_mx_dequantize(codes, scales, rows, cols, out, stream=None) -> None:
    _shape(out, (rows, cols), "out")
    _check("sq_mx_dequantize", load().sq_mx_dequantize(
        *_mx(codes, scales, rows, cols, "codes"), rows, cols, _ptr(out), _type(out), _rows(out, "out"), _stream(stream)))


def sq_mx_gemm_workspace_size(M: int, N: int, K: int) -> int:
    nb = _SZ(0)
    _check("sq_mx_gemm_workspace_size", load().sq_mx_gemm_workspace_size(M, N, K, ct.byref(nb)))
    return nb.value


def sq_mx_gemm(A, A_scales, B, B_scales, K, C, workspace=None, stream=None) -> None:
    M, N = C.shape
    ws, nws = _ws_ptr(workspace)
    _check("sq_mx_gemm", load().sq_mx_gemm(
        *_mx(A, A_scales, M, K, "A"), *_mx(B, B_scales, N, K, "B"), M, N, K, _ptr(C), _type(C), _rows(C, "C"), ws, nws,
        _stream(stream)))


def sq_mx_gemm_experts(A, A_scales, K, offsets, experts, B, B_scales, C, stream=None) -> None:
    M, N = C.shape
    _check("sq_mx_gemm_experts", load().sq_mx_gemm_experts(
        *_mx(A, A_scales, M, K, "A"), M, K, _offsets(offsets, experts), experts, *_mx(B, B_scales, N, K, "B", experts), N,
        _ptr(C), _type(C), _rows(C, "C"), _stream(stream)))


def sq_mx_gemm_experts_wgrad_workspace_size(rows: int, experts: int, M: int, N: int) -> int:
    nb = _SZ(0)
    _check("sq_mx_gemm_experts_wgrad_workspace_size",
           load().sq_mx_gemm_experts_wgrad_workspace_size(rows, experts, M, N, ct.byref(nb)))
    return nb.value


def sq_mx_gemm_experts_wgrad(A, A_scales, B, B_scales, rows, offsets, experts, C, workspace=None, stream=None) -> None:
    """C [experts, M, N], contiguous"""
    if C.dim() != 3 or C.shape[0] != experts or not C.is_contiguous():
        raise ValueError("C: expected a contiguous [experts, M, N] tensor")
    ws, nws = _ws_ptr(workspace)
    inner = sq_mx_segment_cols(rows, experts)
    _check("sq_mx_gemm_experts_wgrad", load().sq_mx_gemm_experts_wgrad(
        *_mx(A, A_scales, C.shape[1], inner, "A"), *_mx(B, B_scales, C.shape[2], inner, "B"), rows,
        _offsets(offsets, experts), experts, C.shape[1], C.shape[2],
        _ptr(C), _type(C), max(C.shape[2], 1), ws, nws, _stream(stream)))


def sq_mx_linear_workspace_size(M: int, K: int, N: int, experts: int = 0) -> int:
    nb = _SZ(0)
    _check("sq_mx_linear_workspace_size", load().sq_mx_linear_workspace_size(M, K, N, experts, ct.byref(nb)))
    return nb.value


def sq_mx_linear(X, W, W_scales, Y, workspace=None, offsets=None, experts=0, stream=None) -> None:
    M, K = X.shape
    N = Y.shape[1]
    _shape(Y, (M, N), "Y")
    ws, nws = _ws_ptr(workspace)
    _check("sq_mx_linear", load().sq_mx_linear(
        _ptr(X), _type(X), M, K, _rows(X, "X"), _offsets(offsets, experts), experts,
        *_mx(W, W_scales, N, K, "W", max(experts, 1)), N, _ptr(Y), _type(Y), _rows(Y, "Y"), ws, nws, _stream(stream)))


class Layer(ct.Structure):
    """sq_mx_layer"""
    _fields_ = ([(n, _I64) for n in ("rows", "c_in", "c_out", "experts")] + [("type", ct.c_int32), ("reserved", ct.c_int32)]
                + [(m + s, ct.c_void_p) for m in ("w", "w_t", "x", "x_t", "dy", "dy_t") for s in ("", "_scales")]
                + [("workspace", ct.c_void_p), ("workspace_bytes", _SZ), ("offsets", ct.c_void_p)])


def sq_mx_layer_workspace_size(layer: Layer) -> int:
    nb = _SZ(0)
    _check("sq_mx_layer_workspace_size", load().sq_mx_layer_workspace_size(ct.addressof(layer), ct.byref(nb)))
    return nb.value


def _of_layer(layer: Layer, t: torch.Tensor, shape, name: str, type_=None) -> int:
    """The pointer of a tensor of the layer's type (or ``type_``) and that shape."""
    _shape(t, shape, name)
    if _type(t) != (layer.type if type_ is None else type_):
        raise TypeError(f"{name}: {t.dtype} is not its type in the layer")
    return t.data_ptr()


def _layer_stack(layer: Layer) -> Tuple[int, ...]:
    one = (layer.c_out, layer.c_in)
    return (layer.experts, *one) if layer.experts else one


def sq_mx_layer_weight(layer: Layer, W, stream=None) -> None:
    """W [c_out, c_in], or [experts, c_out, c_in]"""
    w = _of_layer(layer, W, _layer_stack(layer), "W")
    st = W.stride()
    if st[-1] != 1 and W.shape[-1] > 1:
        raise ValueError("W: expected unit column stride")
    ld = st[-2] if W.shape[-2] > 1 else max(st[-2], W.shape[-1])
    _check("sq_mx_layer_weight", load().sq_mx_layer_weight(ct.addressof(layer), w, ld, st[0], _stream(stream)))


def sq_mx_layer_forward(layer: Layer, X, offsets, Y, stream=None) -> None:
    _check("sq_mx_layer_forward", load().sq_mx_layer_forward(
        ct.addressof(layer), _of_layer(layer, X, (layer.rows, layer.c_in), "X"), _rows(X, "X"),
        _offsets(offsets, layer.experts), _of_layer(layer, Y, (layer.rows, layer.c_out), "Y"), _rows(Y, "Y"),
        _stream(stream)))


def sq_mx_layer_backward(layer: Layer, dY, offsets, dX, dW, stream=None) -> None:
    """dW [c_out, c_in] or [experts, c_out, c_in], contiguous; offsets None: those that the forward kept"""
    if not dW.is_contiguous():
        raise ValueError("dW: expected a contiguous tensor")
    _check("sq_mx_layer_backward", load().sq_mx_layer_backward(
        ct.addressof(layer), _of_layer(layer, dY, (layer.rows, layer.c_out), "dY"), _rows(dY, "dY"),
        None if offsets is None else _offsets(offsets, layer.experts), _of_layer(layer, dX, (layer.rows, layer.c_in), "dX"), _rows(dX, "dX"),
        _of_layer(layer, dW, _layer_stack(layer), "dW", TYPE_F32), max(layer.c_in, 1), _stream(stream)))


def sq_act_size(M: int, F: int, gated: bool) -> Tuple[int, int]:
    a, b = _SZ(0), _SZ(0)
    _check("sq_act_size", load().sq_act_size(M, F, int(gated), ct.byref(a), ct.byref(b)))
    return a.value, b.value


def sq_act_forward(X, kind, gated, H, codes, scales, stream=None) -> None:
    M, F = H.shape
    _like(X, (M, 2 * F if gated else F), H, "X")
    _check("sq_act_forward", load().sq_act_forward(
        _ptr(X), _type(X), kind, int(gated), M, F, _rows(X, "X"), _ptr(H), _rows(H, "H"),
        *_sized(codes, scales, sq_act_size(M, F, gated), "codes"), _stream(stream)))


def sq_act_backward(dH, kind, gated, codes, scales, dX, stream=None) -> None:
    M, F = dH.shape
    _like(dX, (M, 2 * F if gated else F), dH, "dX")
    _check("sq_act_backward", load().sq_act_backward(
        _ptr(dH), _type(dH), kind, int(gated), M, F, _rows(dH, "dH"),
        *_sized(codes, scales, sq_act_size(M, F, gated), "codes"), _ptr(dX), _rows(dX, "dX"), _stream(stream)))


# ---------------------------------------------------------------------------
# layers
# ---------------------------------------------------------------------------
def _workspace(nbytes: int, device) -> Optional[torch.Tensor]:
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def quantize(X: torch.Tensor, rows: bool = True, cols: bool = False, offsets: Optional[torch.Tensor] = None,
             stream=None) -> Tuple[Optional[MxMatrix], Optional[MxMatrix]]:
    """Codes of X [rows, cols] (or a stack of such) with blocks along its columns
    (``rows``: the operand X) and along its rows (``cols``: the operand X^T, by
    expert with ``offsets``), in one read."""
    stack = X.shape[0] if X.dim() == 3 else 0
    M, C = X.shape[-2:]
    experts = 0 if offsets is None else offsets.shape[0] - 1
    a = MxMatrix.empty(M, C, stack, X.device) if rows else None
    t = MxMatrix.empty(C, sq_mx_segment_cols(M, experts) if experts else M, stack, X.device) if cols else None
    sq_mx_quantize(X, a and a.codes, a and a.scales, t and t.codes, t and t.scales, offsets, experts, stream)
    return a, t


# The plans' calls run once per launch or two, so their own time bounds small
# layers (a token through 4096 x 4096: 6.4 us a call through the wrappers above,
# 4.5 us on the GPU): an input is looked at once, and what does not change from
# call to call is kept as integers.
def _checked(t: torch.Tensor, shape, dtype, gpu: int, name: str) -> int:
    """The row stride of a plan's input, after a look at its shape, type, place and strides."""
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.get_device() != gpu:
        raise ValueError(f"{name}: expected a tensor on the plan's GPU, got one on {t.device}")
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: expected unit column stride")
    return st[-2] if shape[-2] > 1 else max(st[-2], shape[-1])


def _gpu_of(t: torch.Tensor) -> int:
    """Index of the GPU of a plan's buffer; no tensor has that of a plan elsewhere."""
    return t.get_device() if t.is_cuda else -2


def _on(gpu: int, stream) -> int:
    """The stream of a plan's launches, which go to the current GPU."""
    if _current_device() != gpu:
        raise ValueError("the plan's GPU is not the current one")
    return _raw_stream(gpu) if stream is None else stream.cuda_stream


class LinearPlan:
    """A linear layer Y = X W^T on M rows with microscaled 4-bit operands, all of
    its buffers allocated once.  ``experts`` > 0: that many weight matrices; the
    rows are sorted by expert and ``offsets`` [experts + 1] says where each
    expert's begin (any split of the M rows).

    Serving: ``forward(x, w)`` with W's codes.  Training (``train=True``):
    ``quantize_weight(W)``, ``forward(x)``, then ``backward(dy)``, which gives dX in
    the layer's type and dW in float32; the forward keeps X's codes and a copy of
    the offsets for it (``self.offsets``).  Results are the plan's buffers, overwritten by its next
    call of the same kind."""

    def __init__(self, M: int, C_in: int, C_out: int, dtype=torch.bfloat16, experts: int = 0, train: bool = False,
                 device="cuda"):
        if dtype not in _TYPES:
            raise TypeError(f"dtype: expected float32 or bfloat16, got {dtype}")
        dev = torch.device(device)
        self.M, self.C_in, self.C_out, self.dtype, self.experts, self.train = M, C_in, C_out, dtype, experts, train
        self._x_shape, self._y_shape = torch.Size((M, C_in)), torch.Size((M, C_out))
        self._w_shape = torch.Size((experts, C_out, C_in) if experts else (C_out, C_in))
        self.Y = torch.empty(self._y_shape, dtype=dtype, device=dev)
        self.offsets, self._type = None, _TYPES[dtype]
        self._y_ptr, self._y_ld, self._lib, self._gpu = self.Y.data_ptr(), max(C_out, 1), load(), _gpu_of(self.Y)
        self._has_weight = self._has_input = False
        if not train:
            self.ws = _workspace(sq_mx_linear_workspace_size(M, C_in, C_out, experts), dev)
            self._ws = _ws_ptr(self.ws)
            self._held = [self.Y, self.ws]      # the pointers kept stay valid as long as the plan
            return
        inner = sq_mx_segment_cols(M, experts) if experts else M
        self.w = MxMatrix.empty(C_out, C_in, experts, dev)
        self.w_t = MxMatrix.empty(C_in, C_out, experts, dev)
        self.x, self.x_t = MxMatrix.empty(M, C_in, 0, dev), MxMatrix.empty(C_in, inner, 0, dev)
        self.dy, self.dy_t = MxMatrix.empty(M, C_out, 0, dev), MxMatrix.empty(C_out, inner, 0, dev)
        self.dX = torch.empty(self._x_shape, dtype=dtype, device=dev)
        self.dW = torch.empty(self._w_shape, dtype=torch.float32, device=dev)
        self.layer = Layer(M, C_in, C_out, experts, _TYPES[dtype], 0)
        self._held = []     # the layer's pointers stay valid as long as the plan
        for name in ("w", "w_t", "x", "x_t", "dy", "dy_t"):
            m = getattr(self, name)
            self._held += [m.codes, m.scales]
            setattr(self.layer, name, m.codes.data_ptr())
            setattr(self.layer, name + "_scales", m.scales.data_ptr())
        self._layer_ptr, self._dw_ld = ct.addressof(self.layer), max(C_in, 1)
        self._dx_ptr, self._dw_ptr = self.dX.data_ptr(), self.dW.data_ptr()
        if experts:
            self.offsets = torch.zeros(experts + 1, dtype=torch.int32, device=dev)
            self.layer.offsets = self.offsets.data_ptr()
        self._held += [self.Y, self.dX, self.dW, self.offsets]
        self.ws = _workspace(sq_mx_layer_workspace_size(self.layer), dev)
        if self.ws is not None:
            self.layer.workspace, self.layer.workspace_bytes = self.ws.data_ptr(), self.ws.nbytes

    def quantize_weight(self, W: torch.Tensor, stream=None) -> None:
        """W [C_out, C_in], or [experts, C_out, C_in]"""
        if not self.train:
            raise ValueError("quantize_weight needs a plan with train=True")
        ld = _checked(W, self._w_shape, self.dtype, self._gpu, "W")
        st = self._lib.sq_mx_layer_weight(
            self._layer_ptr, W.data_ptr(), ld, W.stride(0), _on(self._gpu, stream))
        if st:
            _check("sq_mx_layer_weight", st)
        self._has_weight = True

    def forward(self, x: torch.Tensor, w: Optional[MxMatrix] = None, offsets: Optional[torch.Tensor] = None, stream=None):
        ld = _checked(x, self._x_shape, self.dtype, self._gpu, "x")
        off = _offsets(offsets, self.experts, self._gpu)
        if self.train:
            if w is not None:
                raise ValueError("w: a training plan has its own codes (quantize_weight)")
            if not self._has_weight:
                raise ValueError("forward needs a quantize_weight before it")
            st = self._lib.sq_mx_layer_forward(
                self._layer_ptr, x.data_ptr(), ld, off, self._y_ptr, self._y_ld, _on(self._gpu, stream))
            if st:
                _check("sq_mx_layer_forward", st)
            self._has_input = True
            return self.Y
        if w is None or w.rows != self.C_out or w.cols != self.C_in or (w.stack or 1) != (self.experts or 1):
            raise ValueError(f"w: expected codes of {self.experts or 'one'} [{self.C_out}, {self.C_in}]")
        codes = w.codes
        if codes.get_device() != self._gpu:
            raise ValueError("w: expected codes on the plan's GPU")
        t = self._type
        st = self._lib.sq_mx_linear(
            x.data_ptr(), t, self.M, self.C_in, ld, off, self.experts, codes.data_ptr(), w.scales.data_ptr(), self.C_out,
            self._y_ptr, t, self._y_ld, *self._ws, _on(self._gpu, stream))
        if st:
            _check("sq_mx_linear", st)
        return self.Y

    def backward(self, dy: torch.Tensor, stream=None):
        """(dX, dW) of the last forward"""
        if not self.train:
            raise ValueError("backward needs a plan with train=True")
        ld = _checked(dy, self._y_shape, self.dtype, self._gpu, "dy")
        if not self._has_input:
            raise ValueError("backward needs a forward before it")
        st = self._lib.sq_mx_layer_backward(
            self._layer_ptr, dy.data_ptr(), ld, None, self._dx_ptr, self._dw_ld, self._dw_ptr, self._dw_ld,
            _on(self._gpu, stream))
        if st:
            _check("sq_mx_layer_backward", st)
        return self.dX, self.dW


class ActPlan:
    """An activation on M rows of F outputs, ``act`` "silu" or "gelu" (tanh form),
    ``gated``: h = act(g) u of an input [M, 2 F] with the gate first.  The forward
    keeps the input in 8 bits, the backward reads only that and dh."""

    def __init__(self, M: int, F: int, act: str = "silu", gated: bool = True, dtype=torch.bfloat16, device="cuda"):
        if act not in ACT_KINDS:
            raise ValueError(f"act: expected one of {sorted(ACT_KINDS)}, got {act!r}")
        if dtype not in _TYPES:
            raise TypeError(f"dtype: expected float32 or bfloat16, got {dtype}")
        dev = torch.device(device)
        self.M, self.F, self.kind, self.gated, self.dtype = M, F, ACT_KINDS[act], gated, dtype
        self.width = 2 * F if gated else F
        nc, ns = sq_act_size(M, F, gated)
        self.codes = torch.empty(nc, dtype=torch.int8, device=dev)
        self.scales = torch.empty(ns, dtype=torch.uint8, device=dev)
        self._h_shape, self._x_shape = torch.Size((M, F)), torch.Size((M, self.width))
        self.H = torch.empty(self._h_shape, dtype=dtype, device=dev)
        self.dX = torch.empty(self._x_shape, dtype=dtype, device=dev)
        self._lib, self._type, self._gated, self._gpu = load(), _TYPES[dtype], int(gated), _gpu_of(self.H)
        self._has_input = False
        self._held = (self.codes, self.scales, self.H, self.dX)     # what _ptrs point at
        self._ptrs = tuple(t.data_ptr() for t in self._held)
        self._h_ld, self._x_ld = max(F, 1), max(self.width, 1)

    def forward(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        ld = _checked(x, self._x_shape, self.dtype, self._gpu, "x")
        codes, scales, h, _ = self._ptrs
        st = self._lib.sq_act_forward(
            x.data_ptr(), self._type, self.kind, self._gated, self.M, self.F, ld, h, self._h_ld, codes, scales,
            _on(self._gpu, stream))
        if st:
            _check("sq_act_forward", st)
        self._has_input = True
        return self.H

    def backward(self, dh: torch.Tensor, stream=None) -> torch.Tensor:
        ld = _checked(dh, self._h_shape, self.dtype, self._gpu, "dh")
        if not self._has_input:
            raise ValueError("backward needs a forward before it")
        codes, scales, _, dx = self._ptrs
        st = self._lib.sq_act_backward(
            dh.data_ptr(), self._type, self.kind, self._gated, self.M, self.F, ld, codes, scales, dx, self._x_ld,
            _on(self._gpu, stream))
        if st:
            _check("sq_act_backward", st)
        return self.dX
