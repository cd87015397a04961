"""Layer norm with the residual sum before it, forward and backward
(include/shiftquant.h has the formulas).

As in the ``mx`` module, ``sq_*`` marshal torch tensors to the C entry points one
to one, and ``NormPlan`` keeps the buffers of a fixed shape: its calls only
enqueue work.
"""
from __future__ import annotations

import ctypes as ct
from typing import Optional, Tuple

import torch

from .mx import _TYPES, _checked, _gpu_of, _like, _on, _rows, _shape, _type, _workspace
from .shiftquant import _I64, _P, _SZ, _check, _ptr, _stream, _ws_ptr, load


def _fixed(*values) -> tuple:
    """Arguments that a plan passes in each of its calls, (C type, value), converted once (one
    token's router call takes the host 5.0 us instead of 5.3, an 8-bit layer's 4.75 instead of 4.9)."""
    return tuple(t(v) for t, v in values)


def _vector(t: torch.Tensor, n: int, name: str, like: Optional[torch.Tensor] = None) -> int:
    """The pointer of ``n`` contiguous values on the GPU, of the type of ``like``."""
    if t.shape != (n,) or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name}: expected {n} contiguous values on the GPU")
    if like is not None and t.dtype != like.dtype:
        raise TypeError(f"{name}: expected {like.dtype}, got {t.dtype}")
    return t.data_ptr()


def _floats(t: torch.Tensor, shape, name: str) -> int:
    """The pointer of a contiguous float32 tensor of that shape on the GPU."""
    _shape(t, shape, name)
    if t.dtype != torch.float32 or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name}: expected contiguous float32 values on the GPU")
    return t.data_ptr()


# ---------------------------------------------------------------------------
# one-to-one wrappers of the C entry points
# ---------------------------------------------------------------------------
def sq_norm_forward(X, residual, gamma, beta, eps, H, Y, stats=None, stream=None) -> None:
    M, C = X.shape
    _like(Y, (M, C), X, "Y")
    for t, name in ((residual, "residual"), (H, "H")):
        if t is not None:
            _like(t, (M, C), X, name)
    _check("sq_norm_forward", load().sq_norm_forward(
        _ptr(X), _ptr(residual), _type(X), M, C, _rows(X, "X"), 0 if residual is None else _rows(residual, "residual"),
        _vector(gamma, C, "gamma"), _vector(beta, C, "beta", gamma), _type(gamma), eps, _ptr(H),
        0 if H is None else _rows(H, "H"), _ptr(Y), _rows(Y, "Y"), None if stats is None else _floats(stats, (M, 4), "stats"),
        _stream(stream)))


def sq_norm_backward_workspace_size(M: int, C: int) -> int:
    nb = _SZ(0)
    _check("sq_norm_backward_workspace_size", load().sq_norm_backward_workspace_size(M, C, ct.byref(nb)))
    return nb.value


def sq_norm_backward(dY, H, dH, gamma, stats, dX, dgamma, dbeta, workspace, stream=None) -> None:
    M, C = dY.shape
    for t, name in ((H, "H"), (dX, "dX"), (dH, "dH")):
        if t is not None:
            _like(t, (M, C), dY, name)
    ws, nws = _ws_ptr(workspace)
    _check("sq_norm_backward", load().sq_norm_backward(
        _ptr(dY), _ptr(H), _ptr(dH), _type(dY), M, C, _rows(dY, "dY"), _rows(H, "H"), 0 if dH is None else _rows(dH, "dH"),
        _vector(gamma, C, "gamma"), _type(gamma), _floats(stats, (M, 4), "stats"), _ptr(dX), _rows(dX, "dX"),
        _floats(dgamma, (C,), "dgamma"), _floats(dbeta, (C,), "dbeta"), ws, nws, _stream(stream)))


# ---------------------------------------------------------------------------
class NormPlan:
    """Layer norm of M rows of C, ``residual``: of h = x + residual, which the plan
    keeps in ``H``.  ``forward(x, gamma, beta[, residual])`` gives y; with ``train``
    ``backward(dy, h, gamma[, dh])`` gives (dx, dgamma, dbeta), h the last forward's
    ``H`` (its x without a residual), dh the gradient that reaches h past the norm; dx is the
    residual's gradient too.  gamma and beta [C] of ``param_dtype``, their gradients float32.
    Results are the plan's buffers, overwritten by its next call of the same kind."""

    def __init__(self, M: int, C: int, eps: float = 1e-5, dtype=torch.bfloat16, param_dtype=torch.float32, residual: bool = False,
                 train: bool = False, device="cuda"):
        for name, t in (("dtype", dtype), ("param_dtype", param_dtype)):
            if t not in _TYPES:
                raise TypeError(f"{name}: expected float32 or bfloat16, got {t}")
        dev = torch.device(device)
        nbytes = sq_norm_backward_workspace_size(M, C)      # refuses sizes that the calls refuse
        self.M, self.C, self.eps, self.dtype, self.param_dtype, self.train = M, C, eps, dtype, param_dtype, train
        self._shape, self._c_shape = torch.Size((M, C)), torch.Size((C,))
        self.Y = torch.empty(self._shape, dtype=dtype, device=dev)
        self.H = torch.empty(self._shape, dtype=dtype, device=dev) if residual else None
        self._lib, self._gpu = load(), _gpu_of(self.Y)
        self._has_input = False
        self.stats = self.dX = self.dgamma = self.dbeta = self.ws = None
        if train:
            self.stats = torch.empty((M, 4), dtype=torch.float32, device=dev)
            self.dX = torch.empty(self._shape, dtype=dtype, device=dev)
            self.dgamma, self.dbeta = torch.empty((2, C), dtype=torch.float32, device=dev).unbind(0)
            self.ws = _workspace(nbytes, dev)
        i32, ld = ct.c_int32, (_I64, max(C, 1))
        self._held = (self.Y, self.H, self.stats, self.dX, self.dgamma, self.dbeta, self.ws)    # what the calls point at
        y, h, stats, dx, dgamma, dbeta = ((_P, _ptr(t)) for t in self._held[:-1])
        ws, nws = _ws_ptr(self.ws)
        self._size = _fixed((i32, _TYPES[dtype]), (_I64, M), (_I64, C))
        self._to = _fixed((i32, _TYPES[param_dtype]), (ct.c_float, eps), h, ld, y, ld, stats)
        self._to_back = _fixed((i32, _TYPES[param_dtype]), stats, dx, ld, dgamma, dbeta, (_P, ws), (_SZ, nws))

    def _param(self, t: torch.Tensor, name: str) -> int:
        if t.shape != self._c_shape or not t.is_contiguous() or t.get_device() != self._gpu:
            raise ValueError(f"{name}: expected {self.C} contiguous values on the plan's GPU")
        if t.dtype is not self.param_dtype:
            raise TypeError(f"{name}: expected {self.param_dtype}, got {t.dtype}")
        return t.data_ptr()

    def forward(self, x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, residual: Optional[torch.Tensor] = None,
                stream=None) -> torch.Tensor:
        if (residual is None) != (self.H is None):
            raise ValueError("residual: expected one for a plan with residual=True, and none without")
        ld = _checked(x, self._shape, self.dtype, self._gpu, "x")
        ld_r = 0 if residual is None else _checked(residual, self._shape, self.dtype, self._gpu, "residual")
        st = self._lib.sq_norm_forward(
            x.data_ptr(), _ptr(residual), *self._size, ld, ld_r, self._param(gamma, "gamma"), self._param(beta, "beta"), *self._to,
            _on(self._gpu, stream))
        if st:
            _check("sq_norm_forward", st)
        self._has_input = True
        return self.Y

    def backward(self, dy: torch.Tensor, h: torch.Tensor, gamma: torch.Tensor, dh: Optional[torch.Tensor] = None,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
        """(dX, dgamma, dbeta) of the last forward"""
        if not self.train:
            raise ValueError("backward needs a plan with train=True")
        if not self._has_input:
            raise ValueError("backward needs a forward before it")
        ld_dy = _checked(dy, self._shape, self.dtype, self._gpu, "dy")
        ld_h = _checked(h, self._shape, self.dtype, self._gpu, "h")
        ld_dh = 0 if dh is None else _checked(dh, self._shape, self.dtype, self._gpu, "dh")
        st = self._lib.sq_norm_backward(
            dy.data_ptr(), h.data_ptr(), _ptr(dh), *self._size, ld_dy, ld_h, ld_dh, self._param(gamma, "gamma"), *self._to_back,
            _on(self._gpu, stream))
        if st:
            _check("sq_norm_backward", st)
        return self.dX, self.dgamma, self.dbeta
