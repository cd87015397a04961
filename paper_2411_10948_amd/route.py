"""Routing of tokens to experts, and the exchange of rows between the two
(include/shiftquant.h has the rules, formulas and layouts).

As in the ``mx`` module, ``sq_*`` marshal torch tensors to the C entry points one
to one, and the plans keep the buffers of a fixed shape: their calls only enqueue
work.
"""
from __future__ import annotations

import ctypes as ct
from typing import Optional, Tuple

import torch

from .mx import _TYPES, _checked, _gpu_of, _like, _on, _rows, _shape, _type, _workspace
from .norm import _fixed, _floats
from .shiftquant import _I64, _P, _SZ, _check, _ptr, _stream, _ws_ptr, load

SCORE_SOFTMAX = 0
SCORE_SIGMOID = 1
SCORES = {"softmax": SCORE_SOFTMAX, "sigmoid": SCORE_SIGMOID}


def _ints(t: torch.Tensor, shape, name: str) -> int:
    """The pointer of a contiguous int32 tensor of that shape on the GPU."""
    _shape(t, shape, name)
    if t.dtype != torch.int32 or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name}: expected contiguous int32 values on the GPU")
    return t.data_ptr()


# ---------------------------------------------------------------------------
# one-to-one wrappers of the C entry points
# ---------------------------------------------------------------------------
def sq_route_workspace_size(T: int, E: int) -> int:
    nb = _SZ(0)
    _check("sq_route_workspace_size", load().sq_route_workspace_size(T, E, ct.byref(nb)))
    return nb.value


def sq_route_forward(logits, bias, score, groups, top_groups, renormalize, scale, share, chosen, place, offsets, workspace=None,
                     stream=None) -> None:
    T, E = logits.shape
    k = share.shape[1]
    ws, nws = _ws_ptr(workspace)
    _check("sq_route_forward", load().sq_route_forward(
        _ptr(logits), _type(logits), T, E, _rows(logits, "logits"), None if bias is None else _floats(bias, (E,), "bias"), score, k,
        groups, top_groups, int(renormalize), scale, _floats(share, (T, k), "share"), _ints(chosen, (T, k), "chosen"),
        _ints(place, (T, k), "place"), _ints(offsets, (E + 1,), "offsets"), ws, nws, _stream(stream)))


def sq_route_backward(dshare, logits, score, renormalize, scale, share, chosen, dlogits, stream=None) -> None:
    T, E = logits.shape
    k = share.shape[1]
    _like(dlogits, (T, E), logits, "dlogits")
    _check("sq_route_backward", load().sq_route_backward(
        _floats(dshare, (T, k), "dshare"), _ptr(logits), _type(logits), T, E, _rows(logits, "logits"), score, k, int(renormalize),
        scale, _floats(share, (T, k), "share"), _ints(chosen, (T, k), "chosen"), _ptr(dlogits), _rows(dlogits, "dlogits"),
        _stream(stream)))


def sq_exchange_dispatch(X, place, R, stream=None) -> None:
    (T, D), k = X.shape, place.shape[1]
    _like(R, (R.shape[0], D), X, "R")
    _check("sq_exchange_dispatch", load().sq_exchange_dispatch(
        _ptr(X), _type(X), T, D, _rows(X, "X"), _ints(place, (T, k), "place"), k, _ptr(R), R.shape[0], _rows(R, "R"),
        _stream(stream)))


def sq_exchange_combine(R, place, share, add, out, stream=None) -> None:
    (T, D), k = out.shape, place.shape[1]
    _like(R, (R.shape[0], D), out, "R")
    if add is not None:
        _like(add, (T, D), out, "add")
    _check("sq_exchange_combine", load().sq_exchange_combine(
        _ptr(R), _type(R), R.shape[0], D, _rows(R, "R"), _ints(place, (T, k), "place"),
        None if share is None else _floats(share, (T, k), "share"), T, k, _ptr(add), 0 if add is None else _rows(add, "add"),
        _ptr(out), _rows(out, "out"), _stream(stream)))


def sq_exchange_combine_backward(dout, R, place, share, dR, dshare, stream=None) -> None:
    (T, D), k = dout.shape, place.shape[1]
    _like(R, (R.shape[0], D), dout, "R")
    _like(dR, R.shape, dout, "dR")
    _check("sq_exchange_combine_backward", load().sq_exchange_combine_backward(
        _ptr(dout), _ptr(R), _type(R), R.shape[0], D, _rows(dout, "dout"), _rows(R, "R"), _ints(place, (T, k), "place"),
        _floats(share, (T, k), "share"), T, k, _ptr(dR), _rows(dR, "dR"), _floats(dshare, (T, k), "dshare"), _stream(stream)))


# ---------------------------------------------------------------------------
class RouterPlan:
    """The ``k`` best of E experts for each of T tokens: ``score`` "softmax" or
    "sigmoid", ``groups`` of experts of which the best ``top_groups`` are kept,
    ``renormalize``: shares divided by the sum of the chosen ones, times ``scale``.

    ``forward(logits[, bias])`` gives (share, chosen) [T, k] and fills ``place`` [T, k]
    and ``offsets`` [E + 1], the split of the rows that products by expert take.
    ``backward(dshare, logits)`` gives the gradient of the last forward's logits.
    Results are the plan's buffers, overwritten by its next call of the same kind."""

    def __init__(self, T: int, E: int, k: int, score: str = "softmax", groups: int = 1, top_groups: Optional[int] = None,
                 renormalize: bool = False, scale: float = 1.0, dtype=torch.bfloat16, device="cuda"):
        if score not in SCORES:
            raise ValueError(f"score: expected one of {sorted(SCORES)}, got {score!r}")
        if dtype not in _TYPES:
            raise TypeError(f"dtype: expected float32 or bfloat16, got {dtype}")
        top_groups = groups if top_groups is None else top_groups
        if not 1 <= top_groups <= groups or E % groups or not 1 <= k <= E // groups * top_groups:
            raise ValueError(f"no choice of {k} of {E} experts from {top_groups} of {groups} groups")
        dev = torch.device(device)
        self.ws = _workspace(sq_route_workspace_size(T, E), dev)
        self.T, self.E, self.k, self.dtype = T, E, k, dtype
        self._l_shape, self._k_shape = torch.Size((T, E)), torch.Size((T, k))
        self.share = torch.empty((T, k), dtype=torch.float32, device=dev)
        self.chosen = torch.empty((T, k), dtype=torch.int32, device=dev)
        self.place = torch.empty((T, k), dtype=torch.int32, device=dev)
        self.offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
        self.dlogits = torch.empty((T, E), dtype=dtype, device=dev)
        self._lib, self._gpu = load(), _gpu_of(self.share)
        self._has_input = False
        self._held = (self.share, self.chosen, self.place, self.offsets, self.dlogits, self.ws)     # what the calls point at
        share, chosen, place, offsets, dlogits = ((_P, t.data_ptr()) for t in self._held[:-1])
        i32, (ws, nws) = ct.c_int32, _ws_ptr(self.ws)
        score, k, renorm, scale = (i32, SCORES[score]), (i32, k), (i32, int(renormalize)), (ct.c_float, scale)
        self._size = _fixed((i32, _TYPES[dtype]), (_I64, T), (_I64, E))
        self._to = _fixed(score, k, (i32, groups), (i32, top_groups), renorm, scale, share, chosen, place, offsets, (_P, ws), (_SZ, nws))
        self._to_back = _fixed(score, k, renorm, scale, share, chosen, dlogits, (_I64, E))

    def forward(self, logits: torch.Tensor, bias: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        ld = _checked(logits, self._l_shape, self.dtype, self._gpu, "logits")
        if bias is not None and (bias.dtype is not torch.float32 or bias.shape != (self.E,) or not bias.is_contiguous()
                                 or bias.get_device() != self._gpu):
            raise ValueError(f"bias: expected {self.E} contiguous float32 values on the plan's GPU")
        st = self._lib.sq_route_forward(
            logits.data_ptr(), *self._size, ld, _ptr(bias), *self._to, _on(self._gpu, stream))
        if st:
            _check("sq_route_forward", st)
        self._has_input = True
        return self.share, self.chosen

    def backward(self, dshare: torch.Tensor, logits: torch.Tensor, stream=None) -> torch.Tensor:
        if not self._has_input:
            raise ValueError("backward needs a forward before it")
        _checked(dshare, self._k_shape, torch.float32, self._gpu, "dshare")
        if not dshare.is_contiguous():
            raise ValueError("dshare: expected a contiguous tensor")
        ld = _checked(logits, self._l_shape, self.dtype, self._gpu, "logits")
        st = self._lib.sq_route_backward(
            dshare.data_ptr(), logits.data_ptr(), *self._size, ld, *self._to_back, _on(self._gpu, stream))
        if st:
            _check("sq_route_backward", st)
        return self.dlogits


class ExchangePlan:
    """Rows of T tokens to ``T k`` rows sorted by expert and back, by a router's ``place``
    (-1: no row) and ``share`` [T, k].

    ``dispatch(x, place)`` gives the sorted rows, ``combine(y, place, share[, add])`` the tokens'
    sums; with ``train`` ``combine_backward(dout, y, place, share)`` gives (dy, dshare) and
    ``dispatch_backward(drows, place[, add])`` dx.  Results are the plan's buffers, overwritten by
    its next call of the same kind; rows that no place names keep what they held (zeros at first)."""

    def __init__(self, T: int, k: int, D: int, dtype=torch.bfloat16, train: bool = False, device="cuda"):
        if dtype not in _TYPES:
            raise TypeError(f"dtype: expected float32 or bfloat16, got {dtype}")
        if T < 0 or not 0 <= D < 1 << 20 or not 1 <= k <= 64 or T * k >= 1 << 31:
            raise ValueError(f"no exchange of {T} tokens of {D} with {k} rows each")
        dev = torch.device(device)
        self.T, self.k, self.D, self.rows, self.dtype, self.train = T, k, D, T * k, dtype, train
        self._x_shape, self._r_shape, self._k_shape = torch.Size((T, D)), torch.Size((T * k, D)), torch.Size((T, k))
        self.R = torch.zeros(self._r_shape, dtype=dtype, device=dev)
        self.out = torch.empty(self._x_shape, dtype=dtype, device=dev)
        self._lib, self._gpu = load(), _gpu_of(self.R)
        self.dR = self.dX = self.dshare = None
        if train:
            self.dR, self.dX = torch.zeros_like(self.R), torch.empty_like(self.out)
            self.dshare = torch.empty((T, k), dtype=torch.float32, device=dev)
        self._held = (self.R, self.out, self.dR, self.dX, self.dshare)      # what the calls point at
        r, out, dr, dx, dshare = ((_P, _ptr(t)) for t in self._held)
        kind, slots = (ct.c_int32, _TYPES[dtype]), (ct.c_int32, k)
        t, n, d, ld = (_I64, T), (_I64, T * k), (_I64, D), (_I64, max(D, 1))
        self._x_size, self._r_size, self._slots_of = _fixed(kind, t, d), _fixed(kind, n, d), _fixed(t, slots)
        self._to_rows, self._to_out, self._to_dx = _fixed(slots, r, n, ld), _fixed(out, ld), _fixed(dx, ld)
        self._to_back = _fixed(dr, ld, dshare)

    def _slots(self, t: torch.Tensor, dtype, name: str) -> int:
        if t.dtype is not dtype or t.shape != self._k_shape or not t.is_contiguous() or t.get_device() != self._gpu:
            raise ValueError(f"{name}: expected contiguous {dtype} values of shape {tuple(self._k_shape)} on the plan's GPU")
        return t.data_ptr()

    def dispatch(self, x: torch.Tensor, place: torch.Tensor, stream=None) -> torch.Tensor:
        ld = _checked(x, self._x_shape, self.dtype, self._gpu, "x")
        st = self._lib.sq_exchange_dispatch(
            x.data_ptr(), *self._x_size, ld, self._slots(place, torch.int32, "place"), *self._to_rows, _on(self._gpu, stream))
        if st:
            _check("sq_exchange_dispatch", st)
        return self.R

    def _combine(self, y, place, share, add, to: tuple, stream) -> None:
        ld = _checked(y, self._r_shape, self.dtype, self._gpu, "rows")
        ld_a = 0 if add is None else _checked(add, self._x_shape, self.dtype, self._gpu, "add")
        st = self._lib.sq_exchange_combine(
            y.data_ptr(), *self._r_size, ld, self._slots(place, torch.int32, "place"),
            None if share is None else self._slots(share, torch.float32, "share"), *self._slots_of, _ptr(add), ld_a, *to,
            _on(self._gpu, stream))
        if st:
            _check("sq_exchange_combine", st)

    def combine(self, y: torch.Tensor, place: torch.Tensor, share: torch.Tensor, add: Optional[torch.Tensor] = None,
                stream=None) -> torch.Tensor:
        if share is None:
            raise ValueError("share: missing")
        self._combine(y, place, share, add, self._to_out, stream)
        return self.out

    def combine_backward(self, dout: torch.Tensor, y: torch.Tensor, place: torch.Tensor, share: torch.Tensor,
                         stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(dy, dshare)"""
        if not self.train:
            raise ValueError("combine_backward needs a plan with train=True")
        ld_d = _checked(dout, self._x_shape, self.dtype, self._gpu, "dout")
        ld_y = _checked(y, self._r_shape, self.dtype, self._gpu, "y")
        st = self._lib.sq_exchange_combine_backward(
            dout.data_ptr(), y.data_ptr(), *self._r_size, ld_d, ld_y, self._slots(place, torch.int32, "place"),
            self._slots(share, torch.float32, "share"), *self._slots_of, *self._to_back, _on(self._gpu, stream))
        if st:
            _check("sq_exchange_combine_backward", st)
        return self.dR, self.dshare

    def dispatch_backward(self, drows: torch.Tensor, place: torch.Tensor, add: Optional[torch.Tensor] = None,
                          stream=None) -> torch.Tensor:
        if not self.train:
            raise ValueError("dispatch_backward needs a plan with train=True")
        self._combine(drows, place, None, add, self._to_dx, stream)
        return self.dX
