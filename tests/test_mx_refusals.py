"""Refusals of the microscaled 4-bit entry points that depend on more than one
argument (no GPU: every call is refused before a launch, no pointer is read)."""
import ctypes as ct
import os

import pytest

INVALID, UNSUPPORTED, SMALL = 1, 3, 4
P = ct.c_void_p(0x100000)


@pytest.fixture(scope="module")
def mx():
    from paper_2411_10948_amd import mx, shiftquant
    if not os.path.exists(shiftquant.LIB_PATH):
        from paper_2411_10948_amd import build
        build.build()
    return mx


def _layer(mx, **fields):
    sizes = dict(rows=256, c_in=64, c_out=64, experts=2, type=0, reserved=0, workspace_bytes=1 << 40)
    every = {**{name: 0x100000 for name, _ in mx.Layer._fields_}, **sizes, **fields}
    return ct.byref(mx.Layer(*(every[name] for name, _ in mx.Layer._fields_)))


def test_offsets_of_the_backward(mx):
    from paper_2411_10948_amd.shiftquant import load, sq_last_error
    L = load()

    def back(layer, offsets):
        return L.sq_mx_layer_backward(layer, P, 64, offsets, P, 64, P, 64, None)

    # neither the caller's nor a copy
    assert back(_layer(mx, offsets=None), None) == INVALID and "offsets" in sq_last_error()
    assert back(_layer(mx, offsets=0x100002), None) == INVALID and "offsets" in sq_last_error()
    assert back(_layer(mx, experts=0), P) == INVALID and "offsets" in sq_last_error()
    forward = L.sq_mx_layer_forward(_layer(mx, offsets=0x100002), P, 64, P, P, 64, None)
    assert forward == INVALID and "offsets" in sq_last_error()
    # the forward does not take the copy for the caller's
    assert L.sq_mx_layer_forward(_layer(mx), P, 64, None, P, 64, None) == INVALID
