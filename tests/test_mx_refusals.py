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


def test_the_size_of_a_workspace_is_refused_where_the_call_is(mx):
    from paper_2411_10948_amd.shiftquant import load
    L, n = load(), ct.c_size_t(0)
    most = 1 << 20

    def size(M, K, N, e=0):
        return L.sq_mx_linear_workspace_size(M, K, N, e, ct.byref(n))

    def linear(M, K, N, off=None, e=0):
        # no workspace: what is not refused for its sizes is for that
        return L.sq_mx_linear(P, 0, M, K, K, off, e, P, P, N, P, 0, N, None, 0, None)

    for M, K, N in [(4096, most, 64), (4096, (1 << 23) - 1, 64), (1, most, 64), (4096, 64, most), (1 << 31, 64, 64)]:
        assert size(M, K, N) == INVALID and linear(M, K, N) == INVALID
    assert size(4096, 1 << 23, 64) == linear(4096, 1 << 23, 64) == UNSUPPORTED
    assert size(4096, 64, 64, 1 << 16) == linear(4096, 64, 64, P, 1 << 16) == INVALID
    assert size(4096, most - 1, 64) == 0 and n.value > 0
    for M, N in ((0, 64), (64, 0)):     # nothing to compute
        assert size(M, most, N) == 0 and n.value == 0 and linear(M, most, N) == 0


def test_the_workspace_of_split_sums(mx):
    # few tiles of a long inner axis: the partial sums are the caller's, and never written where there are none
    from paper_2411_10948_amd.shiftquant import load, sq_last_error
    L, n = load(), ct.c_size_t(0)
    odd = ct.c_void_p(0x100008)
    M, N, K = 64, 640, 30000
    assert L.sq_mx_gemm_workspace_size(M, N, K, ct.byref(n)) == 0 and n.value >= 2 * M * N * 4

    def gemm(ws, nws):
        return L.sq_mx_gemm(P, P, P, P, M, N, K, P, 0, N, ws, nws, None)

    assert gemm(None, n.value) == INVALID and "workspace" in sq_last_error()
    assert gemm(odd, n.value) == INVALID
    assert gemm(P, n.value - 1) == SMALL and gemm(P, 0) == SMALL
    part = n.value

    M, N, K = 128, 1024, 12288          # the same behind a quantizer: codes, scales and partial sums
    assert L.sq_mx_gemm_workspace_size(M, N, K, ct.byref(n)) == 0 and n.value >= 2 * M * N * 4
    part = n.value
    assert L.sq_mx_linear_workspace_size(M, K, N, 0, ct.byref(n)) == 0
    assert n.value >= sum(mx.sq_mx_size(M, K)) + part

    def linear(ws, nws):
        return L.sq_mx_linear(P, 0, M, K, K, None, 0, P, P, N, P, 0, N, ws, nws, None)

    assert linear(None, n.value) == INVALID and linear(odd, n.value) == INVALID and linear(P, n.value - 1) == SMALL
    assert linear(P, n.value - part) == SMALL
