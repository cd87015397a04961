"""The 8-bit format's plain implementation (tests/f8_reference.py) against its
definition, and the refusals of the 8-bit entry points (no GPU: every call is
refused, or has nothing to do, before a launch; no pointer is read)."""
import ctypes as ct
import os

import numpy as np
import pytest

from tests import f8_reference as ref

INVALID, UNSUPPORTED, SMALL = 1, 3, 4
P, ODD = ct.c_void_p(0x100000), ct.c_void_p(0x100008)


@pytest.fixture(scope="module")
def L():
    from paper_2411_10948_amd import shiftquant
    if not os.path.exists(shiftquant.LIB_PATH):
        from paper_2411_10948_amd import build
        build.build()
    return shiftquant.load()


def test_elements():
    import torch
    assert len(ref.E4M3) == 127 and ref.E4M3[-1] == 448 and ref.E4M3[8] == 2.0 ** -6 and ref.E4M3[1] == 2.0 ** -9
    assert (torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy() == ref.E4M3).all()


def test_rounding_and_scales():
    import torch
    x = np.zeros((4, 128))
    x[0, :5] = [464, 1, 3.0625, 2.0 ** -10, -(2.0 ** -9) * 1.5]
    x[1, 0] = 464.5
    x[2, 0] = -29.0
    k, s = ref.f8_codes(x)
    assert s[0, 0] == 127 and s[1, 0] == 128 and s[2, 0] == 123 and s[3, 0] == 0
    assert ref.f8_values(x)[0, :5].tolist() == [448, 1, 3.0, 0.0, -2.0 ** -8]       # ties to the even code
    assert ref.f8_values(x)[2, 0] == -28.0
    # unit scale: torch's conversion
    v = np.random.default_rng(0).uniform(-448, 448, (8, 128)) * 2.0 ** np.random.default_rng(1).integers(-16, 1, (8, 128))
    v[:, 0] = 448
    got = ref.f8_codes(v.astype(np.float32))[0]
    assert (torch.from_numpy(v.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy() == got).all()
    # half a step at most: 2^-4 of a normal element
    big = np.random.default_rng(2).standard_normal((300, 260)) * np.exp(3 * np.random.default_rng(3).standard_normal(260))
    for square in (False, True):
        k, s = ref.f8_codes(big, square)
        err = np.abs(ref.f8_values(big, square) - big)
        assert (err <= np.maximum(2.0 ** -4 * np.abs(big), 2.0 ** -10 * 2.0 ** (s - 127.0))).all()
    a, t = ref.f8_values(big, True), ref.f8_values(big.T, True)
    assert (a == t.T).all()


def test_layout_is_one_to_one():
    for rows, cols in ((1, 1), (33, 130), (16, 512), (20, 1030)):
        b, s = ref.f8_places(rows, cols)
        assert len(np.unique(b)) == rows * cols
        assert all(len(np.unique(s[:, c:c + 128])) == rows for c in range(0, cols, 128))


def test_held_numbers_are_held():
    x = ref.held(np.random.default_rng(0), 130, 260)
    assert (ref.f8_values(x) == x).all() and (ref.f8_values(x, True) == x).all()


# ---------------------------------------------------------------------------
def _size(f, *args):
    n = ct.c_size_t(0)
    return f(*args, ct.byref(n)), n.value


def test_sizes(L):
    a, b = ct.c_size_t(0), ct.c_size_t(0)
    for rows, cols, c, s in ((0, 5, 0, 0), (5, 0, 0, 0), (1, 1, 8192, 64), (17, 513, 4 * 8192, 256)):
        assert L.sq_f8_size(rows, cols, ct.byref(a), ct.byref(b)) == 0 and (a.value, b.value) == (c, s)
    assert L.sq_f8_size(-1, 5, ct.byref(a), ct.byref(b)) == L.sq_f8_size(5, 5, None, ct.byref(b)) == INVALID


def test_quantize_refusals(L):
    ok = [P, 0, 300, 64, 64, 0, P, P, P, P, None]
    for i, bad in ((0, None), (0, ct.c_void_p(0x100001)), (1, 2), (2, -1), (2, 1 << 31), (3, 1 << 20), (4, 63), (5, 2), (6, None),
                   (6, ODD), (7, None), (7, ct.c_void_p(0x100002)), (8, None), (8, ODD), (9, None)):
        assert L.sq_f8_quantize(*ok[:i], bad, *ok[i + 1:]) == INVALID, (i, bad)
    assert L.sq_f8_quantize(*ok[:6], None, None, None, None, None) == INVALID
    assert L.sq_f8_quantize(P, 0, 1 << 22, 64, 64, 0, None, None, P, P, None) == UNSUPPORTED
    assert L.sq_f8_quantize(P, 0, (1 << 31) - 1, (1 << 20) - 1, 1 << 20, 0, P, P, None, None, None) == UNSUPPORTED
    assert L.sq_f8_quantize(None, 0, 0, 64, 64, 0, None, None, None, None, None) == 0


def test_product_refusals(L):
    ok = [P, P, P, P, 64, 64, 128, P, 0, 64, None, 0, None]
    for i, bad in ((0, None), (1, None), (2, ODD), (3, None), (4, -1), (5, -1), (6, -1), (7, None), (8, 2), (9, 63)):
        assert L.sq_f8_gemm(*ok[:i], bad, *ok[i + 1:]) == INVALID, (i, bad)
    assert L.sq_f8_gemm(*ok[:6], 1 << 22, *ok[7:]) == UNSUPPORTED
    assert L.sq_f8_gemm(*ok[:4], 0, *ok[5:]) == 0
    # few tiles of a long inner axis: the partial sums are the caller's
    status, need = _size(L.sq_f8_gemm_workspace_size, 64, 64, 30000)
    assert status == 0 and need >= 2 * 64 * 64 * 4
    split = [P, P, P, P, 64, 64, 30000, P, 0, 64]
    assert L.sq_f8_gemm(*split, None, need, None) == L.sq_f8_gemm(*split, ODD, need, None) == INVALID
    assert L.sq_f8_gemm(*split, P, need - 1, None) == SMALL
    assert _size(L.sq_f8_gemm_workspace_size, 64, 64, 1 << 22)[0] == UNSUPPORTED


def test_linear_refusals(L):
    M, K, N = 300, 512, 4096
    status, need = _size(L.sq_f8_linear_workspace_size, M, K, N)
    assert status == 0 and need >= 304 * 512
    ok = [P, 0, M, K, K, P, P, N, P, 0, N, P, need, None]
    for i, bad in ((0, None), (1, 3), (2, -1), (3, 1 << 20), (4, K - 1), (5, None), (6, None), (7, 1 << 20), (8, None), (9, -1),
                   (10, N - 1), (11, None), (11, ODD)):
        assert L.sq_f8_linear(*ok[:i], bad, *ok[i + 1:]) == INVALID, (i, bad)
    assert L.sq_f8_linear(*ok[:12], need - 1, None) == SMALL
    assert _size(L.sq_f8_linear_workspace_size, M, 1 << 20, N)[0] == INVALID
    assert _size(L.sq_f8_linear_workspace_size, 16, 4096, 4096) == (0, 0)       # one launch
    assert L.sq_f8_linear(*ok[:2], 0, *ok[3:]) == 0


def test_layer_refusals(L):
    from paper_2411_10948_amd import f8

    def layer(**fields):
        sizes = dict(rows=256, c_in=64, c_out=64, type=0, reserved=0, workspace_bytes=1 << 40)
        every = {**{name: 0x100000 for name, _ in f8.Layer._fields_}, **sizes, **fields}
        return ct.byref(f8.Layer(*(every[name] for name, _ in f8.Layer._fields_)))

    def forward(l):
        return L.sq_f8_layer_forward(l, P, 64, P, 64, None)

    def backward(l, x=P, w=P, ld=64):
        return L.sq_f8_layer_backward(l, P, ld, x, ld, w, ld, None)
    for bad in (dict(rows=-1), dict(c_in=1 << 20), dict(type=2), dict(w=0), dict(x_scales=0), dict(x_t=0x100008)):
        assert forward(layer(**bad)) == INVALID, bad
    for bad in (dict(w_t=0), dict(dy=0), dict(dy_t_scales=0), dict(x_t=0)):
        assert backward(layer(**bad)) == INVALID, bad
    assert backward(layer(), x=None) == backward(layer(), w=None) == backward(layer(), ld=63) == INVALID
    assert forward(layer(rows=1 << 22)) == backward(layer(rows=1 << 22)) == UNSUPPORTED
    assert L.sq_f8_layer_weight(None, P, 64, None) == L.sq_f8_layer_weight(layer(), None, 64, None) == INVALID
    long = dict(rows=30000)         # the weight gradient is split
    status, need = _size(lambda *a: L.sq_f8_layer_workspace_size(layer(**long), *a))
    assert status == 0 and need > 0
    assert backward(layer(workspace=0, **long)) == INVALID and backward(layer(workspace_bytes=need - 1, **long)) == SMALL


def test_plan_refusals():
    import torch
    from paper_2411_10948_amd import f8
    kw = dict(device="cpu")     # buffers alone: no call reaches a launch
    with pytest.raises(TypeError):
        f8.LinearPlan(4, 64, 64, dtype=torch.float16, **kw)
    plan, x = f8.LinearPlan(4, 64, 32, **kw), torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="plan's GPU"):
        plan.forward(x, f8.F8Matrix.empty(32, 64, "cpu"))
    for call in (plan.quantize_weight, plan.backward):
        with pytest.raises(ValueError, match="train"):
            call(x)
    with pytest.raises(ValueError, match="codes"):
        f8.F8Matrix(torch.zeros(8191, dtype=torch.uint8), torch.zeros(64, dtype=torch.uint8), 16, 512)
