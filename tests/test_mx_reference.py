"""The 64-bit plain implementation that the GPU tests of the microscaled 4-bit
path compare against, pinned on hand-computed values and on its own
definitions, and the refusals of the entry points (no GPU)."""
import ctypes as ct
import os

import numpy as np
import pytest

from tests import mx_reference as ref


@pytest.fixture(scope="module")
def mx():
    from paper_2411_10948_amd import mx, shiftquant
    if not os.path.exists(shiftquant.LIB_PATH):
        from paper_2411_10948_amd import build
        build.build()
    return mx


def test_scale_and_ties_by_hand():
    x = np.zeros(32)
    x[:12] = [7.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.75, -5.0, 6.99, 0.26]
    k, s = ref.mx_codes(x)
    assert s[0] == 127          # 7 still fits scale 1
    assert list(k[0, :12]) == [7, 6, 6, 4, 4, 2, 2, 0, 8 | 2, 8 | 6, 7, 1]
    x[0] = np.nextafter(7.0, 8.0)
    assert ref.mx_codes(x)[1][0] == 128
    assert ref.mx_codes(np.zeros(5))[1][0] == 0
    assert ref.mx_codes(np.array([2.0 ** -130]))[1][0] == 0
    assert ref.mx_codes(np.array([np.inf, 1.0]))[1][0] == 255
    v, code, s = ref.copy8(np.array([127.49, 63.5, -1.0]))
    assert s[0] == 127 and list(code[0, :3]) == [127, 64, -1]
    v, code, s = ref.copy8(np.array([127.5]))
    assert s[0] == 128 and code[0, 0] == 64


def test_no_element_is_off_by_more_than_half_a_step():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((64, 96)) * np.exp(rng.normal(0, 3, (64, 1)))
    s = np.repeat(ref.mx_codes(x)[1].astype(np.int64), 32, -1)[:, :96]
    v = np.abs(x) / 2.0 ** (s - 127)
    step = np.where(v < 2, 0.5, np.where(v < 4, 1.0, 2.0))
    assert (np.abs(ref.mx_values(x) - x) <= 0.5 * step * 2.0 ** (s - 127)).all()
    v, code, s = ref.copy8(x)
    assert np.abs(code).max() <= 127
    assert (np.abs(v - x) <= 0.5 * np.repeat(2.0 ** (s.astype(np.int64) - 127), 32, -1)).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 512), (17, 513), (40, 1300)])
def test_layout_is_a_bijection(mx, rows, cols):
    byte, nib, sc = ref.mx_places(rows, cols)
    nc, ns = mx.sq_mx_size(rows, cols)
    assert byte.max() < nc and sc.max() < ns
    assert len(np.unique(byte * 2 + nib)) == rows * cols
    blocks = np.unique(np.stack([sc.ravel(), np.repeat(np.arange(rows), cols), np.tile(np.arange(cols) // 32, rows)]), axis=1)
    assert blocks.shape[1] == rows * -(-cols // 32) == len(np.unique(sc))


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_slope_against_differences(kind):
    x = np.linspace(-6, 6, 97)
    h = 1e-5
    d = (ref.act(kind, x + h) - ref.act(kind, x - h)) / (2 * h)
    # second-order differences of functions with third derivatives below 4, and their rounding
    np.testing.assert_allclose(ref.act_slope(kind, x), d, rtol=0, atol=4 * h * h + 2e-15 * 10 / h)


def test_sizes(mx):
    assert mx.sq_mx_size(17, 513) == (2 * 2 * 4096, 2 * 2 * 256)
    assert mx.sq_mx_size(0, 5) == (0, 0)
    assert mx.sq_mx_segment_cols(100, 4) % 512 == 0
    rng = np.random.default_rng(1)
    for _ in range(200):        # room for every split
        rows, experts = int(rng.integers(0, 3000)), int(rng.integers(1, 40))
        cut = np.sort(rng.integers(0, rows + 1, experts - 1))
        off = np.concatenate([[0], cut, [rows]])
        need = sum(-(-(b - a) // 512) * 512 for a, b in ref.segments(off))
        assert need <= mx.sq_mx_segment_cols(rows, experts)
    assert mx.sq_mx_segment_cols(20, 20) == 20 * 512       # and no more than the worst one
    assert mx.sq_act_size(3, 33, True) == (3 * 128, 3 * 4)
    assert mx.sq_mx_linear_workspace_size(16, 4096, 4096) == 0
    assert mx.sq_mx_linear_workspace_size(100, 4096, 4096, 64) == 0
    assert mx.sq_mx_linear_workspace_size(4096, 512, 512) > 0


def test_refusals(mx):
    from paper_2411_10948_amd.shiftquant import load, sq_last_error
    L = load()
    p, odd = ct.c_void_p(0x100000), ct.c_void_p(0x100008)     # never read on the host
    n = ct.c_size_t(0)
    INVALID, UNSUPPORTED, SMALL = 1, 3, 4

    def q(X=p, type=0, batch=1, rows=8, cols=8, ld=8, stride=0, off=None, e=0, c=p, s=p, ct_=None, st=None):
        return L.sq_mx_quantize(X, type, batch, rows, cols, ld, stride, off, e, c, s, ct_, st, None)

    assert q(X=None) == INVALID and "X is NULL" in sq_last_error()
    assert q(type=2) == INVALID
    assert q(ld=7) == INVALID
    assert q(c=None, s=None) == INVALID
    assert q(s=None) == INVALID
    assert q(c=odd) == INVALID
    assert q(rows=-1) == INVALID
    assert q(cols=1 << 20, ld=1 << 20) == INVALID
    assert q(batch=2, stride=63) == INVALID
    assert q(off=p, e=0) == INVALID and q(off=None, e=3) == INVALID
    assert q(off=p, e=3, batch=2, stride=64) == INVALID
    assert q(X=ct.c_void_p(0x100002)) == INVALID
    assert q(rows=1 << 23, ct_=p, st=p) == UNSUPPORTED
    assert q(rows=0) == 0 and q(cols=0) == 0 and q(batch=0, X=None) == 0

    def g(A=p, M=1024, N=1024, K=8192, C=p, type=0, ldc=1024, ws=p, nws=1 << 40):
        return L.sq_mx_gemm(A, p, p, p, M, N, K, C, type, ldc, ws, nws, None)

    assert L.sq_mx_gemm_workspace_size(1024, 1024, 8192, ct.byref(n)) == 0
    assert g(A=None) == INVALID and g(A=odd) == INVALID and g(C=None) == INVALID
    assert g(ldc=1023) == INVALID and g(type=5) == INVALID and g(M=-1) == INVALID
    assert g(K=1 << 23) == UNSUPPORTED
    if n.value:
        assert g(ws=None) == INVALID and g(nws=n.value - 1) == SMALL
    assert L.sq_mx_gemm(None, None, None, None, 0, 5, 5, None, 0, 5, None, 0, None) == 0

    def ge(off=p, e=4, M=64, N=64, K=64, C=p, ldc=64):
        return L.sq_mx_gemm_experts(p, p, M, K, off, e, p, p, N, C, 0, ldc, None)

    assert ge(off=None) == INVALID and ge(e=0) == INVALID and ge(C=None) == INVALID and ge(e=1 << 16) == INVALID
    assert ge(M=0) == 0

    def gw(rows=64, off=p, e=4, M=64, N=64, C=p, ldc=64):
        return L.sq_mx_gemm_experts_wgrad(p, p, p, p, rows, off, e, M, N, C, 0, ldc, p, 1 << 40, None)

    assert gw(rows=1 << 23) == UNSUPPORTED and gw(off=None) == INVALID and gw(ldc=63) == INVALID and gw(e=0) == INVALID
    assert gw(M=0) == 0

    def lin(X=p, M=4096, K=512, ld=512, off=None, e=0, N=512, Y=p, ldy=512, ws=p, nws=1 << 40):
        return L.sq_mx_linear(X, 1, M, K, ld, off, e, p, p, N, Y, 1, ldy, ws, nws, None)

    assert lin(X=None) == INVALID and lin(ld=511) == INVALID and lin(ldy=511) == INVALID and lin(ws=None) == INVALID
    assert lin(nws=16) == SMALL and lin(off=p) == INVALID and lin(M=0) == 0

    from paper_2411_10948_amd.mx import Layer
    def layer(**kw):
        names = [f[0] for f in Layer._fields_]
        v = dict(rows=65536, c_in=64, c_out=64, experts=0, type=0, reserved=0, workspace_bytes=1 << 40)
        return Layer(*({**{n: 0x100000 for n in names}, **v, **kw}[n] for n in names))
    ref_ = lambda **kw: ct.byref(layer(**kw))
    assert L.sq_mx_layer_workspace_size(None, ct.byref(n)) == INVALID
    assert L.sq_mx_layer_workspace_size(ref_(type=7), ct.byref(n)) == INVALID
    assert L.sq_mx_layer_workspace_size(ref_(rows=1 << 23), ct.byref(n)) == UNSUPPORTED
    assert L.sq_mx_layer_workspace_size(ref_(), ct.byref(n)) == 0 and n.value > 0      # dW of one tile, 512 steps
    assert L.sq_mx_layer_weight(ref_(), None, 64, 0, None) == INVALID
    assert L.sq_mx_layer_weight(ref_(), p, 63, 0, None) == INVALID
    assert L.sq_mx_layer_forward(ref_(), None, 64, None, p, 64, None) == INVALID
    assert L.sq_mx_layer_forward(ref_(), p, 64, p, p, 64, None) == INVALID             # offsets without experts
    assert L.sq_mx_layer_forward(ref_(experts=2), p, 64, None, p, 64, None) == INVALID
    assert L.sq_mx_layer_forward(ref_(), p, 64, None, p, 63, None) == INVALID
    assert L.sq_mx_layer_forward(ref_(x_t=0x100008), p, 64, None, p, 64, None) == INVALID
    assert L.sq_mx_layer_forward(ref_(workspace_bytes=16), p, 64, None, p, 64, None) == SMALL
    back = lambda l, dY=p, dX=p, dW=p, ldw=64: L.sq_mx_layer_backward(l, dY, 64, None, dX, 64, dW, ldw, None)
    assert back(ref_(), dY=None) == INVALID and back(ref_(), dX=None) == INVALID and back(ref_(), dW=None) == INVALID
    assert back(ref_(), ldw=63) == INVALID and back(ref_(w_t=None)) == INVALID and back(ref_(workspace=None)) == INVALID

    def af(X=p, kind=0, gated=1, M=4, F=64, ldx=128, H=p, ldh=64, c=p, s=p):
        return L.sq_act_forward(X, 0, kind, gated, M, F, ldx, H, ldh, c, s, None)

    def ab(dH=p, kind=0, gated=1, M=4, F=64, ldh=64, c=p, s=p, dX=p, ldx=128):
        return L.sq_act_backward(dH, 0, kind, gated, M, F, ldh, c, s, dX, ldx, None)

    for f in (af, ab):
        assert f(kind=2) == INVALID and f(gated=2) == INVALID and f(ldx=127) == INVALID and f(ldh=63) == INVALID
        assert f(c=None) == INVALID and f(c=odd) == INVALID and f(s=None) == INVALID and f(M=-1) == INVALID
        assert f(M=0) == 0
    assert af(X=None) == INVALID and af(H=None) == INVALID and ab(dH=None) == INVALID and ab(dX=None) == INVALID


def test_binding_refusals(mx):
    import torch
    with pytest.raises(TypeError):
        mx.LinearPlan(4, 8, 8, dtype=torch.float16, device="cpu")
    with pytest.raises(ValueError):
        mx.ActPlan(4, 8, act="relu", device="cpu")
    with pytest.raises(ValueError):
        mx.MxMatrix(torch.empty(10, dtype=torch.uint8), torch.empty(10, dtype=torch.uint8), 8, 8)
    plan = mx.LinearPlan(4, 8, 6, dtype=torch.float32, experts=3, device="cpu")
    x = torch.zeros(4, 8)
    w = mx.MxMatrix.empty(6, 8, 3, "cpu")
    with pytest.raises(ValueError):
        plan.forward(torch.zeros(4, 9), w)
    with pytest.raises(ValueError):
        plan.forward(x, w, torch.zeros(3, dtype=torch.int32))       # experts + 1 offsets
    with pytest.raises(ValueError):
        plan.forward(x, w, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        plan.forward(x, None, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        plan.forward(x, mx.MxMatrix.empty(6, 8, 2, "cpu"), torch.zeros(4, dtype=torch.int32))   # a stack of 2
    with pytest.raises(ValueError):
        plan.forward(x, w, torch.zeros(4, dtype=torch.int32))       # tensors that are not on the GPU
    with pytest.raises(ValueError):
        plan.backward(torch.zeros(4, 6))


def test_refusals_of_layer_buffers(mx):
    """Codes that one of the two products reads and the other does not."""
    from paper_2411_10948_amd.mx import Layer
    from paper_2411_10948_amd.shiftquant import load
    L, p = load(), ct.c_void_p(0x100000)        # never read: every call is refused
    sizes = dict(rows=256, c_in=64, c_out=64, experts=0, type=0, reserved=0, workspace_bytes=1 << 40)
    for name in ("x", "dy", "x_t", "dy_t", "w", "w_t"):
        for field in (name, name + "_scales"):
            for bad in (None, 0x100002):
                layer = Layer(*({**{f[0]: 0x100000 for f in Layer._fields_}, **sizes, field: bad}[f[0]] for f in Layer._fields_))
                if name in ("x", "w"):
                    assert L.sq_mx_layer_forward(ct.byref(layer), p, 64, None, p, 64, None) == 1
                else:
                    assert L.sq_mx_layer_backward(ct.byref(layer), p, 64, None, p, 64, p, 64, None) == 1


def test_refusals_of_places_and_sizes(mx):
    import torch
    b = lambda n: torch.empty(n, dtype=torch.uint8)
    nc, ns = mx.sq_mx_size(16, 512)
    out = torch.empty(16, 16)
    with pytest.raises(ValueError, match="on the GPU"):
        mx.sq_mx_gemm(b(nc), b(ns), b(nc), b(ns), 512, out)
    with pytest.raises(ValueError, match="on the GPU"):
        mx.sq_mx_dequantize(b(nc), b(ns), 16, 512, torch.empty(16, 512))
    with pytest.raises(ValueError, match="H|X"):
        mx.sq_act_forward(torch.empty(4, 64), mx.ACT_SILU, True, torch.empty(4, 64), b(512), b(16))
    plan = mx.LinearPlan(4, 8, 6, dtype=torch.float32, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        plan.forward(torch.zeros(4, 8), mx.MxMatrix.empty(6, 8, 0, "cpu"))
