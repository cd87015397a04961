"""Layer norm on the GPU against the plain implementation in 64 bits
(tests/block_reference.py): every way a row is held, odd sizes, strides, residual
sums, rows far from zero, NaN, other streams, graph replays."""
import numpy as np
import pytest

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
U = ref.U


@pytest.fixture(scope="module")
def norm():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2411_10948_amd import norm, shiftquant
    shiftquant.load()
    return norm


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _rand(rng, shape, dtype, scale=1.0, shift=0.0):
    import torch
    return torch.from_numpy((scale * rng.standard_normal(shape) + shift).astype(np.float32)).cuda().to(_dtype(dtype))


def _np(t):
    return t.detach().double().cpu().numpy()


def _round(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


def _within(got, want, tol, name):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / np.maximum(tol, 1e-300))}"


def _check(h, gamma, beta, eps, y, dtype, dy=None, dh=None, grads=None):
    """The kernel's additions: in a row at most 32 in a thread (C / 1024 where rows are too long for registers), 6 in a
    wave and 16 over the waves, so K roundings of a sum; xh = (h - mean) r is off by the mean's error, K U of the mean
    magnitude of what is left (at most 1 / r), and by half the variance's and a few roundings of its own."""
    M, C = h.shape
    K = 64 + C / 1024
    want, xh, r = ref.norm(h, gamma, beta, eps)
    off = (K + 8) * U * (1 + np.abs(xh))
    _within(y, want, np.abs(gamma) * off + 3 * U * (np.abs(xh * gamma) + np.abs(beta)) + (_round(dtype) * 1.01) * np.abs(want), "y")
    if grads is None:
        return
    dx, dg, db = grads
    wx, wg, wb = ref.norm_backward(h, gamma, eps, dy, 0.0 if dh is None else dh)
    q = np.abs(dy * gamma)
    B = (q * (1 + np.abs(xh))).mean(1, keepdims=True)
    tol = (3 * K + 32) * U * r * (q + q.mean(1, keepdims=True) + (1 + np.abs(xh)) * B) + 2 * U * np.abs(0.0 if dh is None else dh)
    _within(dx, wx, tol + _round(dtype) * (np.abs(wx) + tol), "dx")
    K2 = M / 64 + 64        # rows of a thread, row groups of a block, then blocks in 16 waves
    _within(dg, wg, (np.abs(dy) * (np.abs(xh) * K2 * U + off)).sum(0), "dgamma")
    _within(db, wb, np.abs(dy).sum(0) * K2 * U, "dbeta")


SIZES = [(1, 1), (3, 7), (5, 32), (4, 63), (9, 511), (3152, 64), (130, 768), (17, 769), (33, 1000), (6, 1025), (600, 2048),
         (7, 2050), (19, 4096), (5, 6001), (3, 8192), (4, 11008), (3, 16384), (2, 20001), (2, 32768), (2, 40000), (70, 33000)]


@pytest.mark.parametrize("dtype,param", [("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("M,C", SIZES)
def test_against_64_bits(norm, M, C, dtype, param):
    rng = np.random.default_rng(M * 100003 + C)
    residual = (M + C) % 2 == 0
    x, res, dy, dh = (_rand(rng, (M, C), dtype) for _ in range(4))
    g, b = _rand(rng, (C,), param, 0.3, 1.0), _rand(rng, (C,), param, 0.2)
    plan = norm.NormPlan(M, C, 1e-5, _dtype(dtype), _dtype(param), residual, train=True)
    y = plan.forward(x, g, b, res if residual else None)
    h = x
    if residual:
        h = plan.H
        assert (h == (x.float() + res.float()).to(x.dtype)).all()
    grads = plan.backward(dy, h, g, dh if residual else None)
    _check(_np(h), _np(g), _np(b), 1e-5, _np(y), dtype, _np(dy), _np(dh) if residual else None, [_np(t) for t in grads])
    serve = norm.NormPlan(M, C, 1e-5, _dtype(dtype), _dtype(param), residual)
    assert (serve.forward(x, g, b, res if residual else None) == y).all()
    with pytest.raises(ValueError):
        serve.backward(dy, h, g)


@pytest.mark.parametrize("C", [64, 1000, 5000, 40000])
def test_rows_far_from_zero(norm, C):
    # mean 3000 times the spread: the mean in one fp32 number would be off by 2e-4 of the spread
    rng = np.random.default_rng(C)
    x, dy = _rand(rng, (5, C), "f32", 1.0, 3000.0), _rand(rng, (5, C), "f32")
    g, b = _rand(rng, (C,), "f32", 0.3, 1.0), _rand(rng, (C,), "f32")
    plan = norm.NormPlan(5, C, 1e-5, _dtype("f32"), train=True)
    y = plan.forward(x, g, b)
    _check(_np(x), _np(g), _np(b), 1e-5, _np(y), "f32", _np(dy), None, [_np(t) for t in plan.backward(dy, x, g)])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift,pad", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_strided_and_misaligned(norm, dtype, shift, pad):
    rng = np.random.default_rng(shift)
    M, C = 13, 203

    def view():
        return _rand(rng, (M * (C + pad) + shift + C,), dtype)[shift:].as_strided((M, C), (C + pad, 1))
    x, res, dy, dh = view(), view(), view(), view()
    g, b = _rand(rng, (C,), "f32", 0.3, 1.0), _rand(rng, (C,), "f32")
    plan = norm.NormPlan(M, C, 1e-5, _dtype(dtype), residual=True, train=True)
    y = plan.forward(x, g, b, res)
    assert (plan.H == (x.float() + res.float()).to(x.dtype)).all()
    grads = plan.backward(dy, plan.H, g, dh)
    _check(_np(plan.H), _np(g), _np(b), 1e-5, _np(y), dtype, _np(dy), _np(dh), [_np(t) for t in grads])


@pytest.mark.parametrize("C", [200, 3000, 40000])
def test_nonfinite_rows_and_constant_rows(norm, C):
    import torch
    rng = np.random.default_rng(1)
    x, dy, g, b = _rand(rng, (6, C), "f32"), _rand(rng, (6, C), "f32"), _rand(rng, (C,), "f32"), _rand(rng, (C,), "f32")
    x[1, 5], x[2, 7], x[3, 0] = float("nan"), float("inf"), float("-inf")
    x[4] = 2.5          # no spread: y = beta
    plan = norm.NormPlan(6, C, 1e-5, torch.float32, train=True)
    y = plan.forward(x, g, b)
    dx, dg, db = plan.backward(dy, x, g)
    for t in (y, dx):
        assert t[1:4].isnan().all() and not t[[0, 4, 5]].isnan().any()
    assert (y[4] == b).all() and dg.isnan().all() and not db.isnan().any()


def test_no_rows(norm):
    import torch
    plan = norm.NormPlan(0, 96, train=True)
    x = torch.empty(0, 96, dtype=torch.bfloat16, device="cuda")
    g = torch.ones(96, device="cuda")
    assert plan.forward(x, g, g).shape == (0, 96)
    plan.dgamma.fill_(7), plan.dbeta.fill_(7)
    _, dg, db = plan.backward(x, x, g)
    assert not dg.any() and not db.any()


def test_in_place(norm):
    # H may be the residual's buffer, dX that of dH
    import torch
    rng = np.random.default_rng(3)
    x, res, dy, dh = (_rand(rng, (40, 300), "bf16") for _ in range(4))
    g, b = _rand(rng, (300,), "f32"), _rand(rng, (300,), "f32")
    plan = norm.NormPlan(40, 300, residual=True, train=True)
    want = plan.forward(x, g, b, res).clone()
    dx = plan.backward(dy, plan.H, g, dh)[0].clone()
    y, stats = torch.empty_like(want), torch.empty(40, 4, device="cuda")
    norm.sq_norm_forward(x, res, g, b, 1e-5, res, y, stats)
    assert (y == want).all() and (res == plan.H).all() and (stats == plan.stats).all()
    ws = torch.empty(norm.sq_norm_backward_workspace_size(40, 300), dtype=torch.uint8, device="cuda")
    dg, db = torch.empty(300, device="cuda"), torch.empty(300, device="cuda")
    norm.sq_norm_backward(dy, res, dh, g, stats, dh, dg, db, ws)
    assert (dh == dx).all() and (dg == plan.dgamma).all()


def test_rows_past_32_bit_elements(norm):
    # 2.2e9 elements a tensor: the last rows are those of a small call
    import torch
    M, C = 270000, 8192
    x = torch.zeros(M, C, dtype=torch.bfloat16, device="cuda")
    tail = _rand(np.random.default_rng(2), (3, C), "bf16")
    x[-3:] = tail
    g, b = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    plan, small = norm.NormPlan(M, C, train=True), norm.NormPlan(3, C, train=True)
    assert (plan.forward(x, g, b)[-3:] == small.forward(tail, g, b)).all()
    dy = torch.zeros_like(x)
    dy[-3:] = tail
    dx, dg, _ = plan.backward(dy, x, g)
    wx, wg, _ = small.backward(tail, tail, g)
    assert (dx[-3:] == wx).all() and torch.allclose(dg, wg, rtol=1e-5, atol=1e-4)


def test_other_stream_determinism_and_replays(norm):
    import torch
    rng = np.random.default_rng(4)
    M, C = 700, 1030
    x, res, dy, dh = (_rand(rng, (M, C), "bf16") for _ in range(4))
    g, b = _rand(rng, (C,), "f32"), _rand(rng, (C,), "f32")
    plan = norm.NormPlan(M, C, residual=True, train=True)

    def step():
        y = plan.forward(x, g, b, res)
        return (y, plan.H, *plan.backward(dy, plan.H, g, dh))
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [t.clone() for t in step()]
    s.synchronize()
    assert all((a == b_).all() for a, b_ in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = step()
    for i in range(3):
        x.copy_(_rand(rng, (M, C), "bf16"))
        eager = norm.NormPlan(M, C, residual=True, train=True)
        y = eager.forward(x, g, b, res)
        want = [t.clone() for t in (y, eager.H, *eager.backward(dy, eager.H, g, dh))]
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all((a == b_).all() for a, b_ in zip(out, want)), i
