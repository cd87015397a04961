"""Activations with 8-bit copies on the GPU against the plain implementation in 64
bits: the copy bit for bit, h and the gradients within fp32's rounding, the
gradient against differences, strides, odd widths, extremes."""
import numpy as np
import pytest

from tests import mx_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2411_10948_amd import mx, shiftquant
    shiftquant.load()
    return mx


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _want(kind, gated, F, x, dh):
    g = x[:, :F]
    if not gated:
        g8, code, s = ref.copy8(g)
        return ref.act(kind, g), dh * ref.act_slope(kind, g8), (code, s), None
    g8, gc, gs = ref.copy8(g)
    u8, uc, us = ref.copy8(x[:, F:])
    dx = np.concatenate([dh * u8 * ref.act_slope(kind, g8), dh * ref.act(kind, g8)], 1)
    return ref.act(kind, g) * x[:, F:], dx, (gc, gs), (uc, us)


def _close(got, want, scale, dtype):
    """Relative to `scale`, the result's factors: fp32 products and the sigmoid are each within a few 2^-23, its
    exponent's argument (|t| <= 88 where sigmoid is not 0 or 1) within 2^-24, and the slope's 1 + x (1 - s) t' adds a
    few terms of up to |x| t' s (1 - s) < 2: 64 * 2^-23 covers them.  Then one rounding to the type."""
    tol = 64 * 2.0 ** -23 * scale + 1e-37
    if dtype == "bf16":
        tol = tol + (np.abs(want) + tol) * 2.0 ** -8
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("M,F", [(1, 1), (1, 32), (3, 33), (17, 100), (64, 256), (129, 1000)])
def test_forward_and_backward(mx, M, F, gated, kind, dtype):
    import torch
    rng = np.random.default_rng(M + F)
    W = F * (2 if gated else 1)
    x = torch.from_numpy((rng.standard_normal((M, W)) * np.exp(rng.normal(0, 1.0, W)))).float().cuda().to(_dtype(dtype))
    dh = torch.from_numpy(rng.standard_normal((M, F)) * 0.01).float().cuda().to(_dtype(dtype))
    plan = mx.ActPlan(M, F, kind, gated, _dtype(dtype))
    h = plan.forward(x)
    dx = plan.backward(dh)
    xv, dv = x.double().cpu().numpy(), dh.double().cpu().numpy()
    wh, wdx, g, u = _want(kind, gated, F, xv, dv)
    fp = -(-F // 32) * 32
    codes = plan.codes.view(M, -1).cpu().numpy()
    scales = plan.scales.view(M, -1).cpu().numpy()
    for i, c in enumerate((g, u)):
        if c is not None:
            np.testing.assert_array_equal(codes[:, i * fp:i * fp + F], c[0].reshape(M, -1)[:, :F])
            np.testing.assert_array_equal(scales[:, i * fp // 32:(i + 1) * fp // 32], c[1])
    up = np.abs(xv[:, F:]) if gated else 1.0
    _close(h.double().cpu().numpy(), wh, (np.abs(xv[:, :F]) + 1) * up, dtype)
    g8 = ref.copy8(xv[:, :F])[0]
    scale = np.abs(dv) * (ref.copy8(xv[:, F:])[0].__abs__() if gated else 1.0)
    if gated:
        scale = np.concatenate([scale, np.abs(dv) * (np.abs(g8) + 1)], 1)
    _close(dx.double().cpu().numpy(), wdx, scale, dtype)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("gated", [False, True])
def test_gradient_against_differences(mx, kind, gated):
    # dL/dx of L = sum(dh h) on inputs that the copy holds exactly (whole 64ths below 2), differences of the 64-bit h
    import torch
    rng = np.random.default_rng(3)
    M, F = 8, 64
    W = F * (2 if gated else 1)
    x = rng.integers(-127, 128, (M, W)) / 64.0
    x[:, ::32] = 127 / 64.0
    dh = rng.standard_normal((M, F)).astype(np.float32)
    plan = mx.ActPlan(M, F, kind, gated, torch.float32)
    plan.forward(torch.from_numpy(x).float().cuda())
    dx = plan.backward(torch.from_numpy(dh).cuda()).double().cpu().numpy()

    def h(x):
        return ref.act(kind, x[:, :F]) * (x[:, F:] if gated else 1.0)
    e = 1e-5
    for _ in range(20):
        i, j = int(rng.integers(M)), int(rng.integers(W))
        up, down = x.copy(), x.copy()
        up[i, j] += e
        down[i, j] -= e
        d = (dh.astype(np.float64) * (h(up) - h(down))).sum() / (2 * e)
        # the difference's own error: third derivatives below 4, its terms' rounding; then fp32
        assert abs(dx[i, j] - d) <= (4 * e * e + 1e-10 + 64 * 2.0 ** -23) * 4 * (1 + np.abs(dh).max())


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_extremes(mx, kind):
    import torch
    x = torch.zeros(4, 64, device="cuda")
    x[0, :4] = torch.tensor([1e30, -1e30, 200.0, -200.0])
    x[0, 32:36] = torch.tensor([88.0, -88.0, 1e-30, -1e-30])
    x[1, 3] = float("nan")
    x[2, 40] = float("inf")
    plan = mx.ActPlan(4, 64, kind, False, torch.float32)
    h = plan.forward(x)
    dx = plan.backward(torch.ones(4, 64, device="cuda"))
    assert h[0, 0] == x[0, 0] and h[0, 1].abs() <= 1e-30 and h[0, 2] == 200.0 and h[0, 3].abs() <= 1e-30
    assert torch.isfinite(h[0]).all() and torch.isfinite(dx[0]).all()
    assert dx[0, 0] == 1.0 and dx[0, 1] == 0.0
    assert h[1].isnan().sum() == 1 and h[1, 3].isnan()
    assert h[2, 40] == float("inf")
    # the copy holds no NaN but a whole block of them
    assert dx[1, :32].isnan().all() and not dx[1, 32:].isnan().any()
    assert dx[2, 32:].isnan().all() and not dx[2, :32].isnan().any()
    assert (h[3] == 0).all() and (dx[3] == 0.5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", [64, 60])
def test_strides(mx, dtype, F):
    import torch
    rng = np.random.default_rng(4)
    M = 9
    dt = _dtype(dtype)
    x = torch.from_numpy(rng.standard_normal((M, 2 * F))).float().cuda().to(dt)
    dh = torch.from_numpy(rng.standard_normal((M, F))).float().cuda().to(dt)
    plan = mx.ActPlan(M, F, "silu", True, dt)
    want = plan.forward(x).clone(), plan.backward(dh).clone()
    wide = torch.zeros(M, 2 * F + 7, dtype=dt, device="cuda")[:, 3:3 + 2 * F]
    wide.copy_(x)
    d = torch.zeros(M, F + 5, dtype=dt, device="cuda")[:, 1:1 + F]
    d.copy_(dh)
    assert torch.equal(plan.forward(wide), want[0]) and torch.equal(plan.backward(d), want[1])


def test_more_than_one_launch(mx):
    # over 2^31 pieces of eight columns: the rows go in two launches; compared with a small call on the last rows
    import torch
    F = 32
    M = ((1 << 31) - 256) // 4 + 1000
    if torch.cuda.mem_get_info()[0] < 160e9:
        pytest.skip("needs 160 GB of GPU memory")
    n = 3000
    x = torch.zeros(M, F, dtype=torch.bfloat16, device="cuda")
    x[-n:] = torch.randn(n, F, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    plan, small = mx.ActPlan(M, F, "gelu", False), mx.ActPlan(n, F, "gelu", False)
    h = plan.forward(x)
    assert torch.equal(h[-n:], small.forward(x[-n:])) and not h[:4].any()
    assert torch.equal(plan.codes.view(M, F)[-n:], small.codes.view(n, F))
    dh = x          # any values
    assert torch.equal(plan.backward(dh)[-n:], small.backward(x[-n:]))
