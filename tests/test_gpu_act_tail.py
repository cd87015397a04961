"""Relative accuracy of the fp32 activations where the sigmoid is small."""
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


def _grid(lo, hi):
    """fp32 values, 64 rows of 64"""
    return np.linspace(lo, hi, 4096).astype(np.float32).reshape(64, 64)


def _forward(mx, kind, x):
    import torch
    plan = mx.ActPlan(*x.shape, kind, gated=False, dtype=torch.float32)
    return plan, plan.forward(torch.from_numpy(x).cuda()).double().cpu().numpy()


def test_silu(mx):
    # e = exp(-|x|) within 1 ulp of a normal fp32 (2^-23), 1 + e rounded (2^-24), its reciprocal within 1 ulp, two
    # products rounded: 2^-23 (1 + 1/2 + 1 + 1/2 + 1/2), 4 with the terms of second order
    x = _grid(-87.0, -4.0)
    want = ref.act("silu", x.astype(np.float64))
    got = _forward(mx, "silu", x)[1]
    assert (np.abs(got - want) <= 4 * 2.0 ** -23 * np.abs(want)).all(), np.max(np.abs(got / want - 1)) * 2 ** 23


def test_gelu(mx):
    # t = k (x + b x^3): five roundings and those of k and b, 7 * 2^-24 of |t|, which the exponential turns into as
    # much of a relative error; the rest as above
    x = _grid(-9.0, -2.0)
    v = x.astype(np.float64)
    t = 2 * np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3)
    want = v / (1 + np.exp(-t))         # 1 + tanh would cancel
    keep = t > -87.0
    got = _forward(mx, "gelu", x)[1]
    assert (np.abs(got - want) <= (8 * np.abs(t) + 8) * 2.0 ** -24 * np.abs(want))[keep].all()


def test_silu_slope(mx):
    # at values that the 8-bit copy holds, halves up to 63.5; sg as above, x sg, 1 - sg, their product and the sum
    # rounded (the terms have one sign past x = -1.3 but for the 1 in x - 1 ...: |x| / (|x| - 1) < 1.06 at |x| >= 20), dh
    import torch
    x = -np.tile(np.concatenate([np.arange(40, 71), [127]]), (8, 2)).astype(np.float32) / 2
    x[4:, :31] = -np.arange(97, 128)[::-1] / 2
    plan, _ = _forward(mx, "silu", x)
    dh = np.random.default_rng(0).standard_normal(x.shape).astype(np.float32)
    got = plan.backward(torch.from_numpy(dh).cuda()).double().cpu().numpy()
    want = dh.astype(np.float64) * ref.act_slope("silu", x.astype(np.float64))
    assert (np.abs(got - want) <= 8 * 2.0 ** -23 * np.abs(want)).all(), np.max(np.abs(got / want - 1)) * 2 ** 23


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_far_ends(mx, kind):
    # past the exponential's range: 0 (or what is below the smallest normal number) on one side, x on the other
    x = np.array([[-1e30, -200.0, -105.0, 0.0, -0.0, 105.0, 200.0, 1e30]], np.float32)
    h = _forward(mx, kind, x)[1][0]
    assert (np.abs(h[:3]) <= 2.0 ** -126 * 128).all() and (h[3:5] == 0).all() and (h[5:] == x[0, 5:]).all()
