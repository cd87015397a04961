"""Choices under biases of +-Inf and of fp32's largest values: sums s + bias that are
equal go to the lowest index on every path of the router, whatever lane and register
their experts are in."""
import numpy as np
import pytest

from tests import block_reference as ref

pytestmark = pytest.mark.gpu

INF, MOST = float("inf"), float(np.finfo(np.float32).max)


def _check(logits, k, score, bias, groups=1, top_groups=1):
    import torch
    from paper_2411_10948_amd import route
    T, E = logits.shape
    l, b = logits.astype(np.float32), bias.astype(np.float32)
    plan = route.RouterPlan(T, E, k, score, groups, top_groups, dtype=torch.float32)
    share, chosen = plan.forward(torch.from_numpy(l).cuda(), torch.from_numpy(b).cuda())
    ws, wc, wp, wo = ref.route(l.astype(np.float64), k, score, b.astype(np.float64), groups, top_groups)
    np.testing.assert_array_equal(chosen.cpu().numpy(), wc)
    np.testing.assert_array_equal(plan.place.cpu().numpy(), wp)
    np.testing.assert_array_equal(plan.offsets.cpu().numpy(), wo)
    # an fp32 sum of at most 512 exponentials, 14 additions one after the other, each term to 2 ulp, and one rounding: below 32 U
    assert (np.abs(share.double().cpu().numpy() - ws) <= 32 * ref.U * ws).all()
    return chosen


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k", [(17, 1), (64, 2), (64, 4), (100, 8), (256, 8), (256, 14), (300, 15), (512, 16), (512, 3), (600, 4)])
def test_more_infinite_biases_than_slots(score, E, k):
    rng = np.random.default_rng(E * 64 + k)
    logits = rng.standard_normal((70, E))
    for some in (k, k + 1, k + 2, k + 3, E):
        for high in (INF, MOST):
            bias = 0.1 * rng.standard_normal(E)
            at = rng.permutation(E)
            bias[at[:some]] = high
            bias[at[some:some + 3]] = -high
            _check(logits, k, score, bias)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_equal_sums_that_are_infinite(score):
    bias = np.zeros(64)
    bias[[3, 4, 8, 12, 16]] = INF
    logits = np.random.default_rng(0).standard_normal((5, 64))
    assert _check(logits, 2, score, bias).tolist() == [[3, 4]] * 5
    assert _check(logits, 4, score, np.full(64, INF)).tolist() == [[0, 1, 2, 3]] * 5
    assert _check(logits, 4, score, np.full(64, -INF)).tolist() == [[-1] * 4] * 5


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups,top_groups", [(64, 4, 2), (256, 8, 4), (512, 4, 1), (480, 16, 5)])
def test_infinite_biases_in_groups(score, E, groups, top_groups):
    rng = np.random.default_rng(E)
    logits = rng.standard_normal((70, E))
    logits[::7, ::5] = -INF
    for high in (INF, MOST):
        for part in (0.05, 0.4, 1.0):
            bias = np.where(rng.random(E) < part, high, 0.1 * rng.standard_normal(E))
            _check(logits, 6, score, bias, groups, top_groups)
