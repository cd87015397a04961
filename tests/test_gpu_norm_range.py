"""Layer norm of rows whose squares leave fp32's range, up or (with no eps to hide it)
down, in every way a row is held, against the plain implementation in 64 bits."""
import numpy as np
import pytest

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
U = ref.U
# floats a row: one to four pieces a thread of a wave, blocks of 256 and 512 threads, too long for registers
WIDTHS = [1, 2, 64, 300, 1000, 1501, 2048, 4096, 6001, 16384, 40000]


def _check(h, gamma, beta, eps, y, dy, dh, grads, half):
    """A row's sum is off by at most K U of the sum of its magnitudes: 32 additions in a thread (C / 1024 where rows are
    too long for registers), 6 in a wave, 16 over the waves; that of xh by as much of the deviations' mean, by half the
    variance's and a few roundings of its own (the scale is a power of two); results are rounded once."""
    M, C = h.shape
    K = 64 + C / 1024
    want, xh, r = ref.norm(h, gamma, beta, eps)
    off = (K + 8) * U * (1 + np.abs(xh))
    tol = np.abs(gamma) * off + 3 * U * (np.abs(xh * gamma) + np.abs(beta))
    assert (np.abs(y - want) <= tol + half * (np.abs(want) + tol)).all()
    dx, dg, db = grads
    wx, wg, wb = ref.norm_backward(h, gamma, eps, dy, dh)
    q = np.abs(dy * gamma)
    B = (q * (1 + np.abs(xh))).mean(1, keepdims=True)
    tol = (3 * K + 32) * U * r * (q + q.mean(1, keepdims=True) + (1 + np.abs(xh)) * B) + 2 * U * np.abs(dh)
    assert (np.abs(dx - wx) <= tol + half * (np.abs(wx) + tol) + 2.0 ** -126).all()
    K2 = M / 64 + 64        # rows of a thread, row groups of a block, then blocks in 16 waves
    assert (np.abs(dg - wg) <= (np.abs(dy) * (np.abs(xh) * K2 * U + off)).sum(0)).all()
    assert (np.abs(db - wb) <= np.abs(dy).sum(0) * K2 * U).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_rows_of_every_size(C, dtype):
    import torch
    from paper_2411_10948_amd import norm
    dt, half = (torch.float32, U) if dtype == "f32" else (torch.bfloat16, 2.0 ** -8)
    rng = np.random.default_rng(C)
    # sums of C magnitudes below 2^128; a row alone, with an addend, and between rows of ordinary size
    sizes = np.array([1.0, 2.0 ** 62, 1.0, 2.0 ** 64, 2.0 ** 70, 2.0 ** 104, 2.0 ** 45, 1.0])[:, None]
    t = lambda v: torch.from_numpy(v.astype(np.float32)).cuda().to(dt)
    x, res = (t(sizes * rng.standard_normal((8, C)) + 0.5 * sizes) for _ in range(2))
    dy, dh = t(rng.standard_normal((8, C))), t(rng.standard_normal((8, C)))
    g, b = (torch.from_numpy(v.astype(np.float32)).cuda() for v in (1 + 0.3 * rng.standard_normal(C), 0.2 * rng.standard_normal(C)))
    n = lambda v: v.double().cpu().numpy()
    for with_res in (False, True):
        plan = norm.NormPlan(8, C, 1e-5, dt, residual=with_res, train=True)
        y = plan.forward(x, g, b, res if with_res else None)
        h = plan.H if with_res else x
        grads = plan.backward(dy, h, g, dh)
        _check(n(h), n(g), n(b), 1e-5, n(y), n(dy), n(dh), [n(v) for v in grads], half)


@pytest.mark.parametrize("eps", [0.0, 1e-37])
@pytest.mark.parametrize("C", [2, 64, 300, 1501, 4096, 6001, 40000])
def test_rows_of_small_values(C, eps):
    # one that fp32's smallest squares would lose, next to rows of ordinary size and of zeros
    import torch
    from paper_2411_10948_amd import norm
    rng = np.random.default_rng(C)
    sizes = np.array([1.0, 2.0 ** -60, 2.0 ** -70, 2.0 ** -100, 2.0 ** -50, 1.0])[:, None]
    x = torch.from_numpy((sizes * rng.standard_normal((6, C))).astype(np.float32)).cuda()
    dy = torch.from_numpy((sizes * rng.standard_normal((6, C))).astype(np.float32)).cuda()
    g, b = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    plan = norm.NormPlan(6, C, eps, torch.float32, train=True)
    n = lambda v: v.double().cpu().numpy()
    eps = float(np.float32(eps))
    y = plan.forward(x, g, b)
    _check(n(x), n(g), n(b), eps, n(y), n(dy), np.zeros((6, C)), [n(v) for v in plan.backward(dy, x, g)], U)
    if eps:
        x[2] = 0.0
        assert not plan.forward(x, g, b)[2].any()


def test_sums_past_the_range_are_no_numbers():
    # not a finite result that is wrong
    import torch
    from paper_2411_10948_amd import norm
    for C in (64, 4096, 40000):
        x = torch.randn(3, C, device="cuda")
        x[1] = 3e38 * (1 + x[1].abs()) / 4
        g, b = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
        plan = norm.NormPlan(3, C, dtype=torch.float32, train=True)
        y = plan.forward(x, g, b)
        assert y[1].isnan().all() and not y[[0, 2]].isnan().any()
        dx = plan.backward(torch.ones_like(x), x, g)[0]
        assert dx[1].isnan().all() and not dx[[0, 2]].isnan().any()
