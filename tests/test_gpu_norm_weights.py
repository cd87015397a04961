"""Gradients of layer norm's weights over tensors of more than 2^31 elements, every row
counted: against 64-bit sums, and with gradients in the first and last rows alone."""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24      # half a step of fp32, relative


@pytest.fixture(autouse=True)
def freed():
    yield
    import torch
    torch.cuda.empty_cache()


def _randn(*shape):
    import torch
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)


def _check(h, dy, dgamma, dbeta, eps, adds, step):
    """adds: additions of a sum over the rows, each off by U of the sum of magnitudes; xh is off by (72 + C / 1024) U of
    1 + |xh|, as the rows' sums are."""
    import torch
    M, C = h.shape
    off = (72 + C / 1024) * U
    g, b, mag_g, mag_b = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(4))
    for lo in range(0, M, step):
        x, d = h[lo:lo + step].double(), dy[lo:lo + step].double()
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        x = (x - mean) / torch.sqrt(var + eps)
        g += (d * x).sum(0)
        b += d.sum(0)
        d, x = d.abs(), x.abs()
        mag_g += (d * (x * (adds * U + off) + off)).sum(0)
        mag_b += d.sum(0)
    assert ((dgamma - g).abs() <= mag_g).all(), ((dgamma - g).abs() / mag_g).max()
    assert ((dbeta - b).abs() <= adds * U * mag_b).all(), ((dbeta - b).abs() / mag_b).max()


def _edges(M, C, many):
    """Rows without a gradient add exact zeros: those with one are all there is."""
    import torch
    from paper_2411_10948_amd import norm
    x, dy, gamma, beta = _randn(M, C), torch.zeros(M, C, dtype=torch.bfloat16, device="cuda"), torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    at = torch.cat([torch.arange(many), torch.arange(M - many, M)]).cuda()
    dy[at] = _randn(2 * many, C)
    p = norm.NormPlan(M, C, train=True)
    p.forward(x, gamma, beta)
    _, dgamma, dbeta = p.backward(dy, x, gamma)
    _check(x[at], dy[at], dgamma, dbeta, 1e-5, 2 * many, 2 * many)


def test_many_rows():
    import torch
    from paper_2411_10948_amd import norm
    M, C = (1 << 25) + 77, 64
    x, gamma, beta = _randn(M, C), torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    p = norm.NormPlan(M, C, train=True)
    y = p.forward(x, gamma, beta)
    _, dgamma, dbeta = p.backward(y, x, gamma)
    # 512 blocks of 8 rows at a time, the 8, then the blocks in 32 sums and these
    _check(x, y, dgamma, dbeta, 1e-5, M / 4096 + 8 + 16 + 32, 1 << 21)


def test_first_and_last_of_many_rows():
    _edges((1 << 25) + 77, 64, 50)


def test_long_rows():
    import torch
    from paper_2411_10948_amd import norm
    M, C = 2100, (1 << 20) - 8
    x, dy, gamma, beta = _randn(M, C), _randn(M, C), torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    p = norm.NormPlan(M, C, train=True)
    p.forward(x, gamma, beta)
    _, dgamma, dbeta = p.backward(dy, x, gamma)
    # every 64th row a thread, 2 of these 64 sums each of 32 threads, then these
    _check(x, dy, dgamma, dbeta, 1e-5, M / 64 + 2 + 32, 60)


def test_first_and_last_of_long_rows():
    _edges(2100, (1 << 20) - 8, 2)
