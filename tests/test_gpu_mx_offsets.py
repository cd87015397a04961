"""Offsets of the products by expert: what a training plan keeps of them between
its forward and its backward pass, and the rows that they leave out."""
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


def _ints(values):
    import torch
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("M,K,N,first,then", [
    (1100, 96, 64, [0, 700, 700, 1050, 1100], [0, 20, 500, 600, 1100]),
    (256, 72, 40, [5, 37, 37, 200, 256], [0, 0, 0, 0, 256]),
    (3000, 520, 300, [0] * 70 + [1000] * 30 + [3000], list(range(0, 3000, 30)) + [3000])])
def test_backward_takes_the_forwards_split(mx, M, K, N, first, then, dtype):
    # one buffer of offsets that the program fills again before the backward pass
    import torch
    dt, E = getattr(torch, dtype), len(first) - 1
    g = torch.Generator(device="cuda").manual_seed(M)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)
    x, dy, w = r(M, K), r(M, N), r(E, N, K)
    plans = [mx.LinearPlan(M, K, N, dtype=dt, experts=E, train=True) for _ in range(2)]
    got = []
    for plan, rewrite in zip(plans, (False, True)):
        plan.dX.fill_(7.0)
        plan.quantize_weight(w)
        offsets = _ints(first)
        plan.forward(x, offsets=offsets)
        if rewrite:
            offsets.copy_(_ints(then[:E + 1]))
        got.append([t.clone() for t in plan.backward(dy)])
    for want, have in zip(*got):
        assert torch.equal(want, have)


def test_two_layers_share_one_buffer_of_offsets(mx):
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    M, K, N, splits = 600, 128, 96, ([0, 13, 400, 600], [0, 300, 310, 600])
    x, dy, w = r(M, K), r(M, N), r(3, N, K)
    alone, shared, buffer = [], [], _ints(splits[0])
    plans = [mx.LinearPlan(M, K, N, experts=3, train=True) for _ in splits]
    for plan, split in zip(plans, splits):
        plan.quantize_weight(w)
        plan.forward(x, offsets=_ints(split))
        alone.append([t.clone() for t in plan.backward(dy)])
    for plan, split in zip(plans, splits):
        buffer.copy_(_ints(split))
        plan.forward(x, offsets=buffer)
    for plan in plans:
        shared.append(plan.backward(dy))
    for a, b in zip(alone, shared):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
