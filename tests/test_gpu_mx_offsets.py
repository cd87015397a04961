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


OUTSIDE = [(2000, 520, 700, [300, 300, 900, 1500]), (4100, 300, 600, [0, 5, 4000]), (2100, 1030, 800, [2050, 2051, 2100]),
           (3000, 256, 1100, [7] * 9)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("M,K,N,off", OUTSIDE)
def test_rows_outside_are_left_alone(mx, M, K, N, off, dtype):
    # the serving call that quantizes first: its codes of rows that no expert has, and their outputs, keep what they held
    import torch
    dt, E = getattr(torch, dtype), len(off) - 1
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randn(M, K, generator=g, device="cuda").to(dt)
    w = torch.randn(E, N, K, generator=g, device="cuda").to(dt)
    plan = mx.LinearPlan(M, K, N, dtype=dt, experts=E)
    assert plan.ws is not None      # not the call of few rows, which has no codes
    plan.ws.fill_(0x5A)
    plan.Y.fill_(7.0)
    y = plan.forward(x, mx.quantize(w)[0], _ints(off)).double().cpu().numpy()
    byte, _, sc = ref.mx_places(M, K)
    ws, at = plan.ws.cpu().numpy(), -(-mx.sq_mx_size(M, K)[0] // 256) * 256
    out = np.ones(M, bool)
    out[off[0]:off[-1]] = False
    assert (ws[byte][out] == 0x5A).all() and (ws[at:][sc][out] == 0x5A).all() and (y[out] == 7.0).all()
    xv, wv = x.double().cpu().numpy(), w.double().cpu().numpy()
    codes, scales = ref.mx_unpack(ws, ws[at:], M, K)
    k, s = ref.mx_codes(xv)
    np.testing.assert_array_equal(codes[~out], k.reshape(M, -1)[~out, :K])
    np.testing.assert_array_equal(scales[~out], np.repeat(s, 32, -1)[~out, :K])
    for e, (lo, hi) in enumerate(ref.segments(off)):
        if hi == lo:
            continue
        want, mag = ref.mx_product(ref.mx_values(xv[lo:hi]), ref.mx_values(wv[e]))
        tol = mag * (K + 2) * 2.0 ** -23        # an fp32 sum of K exact products, then one rounding
        if dtype == "bfloat16":
            tol = tol + (np.abs(want) + tol) * 2.0 ** -8
        assert (np.abs(y[lo:hi] - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("off", [[0, 64, 256], [5, 37, 37, 200], [0] * 70 + [3] * 30 + [250], [17, 17], [130, 131], [256, 256]])
def test_quantize_rows_by_expert(mx, off, dtype):
    # codes along the columns alone, with offsets: inside as ever, outside untouched
    import torch
    M, C, E = 256, 200, len(off) - 1
    x = torch.randn(M, C, generator=torch.Generator(device="cuda").manual_seed(E), device="cuda").to(getattr(torch, dtype))
    a = mx.MxMatrix.empty(M, C)
    a.codes.fill_(0x5A)
    a.scales.fill_(0x5A)
    mx.sq_mx_quantize(x, a.codes, a.scales, None, None, _ints(off), E)
    byte, _, sc = ref.mx_places(M, C)
    codes, scales = a.codes.view(-1).cpu().numpy(), a.scales.view(-1).cpu().numpy()
    out = np.ones(M, bool)
    out[off[0]:off[-1]] = False
    assert (codes[byte][out] == 0x5A).all() and (scales[sc][out] == 0x5A).all()
    got, s8 = ref.mx_unpack(codes, scales, M, C)
    k, s = ref.mx_codes(x.double().cpu().numpy())
    np.testing.assert_array_equal(got[~out], k.reshape(M, -1)[~out, :C])
    np.testing.assert_array_equal(s8[~out], np.repeat(s, 32, -1)[~out, :C])
