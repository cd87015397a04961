"""Router and exchange of rows on the GPU against the plain implementation in 64
bits (tests/block_reference.py): choices and places equal, ties, groups, biases,
tokens without experts, NaN, strides, other streams, graph replays."""
import numpy as np
import pytest

from tests import block_reference as ref

pytestmark = pytest.mark.gpu
U = ref.U
# Shares: an fp32 sum of at most 1024 exponentials (22 additions one after the other, each term to 2 ulp) and one
# rounding, 32 U at most.  Gradients: twice that, relative to the magnitudes of their terms.
SHARE, GRAD = 32 * U, 64 * U


@pytest.fixture(scope="module")
def route():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2411_10948_amd import route, shiftquant
    shiftquant.load()
    return route


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _cuda(x, dtype="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(_dtype(dtype))


def _np(t):
    return t.detach().double().cpu().numpy()


def _check(route, logits, k, score="softmax", bias=None, groups=1, top_groups=1, renorm=False, scale=1.0, seed=0):
    """logits: a tensor on the GPU; forward and backward against the reference"""
    T, E = logits.shape
    l = _np(logits)
    dtype = "f32" if logits.element_size() == 4 else "bf16"
    b = None if bias is None else _cuda(bias)
    plan = route.RouterPlan(T, E, k, score, groups, top_groups, renorm, scale, dtype=logits.dtype)
    share, chosen = plan.forward(logits, b)
    # Sums of different scores can be equal but for their rounding (sigma(1) + sigma(-1) = sigma(2) + sigma(-2) = 1): a
    # total of two scores below 1 and two biases, each score off by its exponential's and its quotient's rounding, is
    # off by less than 16 2^-53, two of them by 2^-48 together, and either order is right.
    ws, wc, wp, wo = ref.route(l, k, score, None if bias is None else _np(b), groups, top_groups, renorm, scale,
                               chosen.cpu().numpy(), 2.0 ** -48)
    np.testing.assert_array_equal(chosen.cpu().numpy(), wc)
    np.testing.assert_array_equal(plan.place.cpu().numpy(), wp)
    np.testing.assert_array_equal(plan.offsets.cpu().numpy(), wo)
    np.testing.assert_array_equal(np.isnan(_np(share)), np.isnan(ws))
    ok = ~np.isnan(ws)
    # fp32's smallest normal: what rounds below it
    assert (np.abs(_np(share) - ws)[ok] <= (SHARE * np.abs(ws) + 2.0 ** -126)[ok]).all()
    d = np.random.default_rng(seed).standard_normal((T, k)).astype(np.float32)
    got = _np(plan.backward(_cuda(d), logits))
    nan = np.isnan(ws).any(1)
    assert np.isnan(got[nan]).all()
    with np.errstate(invalid="ignore"):
        want, mag = ref.route_backward(np.where(nan[:, None], 0.0, l), np.where(nan[:, None], -1, wc), d.astype(np.float64), score, renorm, scale)
    tol = GRAD * mag + 2.0 ** -126
    if dtype == "bf16":
        tol = tol + (np.abs(want) + tol) * 2.0 ** -8
    bad = ~(np.abs(got - want) <= tol)[~nan]
    assert not bad.any(), f"{bad.sum()} gradients off, worst {np.nanmax((np.abs(got - want) / tol)[~nan])}"
    return plan


RULES = [dict(), dict(renorm=True), dict(score="sigmoid"), dict(score="sigmoid", renorm=True, scale=2.5),
         dict(bias=True), dict(score="sigmoid", bias=True, renorm=True), dict(groups=4, top_groups=2, scale=0.5),
         dict(score="sigmoid", groups=4, top_groups=1, bias=True, renorm=True), dict(groups=4, top_groups=3, renorm=True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rule", range(len(RULES)))
@pytest.mark.parametrize("T,E,k", [(1, 64, 8), (1, 4, 1), (3, 12, 2), (64, 8, 2), (65, 100, 5), (200, 256, 8), (130, 512, 16),
                                   (40, 1024, 10), (700, 60, 6)])
def test_against_64_bits(route, T, E, k, rule, dtype):
    rng = np.random.default_rng(T * 7919 + E * 31 + rule)
    r = dict(RULES[rule])
    if r.get("groups"):
        k = min(k, E // r["groups"] * r["top_groups"])
    if r.pop("bias", None):
        r["bias"] = 0.1 * rng.standard_normal(E)
    logits = 1.5 * rng.standard_normal((T, E)) + 0.5 * rng.standard_normal(E)
    logits[T // 2:T // 2 + T // 10] = -np.inf           # padding
    _check(route, _cuda(logits, dtype), k, seed=rule, **r)


@pytest.mark.parametrize("groups,top_groups", [(1, 1), (2, 1), (3, 2), (5, 5), (6, 1), (15, 4), (30, 11), (60, 7)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_ties_go_to_the_lowest_index(route, groups, top_groups, score):
    rng = np.random.default_rng(groups)
    logits = rng.integers(-2, 3, (150, 60)).astype(np.float64)
    logits[rng.random((150, 60)) < 0.3] = -np.inf
    logits[3], logits[4] = 0.0, -np.inf
    logits[5], logits[5, ::2] = 0.0, -0.0       # equal
    logits[6], logits[6, 37] = -np.inf, -5.0    # one expert
    k = min(9, 60 // groups * top_groups)
    for bias in (None, 0.25 * rng.integers(-1, 2, 60)):
        _check(route, _cuda(logits), k, score, bias, groups, top_groups, renorm=True)


@pytest.mark.parametrize("k", [1, 8, 14, 15, 16, 20])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [1, 4])
def test_sums_that_fp32_cannot_tell_apart(route, score, groups, k):
    # experts an ulp of their logits apart, in runs of equal and of nearly equal ones, under biases that hide it in fp32
    rng = np.random.default_rng(k)
    step = np.float32(0.5) + rng.integers(0, 40, (60, 96)) * np.float32(2.0 ** -24)
    for bias in (np.full(96, 0.75), np.zeros(96), np.repeat([1.0, -1.0, 0.5], 32)):
        _check(route, _cuda(step), k, score, bias, groups, groups, renorm=True)
    step[:, ::3] = rng.standard_normal((60, 32))
    _check(route, _cuda(step), k, score, 0.1 * rng.standard_normal(96), groups, max(1, groups - 1))


@pytest.mark.parametrize("E,groups,top_groups", [(64, 16, 5), (256, 8, 4), (512, 4, 2), (1000, 10, 7)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_groups_that_fp32_cannot_tell_apart(route, score, E, groups, top_groups):
    # the same logits in every group, each in an order of its own, the highest up to two ulp apart; some tokens with NaN
    rng = np.random.default_rng(E)
    per = E // groups
    v = np.sort(rng.standard_normal((130, 1, per)).astype(np.float32), 2).repeat(groups, 1)
    for _ in range(2):
        up = rng.random((130, groups)) < 0.4
        v[:, :, -1] = np.where(up, np.nextafter(v[:, :, -1], np.float32(9)), v[:, :, -1])
    logits = rng.permuted(v, axis=2).reshape(130, E)
    logits[::9, 3] = np.nan
    for bias in (None, np.full(E, 0.25)):
        _check(route, _cuda(logits), 6, score, bias, groups, top_groups, renorm=True)


@pytest.mark.parametrize("E,k", [(1, 1), (5, 5), (64, 64), (65, 64), (1024, 64)])
def test_every_expert_chosen(route, E, k):
    _check(route, _cuda(np.random.default_rng(E).standard_normal((70, E))), k, renorm=True)
    _check(route, _cuda(np.random.default_rng(E).standard_normal((70, E))), k, "sigmoid")


@pytest.mark.parametrize("rule", [dict(), dict(score="sigmoid", renorm=True), dict(bias=True), dict(score="sigmoid", groups=2)])
def test_nonfinite_and_extreme_logits(route, rule):
    r = dict(rule)
    rng = np.random.default_rng(9)
    l = rng.standard_normal((12, 8))
    l[0, 3], l[1, 7], l[2, 0] = np.nan, np.inf, -np.inf
    l[3], l[4] = np.finfo(np.float32).min, np.finfo(np.float32).max     # masks of the type's lowest value
    l[5] = -200.0 + l[5]                # scores below fp32's range under sigmoid
    l[6] = -800.0 + l[6]                # and below fp64's
    l[7] = 90.0 * l[7]
    l[8], l[8, 2] = -np.inf, np.nan
    l[9], l[9, 4] = np.finfo(np.float32).min, 0.0
    if r.pop("bias", None):
        r["bias"] = np.array([0.0, 1.0, -1.0, 0.0, 0.5, 0.0, 0.0, -np.inf])
    _check(route, _cuda(l), 3, **r)


def test_a_bias_that_is_nan_or_infinite(route):
    import torch
    l = np.random.default_rng(1).standard_normal((4, 6))
    l[0, 2] = -np.inf
    _check(route, _cuda(l), 2, bias=np.array([0, 0, np.nan, 0, 0, 0.0]))     # of an expert that token 0 cannot have
    plan = _check(route, _cuda(l), 2, bias=np.array([0, np.inf, 0, 0, np.inf, 0.0]))
    assert plan.chosen.cpu().tolist() == [[1, 4]] * 4
    assert isinstance(plan.share, torch.Tensor)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift,pad", [(0, 1), (1, 3), (4, 0)])
def test_strided_logits(route, dtype, shift, pad):
    T, E = 90, 48
    base = _cuda(np.random.default_rng(shift).standard_normal(T * (E + pad) + shift + E), dtype)
    _check(route, base[shift:].as_strided((T, E), (E + pad, 1)), 4, renorm=True)


@pytest.mark.parametrize("T,E,k", [(30000, 16, 2), (5000, 256, 8)])
def test_many_tokens(route, T, E, k):
    # places of many blocks of tokens, some experts without rows
    import torch
    g = torch.Generator(device="cuda").manual_seed(T)
    logits = torch.randn(T, E, generator=g, device="cuda") + 2 * torch.randn(E, generator=g, device="cuda")
    logits[:, E // 2] = -float("inf")
    plan = route.RouterPlan(T, E, k, dtype=torch.float32)
    share, chosen = plan.forward(logits)
    want = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    assert (chosen == want).all()
    flat = chosen.reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    assert (plan.place.reshape(-1)[order] == torch.arange(T * k, device="cuda")).all()
    counts = torch.zeros(E, dtype=torch.long, device="cuda").index_add_(0, flat, torch.ones_like(flat))
    assert (plan.offsets[1:].long() == torch.cumsum(counts, 0)).all() and plan.offsets[0] == 0
    p = torch.softmax(logits.double(), 1).gather(1, chosen.long())
    assert ((share.double() - p).abs() <= SHARE * p).all()


def test_no_tokens(route):
    import torch
    plan = route.RouterPlan(0, 8, 2)
    plan.offsets.fill_(5)
    l = torch.empty(0, 8, dtype=torch.bfloat16, device="cuda")
    share, _ = plan.forward(l)
    assert share.shape == (0, 2) and not plan.offsets.any()
    assert plan.backward(share, l).shape == (0, 8)
    ex = route.ExchangePlan(0, 2, 64, train=True)
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    assert ex.dispatch(x, plan.place).shape == (0, 64) and ex.combine(x, plan.place, share).shape == (0, 64)
    ex.combine_backward(x, x, plan.place, share), ex.dispatch_backward(x, plan.place)


def test_gradient_in_place(route):
    import torch
    l = _cuda(np.random.default_rng(5).standard_normal((33, 20)))
    for score, renorm in (("softmax", False), ("softmax", True), ("sigmoid", False)):
        plan = route.RouterPlan(33, 20, 3, score, renormalize=renorm, dtype=torch.float32)
        plan.forward(l)
        d = torch.randn(33, 3, device="cuda")
        want, at = plan.backward(d, l).clone(), l.clone()
        route.sq_route_backward(d, at, route.SCORES[score], renorm, 1.0, plan.share, plan.chosen, at)
        assert (at == want).all()


# ---------------------------------------------------------------------------
def _exchange(route, T, k, D, dtype, holes=0.0, shift=0, pad=0):
    import torch
    rng = np.random.default_rng(T * 131 + k * 17 + D)
    place = rng.permutation(T * k).reshape(T, k).astype(np.int32)
    place[rng.random((T, k)) < holes] = -1
    share = rng.standard_normal((T, k)).astype(np.float32)

    def rows(n):
        base = _cuda(rng.standard_normal(n * (D + pad) + shift + D), dtype)
        return base[shift:].as_strided((n, D), (D + pad, 1))
    x, y, add, dout, drows, more = rows(T), rows(T * k), rows(T), rows(T), rows(T * k), rows(T)
    plan = route.ExchangePlan(T, k, D, _dtype(dtype), train=True)
    p, s = torch.from_numpy(place).cuda(), torch.from_numpy(share).cuda()
    plan.R.fill_(3.0), plan.dR.fill_(5.0)
    one = 2.0 ** -8 if dtype == "bf16" else U       # one rounding to the type
    np.testing.assert_array_equal(_np(plan.dispatch(x, p)), ref.dispatch(_np(x), place, np.full((T * k, D), 3.0)))

    def near(got, want, mag, terms, rnd):
        tol = (terms + 1) * U * mag
        assert (np.abs(_np(got) - want) <= tol + rnd * (np.abs(want) + tol)).all()
    for a in (None, add):
        near(plan.combine(y, p, s, a), *ref.combine(_np(y), place, share.astype(np.float64), 0.0 if a is None else _np(a)), k, one)
    for a in (None, more):
        near(plan.dispatch_backward(drows, p, a), *ref.combine(_np(drows), place, None, 0.0 if a is None else _np(a)), k, one)
    dy, dshare = plan.combine_backward(dout, y, p, s)
    wy, ws, mag = ref.combine_backward(_np(dout), _np(y), place, share.astype(np.float64), np.full((T * k, D), 5.0))
    near(dy, wy, np.abs(wy), 0, one)
    # D / 64 pieces of 16 bytes a lane at most, 6 additions in the wave, 3 more over the waves
    near(dshare, ws, mag, min(D, D / 64 + 8) + 9, 0.0)
    return plan


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,D", [(1, 8, 2048), (1, 1, 1), (3, 2, 7), (5, 3, 64), (40, 8, 1000), (129, 1, 130), (33, 9, 513),
                                   (7, 64, 96), (300, 2, 1024), (2, 17, 8192), (4, 2, 30001)])
def test_exchange(route, T, k, D, dtype):
    _exchange(route, T, k, D, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift,pad,holes", [(0, 0, 0.3), (1, 0, 0.0), (3, 5, 0.5), (8, 8, 1.0)])
def test_exchange_strided_and_without_rows(route, dtype, shift, pad, holes):
    _exchange(route, 30, 3, 202, dtype, holes, shift, pad)
    _exchange(route, 10, 3, 1202, dtype, holes, shift, pad)


def test_places_outside_of_the_rows_are_none(route):
    import torch
    place = torch.tensor([[0, 4], [-7, 2], [3, 2147483647]], dtype=torch.int32, device="cuda")
    share = torch.ones(3, 2, device="cuda")
    share[0, 1], share[1, 0] = float("nan"), float("inf")       # of no row
    x, R = torch.randn(3, 40, device="cuda"), torch.full((4, 40), 9.0, device="cuda")
    route.sq_exchange_dispatch(x, place, R)
    assert (R[0] == x[0]).all() and (R[1] == 9).all() and (R[2] == x[1]).all() and (R[3] == x[2]).all()
    out, dR, dshare = torch.empty(3, 40, device="cuda"), torch.full((4, 40), 9.0, device="cuda"), torch.empty(3, 2, device="cuda")
    route.sq_exchange_combine(R, place, share, None, out)
    assert (out == x).all()
    route.sq_exchange_combine_backward(x, R, place, share, dR, dshare)
    assert (dR[[0, 2, 3]] == x).all() and (dR[1] == 9).all()
    assert dshare[0, 1] == 0 and dshare[1, 0] == 0 and dshare[2, 1] == 0
    R = torch.empty(0, 40, device="cuda")                       # no rows at all
    route.sq_exchange_dispatch(x, place, R)
    route.sq_exchange_combine(R, place, share, x, out)
    assert (out == x).all()
    route.sq_exchange_combine_backward(x, R, place, share, R, dshare)
    assert not dshare.any()


def test_nan_of_rows_that_no_token_has_stays_out(route):
    import torch
    place = torch.tensor([[1, -1]], dtype=torch.int32, device="cuda")
    y = torch.full((2, 100), float("nan"), device="cuda")
    y[1] = 2.0
    plan = route.ExchangePlan(1, 2, 100, torch.float32, train=True)
    share = torch.tensor([[0.5, 0.0]], device="cuda")
    assert (plan.combine(y, place, share) == 1.0).all()
    dy, dshare = plan.combine_backward(torch.ones(1, 100, device="cuda"), y, place, share)
    assert dshare.tolist() == [[200.0, 0.0]] and (dy[1] == 0.5).all() and not dy[0].any()


def test_rows_past_32_bit_elements(route):
    import torch
    T, k, D = 33000, 8, 8192            # 2.16e9 elements of sorted rows
    plan = route.ExchangePlan(T, k, D)
    x = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.arange(D, device="cuda") % 251
    place = torch.arange(T * k, dtype=torch.int32, device="cuda").view(T, k)
    R = plan.dispatch(x, place)
    assert (R[-k:] == x[-1]).all() and not R[-k - 8:-k].any()
    share = torch.zeros(T, k, device="cuda")
    share[-1, -1] = 1.0
    out = plan.combine(R, place, share)
    assert (out[-1] == x[-1]).all() and not out[:-1].any()


def test_router_and_exchange_together_on_a_stream_and_in_a_graph(route):
    import torch
    T, E, k, D = 300, 24, 4, 520
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    logits, bias, x, dout = r(T, E), 0.1 * r(E), r(T, D), r(T, D)
    dt = torch.float32

    def make():
        return (route.RouterPlan(T, E, k, "sigmoid", 4, 2, True, 2.5, dtype=dt), route.ExchangePlan(T, k, D, dt, train=True))

    def step(router, ex):
        share, chosen = router.forward(logits, bias)
        rows = ex.dispatch(x, router.place)
        out = ex.combine(rows, router.place, share)
        dy, dshare = ex.combine_backward(dout, rows, router.place, share)
        dx = ex.dispatch_backward(dy, router.place)
        return share, chosen, router.place, router.offsets, rows, out, dy, dshare, dx, router.backward(dshare, logits)
    mine = make()
    want = [t.clone() for t in step(*mine)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [t.clone() for t in step(*mine)]
    s.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))
    # x is its rows' sum times the shares' sum, 2.5: shares to 32 U, k additions
    total = want[0].double().sum(1, keepdim=True)
    assert ((want[5].double() - x.double() * total).abs() <= 8 * U * (x.double().abs() * total)).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = step(*mine)
    for i in range(4):
        logits.copy_(r(T, E))
        x.copy_(r(T, D))
        if i == 2:
            logits[100:160] = -float("inf")
        want = [t.clone() for t in step(*make())]
        if i == 2:
            assert want[3][-1] == (T - 60) * k
        graph.replay()
        torch.cuda.synchronize()
        live = int(want[3][-1])
        for a, b in zip(out, want):
            n = live if a.shape[0] == T * k else a.shape[0]     # rows behind the last one stay as they were
            assert (a[:n] == b[:n]).all(), i
