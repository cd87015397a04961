"""Layer norm, router, exchange of rows and 8-bit dense layers on tensors of more than
2^31 elements or bytes: the last rows, columns and tokens against the same ones in a
small call or by themselves.  Every row is checked where the result is a copy."""
import pytest

pytestmark = pytest.mark.gpu

WIDE = (1 << 20) - 8       # columns, below the limit of 2^20
ROWS = 2100                # 2.2e9 elements


@pytest.fixture(autouse=True)
def freed():
    yield
    import torch
    torch.cuda.empty_cache()


def _randn(*shape):
    import torch
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)


def test_exchange():
    import torch
    from paper_2411_10948_amd import route
    x = _randn(ROWS, WIDE)
    place = torch.arange(ROWS - 1, -1, -1, dtype=torch.int32, device="cuda").view(-1, 1)
    p = route.ExchangePlan(ROWS, 1, WIDE, train=True)
    rows = p.dispatch(x, place)
    assert all((rows[ROWS - 1 - t] == x[t]).all() for t in range(ROWS))
    out = p.combine(rows, place, torch.full((ROWS, 1), 0.5, device="cuda"))
    assert all((out[t] == 0.5 * x[t]).all() for t in range(ROWS))
    dy, dshare = p.combine_backward(x, rows, place, torch.full((ROWS, 1), 2.0, device="cuda"))
    assert all((dy[ROWS - 1 - t] == 2 * x[t]).all() for t in range(ROWS))
    want = (x[-1].double() ** 2).sum()      # a thread adds 2^20 / 256 squares up, 2^-24 of the sum at most for each, then 8 sums
    assert abs(dshare[-1, 0].double() - want) <= (4096 + 8) * 2.0 ** -24 * want


def test_norm_of_long_rows():
    import torch
    from paper_2411_10948_amd import norm
    x, gamma, beta = _randn(ROWS, WIDE), torch.ones(WIDE, device="cuda"), torch.zeros(WIDE, device="cuda")
    p, one = norm.NormPlan(ROWS, WIDE, train=True), norm.NormPlan(1, WIDE, train=True)
    y = p.forward(x, gamma, beta)
    dx, dgamma, _ = p.backward(y, x, gamma)
    for t in (0, ROWS - 1):
        assert (one.forward(x[t:t + 1], gamma, beta) == y[t]).all()
        assert (one.backward(y[t:t + 1], x[t:t + 1], gamma)[0] == dx[t]).all()
    assert torch.isfinite(dgamma).all()


def test_norm_of_many_rows():
    import torch
    from paper_2411_10948_amd import norm
    M, C = (1 << 25) + 77, 64
    x, r, gamma, beta = _randn(M, C), _randn(M, C), torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    p, few = norm.NormPlan(M, C, residual=True, train=True), norm.NormPlan(99, C, residual=True, train=True)
    y = p.forward(x, gamma, beta, r)
    dx, dgamma, dbeta = p.backward(y, p.H, gamma)
    last = slice(M - 99, M)
    assert (few.forward(x[last], gamma, beta, r[last]) == y[last]).all() and (few.H == p.H[last]).all()
    assert (few.backward(y[last], few.H, gamma)[0] == dx[last]).all()
    # y's squares add up to almost one a row, each rounded to bf16 (2^-8 of it), sums of at most 2^17 rows in fp32
    assert ((dgamma / M - 1).abs() < 0.02).all() and torch.isfinite(dbeta).all()


def test_router():
    import torch
    from paper_2411_10948_amd import route
    T, E = (1 << 22) + 5, 520
    logits = _randn(T, E)
    p = route.RouterPlan(T, E, 2)
    share, chosen = p.forward(logits)
    offsets, place = p.offsets.long(), p.place.long()
    assert offsets[-1] == 2 * T and (torch.bincount(chosen.flatten().long(), minlength=E) == offsets.diff()).all()
    seen = torch.zeros(2 * T, dtype=torch.int8, device="cuda")
    seen[place.flatten()] = 1
    assert seen.all()
    e = chosen.flatten().long()
    assert ((place.flatten() >= offsets[e]) & (place.flatten() < offsets[e + 1])).all()
    few = route.RouterPlan(99, E, 2)
    s, c = few.forward(logits[-99:])
    assert (c == chosen[-99:]).all() and (s == share[-99:]).all()
    d = torch.ones(T, 2, device="cuda")
    d[:, 1] = 0
    g = p.backward(d, logits)
    assert (few.backward(d[-99:].contiguous(), logits[-99:]) == g[-99:]).all()


def _held(*shape):
    """+-{1, 2, 3, 4, 6, 8, 12, 15}: codes hold them whatever block they are in, and sums of 2^24 / 225 products are exact in
    any order."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    values = torch.tensor([1, 2, 3, 4, 6, 8, 12, 15, -1, -2, -3, -4, -6, -8, -12, -15], dtype=torch.bfloat16, device="cuda")
    return values[torch.randint(0, 16, shape, generator=g, device="cuda", dtype=torch.uint8).int()]


def test_products():
    import torch
    from paper_2411_10948_amd import f8
    N, K = 1 << 18, 16392      # 4.3e9 bytes of W's codes
    w = _held(N, K)
    codes, codes_t = f8.quantize(w, True, True, True)
    edge = f8.quantize(w[:, 16384:].contiguous(), True)[0].values()
    nc, ns = f8.sq_f8_size(8, N)
    assert (f8.F8Matrix(codes_t.codes[-nc:], codes_t.scales[-ns:], 8, N).values().t() == edge).all()
    tail = w[N - 100:].clone()
    del w, codes_t
    for m in (1, 70):
        x = _held(m, K)
        y = f8.LinearPlan(m, K, N).forward(x, codes)
        assert (y[:, N - 100:] == (x.double() @ tail.double().t()).bfloat16()).all()


def test_long_results():
    import torch
    from paper_2411_10948_amd import f8
    M, N, K = 66000, 33000, 130        # 2.2e9 elements
    x, w = _held(M, K), _held(N, K)
    b = f8.quantize(w, True)[0]
    y = f8.LinearPlan(M, K, N).forward(x, b)
    for part in (slice(0, 200), slice(M - 200, M)):
        assert (y[part] == (x[part].double() @ w.double().t()).bfloat16()).all()
    C = torch.empty(M, N, device="cuda")
    a = f8.quantize(x)[0]
    f8.sq_f8_gemm(a.codes, a.scales, b.codes, b.scales, K, C)
    assert (C[-200:].double() == x[-200:].double() @ w.double().t()).all()
