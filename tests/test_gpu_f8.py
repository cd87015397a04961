"""Dense layers in 8-bit floating point on the GPU against the plain implementation
in 64 bits (tests/f8_reference.py): codes and scales byte for byte in their
documented places, products within the bound of an fp32 sum and equal where sums
are exact, strided and misaligned inputs, NaN, other streams, graph replays."""
import numpy as np
import pytest

from tests import f8_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def f8():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2411_10948_amd import f8, shiftquant
    shiftquant.load()
    return f8


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _cuda(x, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().to(_dtype(dtype))


def _rand(rng, shape, dtype, spread=1.0):
    return _cuda(rng.standard_normal(shape) * np.exp(rng.normal(0, spread, (shape[-1],))), dtype)


def _np(t):
    return t.detach().double().cpu().numpy()


def _check_matrix(m, want, rows, cols):
    byte, sc = ref.f8_places(rows, cols)
    k, s = want
    np.testing.assert_array_equal(m.scales.cpu().numpy()[sc], s)
    np.testing.assert_array_equal(m.codes.cpu().numpy()[byte], k)


def _pieces(v):
    """The largest magnitude of each 16 elements of the inner axis."""
    v = np.pad(np.abs(v), ((0, 0), (0, -v.shape[1] % 16)))
    return v.reshape(v.shape[0], -1, 16).max(2)


def _close(got, a, b, dtype):
    """a b^T within the error of an fp32 sum of K exact products in any order (at most 2^-23 of the running sum for each
    addition, were they cut and not rounded); in bf16 one rounding, and sums of 16 products first, each of which is cut 13
    bits below the largest one's exponent: off by less than 15 2^-13 of that product (which is exact), and products are
    at most those of the pieces' largest elements."""
    want, tol = a @ b.T, (np.abs(a) @ np.abs(b).T) * (a.shape[1] + 2) * 2.0 ** -23
    if dtype == "bf16":
        tol = tol + 15 * 2.0 ** -13 * (_pieces(a) @ _pieces(b).T)
        tol = tol + (np.abs(want) + tol) * 2.0 ** -8
    bad = ~(np.abs(_np(got) - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(_np(got) - want) / np.maximum(tol, 1e-300))}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("M,C", [(1, 1), (1, 128), (3, 129), (16, 512), (31, 130), (128, 64), (129, 511), (130, 520), (257, 96), (700, 1030)])
def test_quantize_both_axes(f8, M, C, square, dtype):
    x = _rand(np.random.default_rng(M * 1009 + C), (M, C), dtype, 3.0)
    v = _np(x)
    a, t = f8.quantize(x, square, True, True)
    _check_matrix(a, ref.f8_codes(v, square), M, C)
    _check_matrix(t, ref.f8_codes(v.T, square), C, M)
    only, none = f8.quantize(x, square)
    assert none is None and (only.values() == a.values()).all()
    _, only = f8.quantize(x, square, False, True)
    assert (only.values() == t.values()).all()
    np.testing.assert_array_equal(_np(a.values()), ref.f8_values(v, square))
    np.testing.assert_array_equal(_np(a.values(_dtype("bf16"))), ref.f8_values(v, square))


# more than 128 and 256 tiles of 128 x 128: one block for both axes
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("M,C", [(1500, 1540), (2060, 2100)])
def test_quantize_both_axes_of_many_tiles(f8, M, C, square, dtype):
    x = _rand(np.random.default_rng(M), (M, C), dtype, 3.0)
    v = _np(x)
    a, t = f8.quantize(x, square, True, True)
    _check_matrix(a, ref.f8_codes(v, square), M, C)
    _check_matrix(t, ref.f8_codes(v.T, square), C, M)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_padding_of_the_last_tile_is_zero(f8, dtype):
    # K up to a multiple of 128 is multiplied
    x = _rand(np.random.default_rng(0), (20, 150), dtype)
    a, t = f8.F8Matrix.empty(20, 150), f8.F8Matrix.empty(150, 20)
    for m in (a, t):
        m.codes.fill_(0x55)
    f8.sq_f8_quantize(x, False, a.codes, a.scales, t.codes, t.scales)
    for m, rows, cols in ((a, 20, 150), (t, 150, 20)):
        byte, _ = ref.f8_places(rows, -(-cols // 128) * 128)
        assert not m.codes.cpu().numpy()[byte][:, cols:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_rounding(f8, dtype):
    # halfway points of all elements, and their neighbours in the input's type, at several scales
    import torch
    mid = (ref.E4M3[1:] + ref.E4M3[:-1]) / 2
    v = np.concatenate([ref.E4M3, mid, [464.0, 2.0 ** -10 * 1.0001]])
    t = _cuda(v, dtype)
    bits = t.view(torch.int32 if dtype == "f32" else torch.int16)
    t = torch.cat([t, (bits + 1).view(t.dtype), (bits - 1).view(t.dtype)])
    t = t[(t <= 464) & (t >= 0)]
    rows = []
    for sign in (1, -1):
        for e in (0, -120, 100, 11):
            x = torch.zeros(-(-t.numel() // 127) * 127, dtype=t.dtype, device="cuda")
            x[:t.numel()] = t
            x = torch.cat([torch.full((x.numel() // 127, 1), 464.0, dtype=t.dtype, device="cuda"), x.view(-1, 127)], 1)
            rows.append(x * sign * 2.0 ** e)
    x = torch.cat(rows)
    v = _np(x)
    a, tr = f8.quantize(x.contiguous(), False, True, False)[0], f8.quantize(x.t().contiguous(), False, False, True)[1]
    for m in (a, tr):
        _check_matrix(m, ref.f8_codes(v), *v.shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("square", [False, True])
def test_extremes_and_nonfinite(f8, square, dtype):
    x = np.zeros((300, 260), np.float32)
    x[0, :3] = [464.0, 466.0, -464.0]
    x[1, :2] = [464.0, 1.0]
    x[3] = 2.0 ** -126
    x[4] = 2.0 ** -133                                   # subnormal in fp32 and bf16
    x[5] = 3.3895313892515355e38                         # bf16's largest
    x[6, 5], x[7, 140], x[8, 259] = np.inf, -np.inf, np.nan
    x[9] = -0.0
    x[10, 0], x[10, 1] = 2.0 ** 100, 2.0 ** -100
    x[130:] = np.random.default_rng(0).integers(-64, 65, (170, 260))
    t = _cuda(x, dtype)
    v = _np(t)
    a, tr = f8.quantize(t, square, True, True)
    with np.errstate(invalid="ignore"):
        _check_matrix(a, ref.f8_codes(v, square), 300, 260)
        _check_matrix(tr, ref.f8_codes(v.T, square), 260, 300)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift,pad", [(0, 1), (1, 0), (3, 5), (8, 8)])
def test_strided_and_misaligned(f8, dtype, shift, pad):
    M, C, N = 70, 200, 40
    rng = np.random.default_rng(5)
    x = _rand(rng, (M * (C + pad) + shift + C,), dtype)[shift:].as_strided((M, C), (C + pad, 1))
    v = _np(x)
    a, t = f8.quantize(x, False, True, True)
    _check_matrix(a, ref.f8_codes(v), M, C)
    _check_matrix(t, ref.f8_codes(v.T), C, M)
    w = _rand(rng, (N, C), dtype)
    wq = f8.quantize(w, True)[0]
    for rows in (1, 16, 70):        # one launch, and the quantizer and the product
        _close(f8.LinearPlan(rows, C, N, _dtype(dtype)).forward(x[:rows], wq), ref.f8_values(v[:rows]), ref.f8_values(_np(w), True), dtype)


PRODUCTS = [(1, 1, 1), (1, 16, 128), (3, 33, 129), (16, 100, 700), (17, 33, 65), (64, 64, 512), (100, 130, 1000), (129, 257, 300),
            (300, 700, 520), (1100, 2100, 260), (2000, 1900, 400), (3300, 3900, 200), (4096, 3200, 1152)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_products(f8, M, N, K, dtype):
    # every kind of tile, ragged on every side
    import torch
    rng = np.random.default_rng(M + N + K)
    x, w = _rand(rng, (M, K), dtype), _rand(rng, (N, K), dtype)
    a, b = f8.quantize(x)[0], f8.quantize(w, True)[0]
    va, vb = ref.f8_values(_np(x)), ref.f8_values(_np(w), True)
    need = f8.sq_f8_gemm_workspace_size(M, N, K)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    full = torch.full((M + 1, N + 3), 7.0, dtype=_dtype(dtype), device="cuda")
    C = full[:M, :N]
    f8.sq_f8_gemm(a.codes, a.scales, b.codes, b.scales, K, C, ws)
    _close(C, va, vb, dtype)
    assert (full[M:] == 7).all() and (full[:, N:] == 7).all()
    y = f8.LinearPlan(M, K, N, _dtype(dtype)).forward(x, b)
    _close(y, va, vb, dtype)


@pytest.mark.parametrize("M,N,K", [(5, 64, 512), (40, 64, 512), (300, 300, 4096), (1300, 1400, 700)])
def test_float32_results_keep_fp32_sums(f8, M, N, K):
    # products that span 2^26 in a piece of 16: 2^-24 a product and addition, where the 8-bit instructions cut at 2^-13
    rng = np.random.default_rng(K)
    x, w = (_cuda(rng.choice([-1, 1], s) * 2.0 ** rng.uniform(-9, 8.5, s), "f32") for s in ((M, K), (N, K)))
    y = f8.LinearPlan(M, K, N, _dtype("f32")).forward(x, f8.quantize(w, True)[0])
    a, b = ref.f8_values(_np(x)), ref.f8_values(_np(w), True)
    # a random walk of K roundings, 2^-24 sqrt(K) of the largest sums, 6 times over; 2^-13 would be 100 times as much
    assert np.linalg.norm(_np(y) - a @ b.T) <= 6 * 2.0 ** -24 * np.sqrt(K) * np.linalg.norm(a @ b.T)


# rows, columns, inner axis; sums exact in fp32: nothing of a long inner axis is lost, in any split
@pytest.mark.parametrize("M,N,K", [(1, 40, 20500), (16, 16, 5000), (17, 33, 8200), (70, 130, 11000), (128, 1024, 12288), (64, 640, 30000),
                                   (300, 300, 640), (1500, 1400, 2050), (3100, 4200, 1030), (257, 8193, 513)])
def test_products_are_exact_where_sums_are(f8, M, N, K):
    import torch
    rng = np.random.default_rng(K)
    x, w = ref.held(rng, M, K), ref.held(rng, N, K)
    want = torch.from_numpy(x).cuda().double() @ torch.from_numpy(w).cuda().double().T
    y = f8.LinearPlan(M, K, N, _dtype("f32")).forward(_cuda(x, "f32"), f8.quantize(_cuda(w, "f32"), True)[0])
    assert (y.double() == want).all()
    a, b = f8.quantize(_cuda(x, "bf16"))[0], f8.quantize(_cuda(w, "bf16"), True)[0]
    need = f8.sq_f8_gemm_workspace_size(M, N, K)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    C = torch.empty(M, N, device="cuda")
    f8.sq_f8_gemm(a.codes, a.scales, b.codes, b.scales, K, C, ws)
    assert (C.double() == want).all()


# where the codes' values pass below the normal numbers of fp32 and bf16
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("e", [-105, -116, -122, -140])
@pytest.mark.parametrize("M,N,K", [(5, 40, 700), (150, 270, 1400)])
def test_products_of_tiny_values(f8, M, N, K, e, dtype):
    import torch
    rng = np.random.default_rng(M)
    x, w = _cuda(np.ldexp(rng.standard_normal((M, K)), e), "f32"), _cuda(np.ldexp(rng.standard_normal((N, K)), 100), "f32")
    a, b = f8.quantize(x)[0], f8.quantize(w, True)[0]
    va, vb = ref.f8_values(_np(x)), ref.f8_values(_np(w), True)
    want, y = va @ vb.T, torch.empty(M, N, dtype=_dtype(dtype), device="cuda")
    need = f8.sq_f8_linear_workspace_size(M, K, N)
    f8.sq_f8_linear(x, b.codes, b.scales, y, torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
    tol = (np.abs(va) @ np.abs(vb).T) * (K + 2) * 2.0 ** -23
    if dtype == "bf16":
        tol = tol + 15 * 2.0 ** -13 * (_pieces(va) @ _pieces(vb).T) + 2.0 ** -8 * np.abs(want)
    else:       # operands in bf16, whose least step is 2^-133
        tol = tol + 2.0 ** -134 * np.abs(vb).sum(1)
    np.testing.assert_array_less(np.abs(_np(y) - want), tol + 2.0 ** -149)
    np.testing.assert_array_equal(a.values().double().cpu().numpy(), np.round(va * 2.0 ** 149) / 2.0 ** 149)


def test_scales_reach_every_block(f8):
    # each block of 128 with a scale of its own on both sides
    import torch
    M, N, K = 150, 270, 1400
    rng = np.random.default_rng(2)
    e = np.repeat(rng.integers(-3, 4, (M, -(-K // 128))), 128, 1)[:, :K]
    f = np.repeat(np.repeat(rng.integers(-3, 4, (-(-N // 128), -(-K // 128))), 128, 0)[:N], 128, 1)[:, :K]
    x, w = ref.held(rng, M, K) * 2.0 ** e, ref.held(rng, N, K) * 2.0 ** f
    want = torch.from_numpy(x).cuda() @ torch.from_numpy(w).cuda().T      # multiples of 2^-6 below 2^19: exact in fp64
    for rows in (M, 9):
        y = f8.LinearPlan(rows, K, N, _dtype("f32")).forward(_cuda(x[:rows], "f32"), f8.quantize(_cuda(w, "f32"), True)[0])
        mag = np.abs(x[:rows]) @ np.abs(w).T
        assert (np.abs(_np(y) - _np(want)[:rows]) <= mag * (K + 2) * 2.0 ** -23).all()


STEPS = [(1, 1, 1), (16, 64, 48), (100, 130, 70), (197, 768, 96), (300, 520, 1000), (3152, 768, 768), (1030, 2000, 2100), (2500, 300, 4100)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", STEPS)
def test_training_step(f8, M, K, N, dtype):
    rng = np.random.default_rng(M * 3 + K * 5 + N)
    x, w, dy = _rand(rng, (M, K), dtype), _rand(rng, (N, K), dtype), _rand(rng, (M, N), dtype)
    plan = f8.LinearPlan(M, K, N, _dtype(dtype), train=True)
    with pytest.raises(ValueError):
        plan.forward(x)
    plan.quantize_weight(w)
    with pytest.raises(ValueError):
        plan.backward(dy)
    y = plan.forward(x)
    dx, dw = plan.backward(dy)
    v, vw, vd = _np(x), ref.f8_values(_np(w), True), _np(dy)
    _close(y, ref.f8_values(v), vw, dtype)
    _close(dx, ref.f8_values(vd), vw.T, dtype)
    _close(dw, ref.f8_values(vd.T), ref.f8_values(v.T), "f32")


def test_gradients_are_differences_of_the_layer(f8):
    # d sum(dy y) of the products' values: Y is linear in X and W where these change by whole steps of their codes
    import torch
    rng = np.random.default_rng(1)
    M, K, N = 40, 150, 60
    x, w, dy = (ref.held(rng, *s).astype(np.float64) for s in ((M, K), (N, K), (M, N)))
    x[:, 0], w[:, 0] = 15, 15       # no change below moves a scale

    def loss(x, w):
        plan = f8.LinearPlan(M, K, N, _dtype("f32"), train=True)
        plan.quantize_weight(_cuda(w, "f32"))
        return float((plan.forward(_cuda(x, "f32")).double() * torch.from_numpy(dy).cuda()).sum()), plan
    base, plan = loss(x, w)
    dx, dw = (_np(t) for t in plan.backward(_cuda(dy, "f32")))
    for _ in range(6):
        i, j, k = int(rng.integers(M)), int(rng.integers(N)), int(rng.integers(1, K))
        up = x.copy()
        up[i, k] = -up[i, k]
        assert loss(up, w)[0] - base == dx[i, k] * -2 * x[i, k]
        up = w.copy()
        up[j, k] = -up[j, k]
        assert loss(x, up)[0] - base == dw[j, k] * -2 * w[j, k]


@pytest.mark.parametrize("M", [5, 300])
def test_nonfinite_values_reach_their_results_and_no_others(f8, M):
    import torch
    rng = np.random.default_rng(4)
    K, N = 400, 300
    x, w, dy = _rand(rng, (M, K), "bf16"), _rand(rng, (N, K), "bf16"), _rand(rng, (M, N), "bf16")
    x[2, 130], w[140, 300] = float("nan"), float("inf")
    y = f8.LinearPlan(M, K, N).forward(x, f8.quantize(w, True)[0])
    nan = y.isnan()
    assert nan[2].all() and nan[:, 128:256].all()       # the square block of W
    nan[2], nan[:, 128:256] = False, False
    assert not nan.any()
    plan = f8.LinearPlan(M, K, N, train=True)
    plan.quantize_weight(w)
    plan.forward(x)
    dx, dw = plan.backward(dy)
    assert dx[:, 256:384].isnan().all() and not dx[:, :256].isnan().any() and not dx[:, 384:].isnan().any()
    assert dw[:, 130].isnan().all() and not torch.cat([dw[:, :130], dw[:, 131:]], 1).isnan().any()


def test_empty_axes(f8):
    import torch
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = _rand(np.random.default_rng(0), (32, 64), "bf16")
    assert f8.LinearPlan(0, 64, 32).forward(x, f8.quantize(w, True)[0]).shape == (0, 32)
    plan = f8.LinearPlan(0, 64, 32, train=True)
    plan.quantize_weight(w)
    plan.forward(x)
    plan.dW.fill_(5)
    assert not plan.backward(torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"))[1].any()
    x, w = torch.empty(20, 0, device="cuda"), torch.empty(32, 0, device="cuda")
    for m in (20, 300):
        plan = f8.LinearPlan(m, 0, 32, torch.float32)
        plan.Y.fill_(5)
        assert not plan.forward(torch.empty(m, 0, device="cuda"), f8.quantize(w, True)[0]).any()


def test_operands_past_32_bit_elements(f8):
    # 2.2e9 elements of X: the last rows are those of a small call
    import torch
    M, K, N = 540000, 4096, 64
    w = f8.quantize(_rand(np.random.default_rng(1), (N, K), "bf16"), True)[0]
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    x[-40:] = _rand(np.random.default_rng(2), (40, K), "bf16")
    a = f8.quantize(x)[0]
    y = torch.empty(M, N, device="cuda")
    need = f8.sq_f8_gemm_workspace_size(M, N, K)
    f8.sq_f8_gemm(a.codes, a.scales, w.codes, w.scales, K, y, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
    b = f8.quantize(x[-40:])[0]
    small = torch.empty(40, N, device="cuda")
    need = f8.sq_f8_gemm_workspace_size(40, N, K)
    f8.sq_f8_gemm(b.codes, b.scales, w.codes, w.scales, K, small, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
    mag = b.values().double().abs() @ w.values().double().abs().T
    assert ((y[-40:].double() - small.double()).abs() <= 2 * mag * (K + 2) * 2.0 ** -23).all() and not y[:-40].any()


@pytest.mark.parametrize("M,K,N", [(1, 300, 200), (200, 300, 400), (64, 9000, 64)])
def test_other_stream_determinism_and_replays(f8, M, K, N):
    import torch
    rng = np.random.default_rng(M)
    x, w, dy = _rand(rng, (M, K), "bf16"), _rand(rng, (N, K), "bf16"), _rand(rng, (M, N), "bf16")

    def step(plan, serve):
        plan.quantize_weight(w)
        y = plan.forward(x)
        return (y, *plan.backward(dy), serve.forward(x, plan.w))
    plan, serve = f8.LinearPlan(M, K, N, train=True), f8.LinearPlan(M, K, N)
    want = [t.clone() for t in step(plan, serve)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [t.clone() for t in step(plan, serve)]
    s.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = step(plan, serve)
    for i in range(3):
        x.copy_(_rand(rng, (M, K), "bf16"))
        w.copy_(_rand(rng, (N, K), "bf16"))
        want = [t.clone() for t in step(f8.LinearPlan(M, K, N, train=True), f8.LinearPlan(M, K, N))]
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all((a == b).all() for a, b in zip(out, want)), i
