"""The branches of the microscaled 4-bit calls by size, each pinned by its
workspace: few rows in one launch, quantizer and product, split sums, both
gradients in one launch.  Sums are exact in fp32 (tests/mx_exact.py), so outputs
have to equal those in 64 bits."""
import numpy as np
import pytest

from tests import mx_exact

pytestmark = pytest.mark.gpu
DTYPES = ["float32", "bfloat16"]


@pytest.fixture(scope="module")
def mx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2411_10948_amd import mx, shiftquant
    shiftquant.load()
    return mx


def _held(seed, *shape, dtype):
    import torch
    return torch.from_numpy(mx_exact.held(np.random.default_rng(seed), *shape)).cuda().to(getattr(torch, dtype))


def _experts(off):
    return enumerate(zip(off[:-1], off[1:]))


def _offsets(off):
    import torch
    return torch.tensor(off, dtype=torch.int32, device="cuda")


def _bytes(n):
    return -(-n // 256) * 256


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N,parts", [(4096, 512, 512, 1), (4096, 260, 517, 1), (1100, 1041, 1300, 1), (3000, 3000, 2100, 1),
                                         (2600, 1537, 2070, 1), (8300, 65, 8200, 1), (40000, 1, 70, 1), (128, 12288, 1024, 2),
                                         (130, 15500, 1000, 3), (250, 20481, 650, 4)])
def test_linear_by_quantizer_and_product(mx, M, K, N, parts, dtype):
    import torch
    assert mx.sq_mx_gemm_workspace_size(M, N, K) == (_bytes(parts * M * N * 4) if parts > 1 else 0)
    plan = mx.LinearPlan(M, K, N, dtype=getattr(torch, dtype))
    assert plan.ws.numel() == sum(map(_bytes, mx.sq_mx_size(M, K))) + mx.sq_mx_gemm_workspace_size(M, N, K)
    plan.Y.fill_(float("nan"))
    x, w = _held(M, M, K, dtype=dtype), _held(N, N, K, dtype=dtype)
    mx_exact.equal(plan.forward(x, mx.quantize(w)[0]), x, w)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_columns_by_quantizer_and_product(mx, dtype):
    import torch
    plan = mx.LinearPlan(40000, 0, 70, dtype=getattr(torch, dtype))
    plan.Y.fill_(3.0)
    w = mx.quantize(torch.ones(70, 0, device="cuda"))[0]
    assert not plan.forward(torch.ones(40000, 0, dtype=getattr(torch, dtype), device="cuda"), w).any()


# one launch for few rows, 64 columns a block (512 blocks of 16 and more) or 16, a wave's part of the inner axis from
# one tile to sixteen
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", [(1, 4096, 11008), (3, 2077, 9000), (16, 8200, 8197), (7, 15361, 8300), (1, 16384, 500),
                                   (40, 4099, 200), (300, 600, 130)])
def test_linear_of_few_rows(mx, M, K, N, dtype):
    import torch
    plan = mx.LinearPlan(M, K, N, dtype=getattr(torch, dtype))
    plan.Y.fill_(float("nan"))
    x, w = _held(M, M, K, dtype=dtype), _held(N, N, K, dtype=dtype)
    c = mx.quantize(w)[0]
    y = plan.forward(x, c)
    # this call needs no workspace (the plan's has room for the other type's call)
    from paper_2411_10948_amd.shiftquant import load
    bare = torch.full_like(y, float("nan"))
    assert load().sq_mx_linear(x.data_ptr(), mx._TYPES[x.dtype], M, K, K, None, 0, c.codes.data_ptr(), c.scales.data_ptr(), N,
                               bare.data_ptr(), mx._TYPES[x.dtype], N, None, 0, mx._stream(None)) == 0
    mx_exact.equal(y, x, w)
    assert torch.equal(y, bare)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N,off", [
    (8, 2048, 1024, list(range(8)) + [8] * 57),                     # one row on each of 8 of 64 experts
    (64, 4500, 1030, [0] * 20 + [3, 3, 20] + [40] * 10 + [64]),     # few rows, several tiles of the inner axis a wave
    (30, 2077, 650, [0, 30, 30]),
    (5000, 700, 900, [0, 13, 13, 2100, 4990, 5000]),                # quantizer and product
    (3000, 2050, 1040, [7, 900, 901, 2990]),
    (16384, 300, 1400, list(range(0, 16384, 256)) + [16384]),
    (9000, 1600, 4099, [0, 4000, 9000])])
def test_experts_serving(mx, M, K, N, off, dtype):
    import torch
    E = len(off) - 1
    plan = mx.LinearPlan(M, K, N, dtype=getattr(torch, dtype), experts=E)
    assert (plan.ws is None) == (M <= 64)
    plan.Y.fill_(7.0)
    x, w = _held(M, M, K, dtype=dtype), _held(N, E, N, K, dtype=dtype)
    y = plan.forward(x, mx.quantize(w)[0], _offsets(off))
    for e, (lo, hi) in _experts(off):
        mx_exact.equal(y[lo:hi], x[lo:hi], w[e])
    assert (y[:off[0]] == 7.0).all() and (y[off[-1]:] == 7.0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N,off", [
    (16384, 1024, 1024, None),      # both gradients in one launch of large tiles, one of them split
    (14000, 65, 70, None), (300, 30000, 33, None), (3000, 768, 700, None), (5000, 2048, 2600, None), (20, 40, 50, None),
    (6000, 1100, 900, [0, 11, 11, 4000, 5980, 6000]), (1200, 130, 520, [3, 40, 600, 601, 1150]),
    (9000, 2048, 1500, [0, 8000, 9000]), (40, 64, 96, [0, 40])])
def test_training_step(mx, M, K, N, off, dtype):
    import torch
    E = len(off) - 1 if off else 0
    plan = mx.LinearPlan(M, K, N, dtype=getattr(torch, dtype), experts=E, train=True)
    plan.Y.fill_(7.0)
    plan.dX.fill_(7.0)
    plan.dW.fill_(float("nan"))
    x, dy = _held(M, M, K, dtype=dtype), _held(M + 1, M, N, dtype=dtype)
    w = _held(N, *((E, N, K) if E else (N, K)), dtype=dtype)
    plan.quantize_weight(w)
    y = plan.forward(x, offsets=_offsets(off) if E else None)
    dx, dw = plan.backward(dy)
    for e, (lo, hi) in _experts(off or [0, M]):
        we, dwe = (w[e], dw[e]) if E else (w, dw)
        mx_exact.equal(y[lo:hi], x[lo:hi], we)
        mx_exact.equal(dx[lo:hi], dy[lo:hi], we.t())
        mx_exact.equal(dwe, dy[lo:hi].t(), x[lo:hi].t())
    if E:
        for t in (y, dx):
            assert (t[:off[0]] == 7.0).all() and (t[off[-1]:] == 7.0).all()


def test_the_split_gradient_shares_a_launch(mx):
    # 2 parts of dW, no split of dX or of Y: what the first size of test_training_step is there for
    assert mx.sq_mx_gemm_workspace_size(1024, 1024, 16384) == _bytes(2 * 1024 * 1024 * 4)
    assert mx.sq_mx_gemm_workspace_size(16384, 1024, 1024) == 0
    plan = mx.LinearPlan(16384, 1024, 1024, train=True)
    assert plan.ws.numel() == _bytes(2 * 1024 * 1024 * 4)


# ---------------------------------------------------------------------------
# NaN and Inf, in every branch: the row of A and the column of B that hold one, and nothing else
def _spoil(x, places):
    for at, v in places:
        x[at] = v
    return x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", [(4096, 512, 512), (2600, 1537, 2070), (128, 12288, 1024), (3, 2077, 9000)])
def test_nan_in_linear(mx, M, K, N, dtype):
    import torch
    x = _spoil(_held(0, M, K, dtype=dtype), [((M // 2, K - 1), float("inf")), ((0, 0), float("nan"))])
    w = _spoil(_held(1, N, K, dtype=dtype), [((N - 1, K // 2), float("nan")), ((7, 3), -float("inf"))])
    got = mx.LinearPlan(M, K, N, dtype=getattr(torch, dtype)).forward(x, mx.quantize(w)[0])
    want = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    want[[0, M // 2]] = True
    want[:, [7, N - 1]] = True
    assert torch.equal(got.isnan(), want)


@pytest.mark.parametrize("M,K,N,off", [(2000, 520, 700, [0, 700, 701, 2000]), (64, 2100, 650, [0, 20, 21, 64])])
def test_nan_in_serving_by_expert(mx, M, K, N, off):
    import torch
    x = _spoil(_held(0, M, K, dtype="bfloat16"), [((off[1] - 1, 5), float("nan"))])
    w = _spoil(_held(1, 3, N, K, dtype="bfloat16"), [((2, 9, K - 1), float("inf"))])
    got = mx.LinearPlan(M, K, N, experts=3).forward(x, mx.quantize(w)[0], _offsets(off))
    want = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    want[off[1] - 1] = True
    want[off[2]:, 9] = True
    assert torch.equal(got.isnan(), want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N,off", [(14000, 65, 70, None), (700, 300, 200, None), (4096, 1024, 2048, None),
                                       (1200, 130, 520, [0, 40, 600, 1200]), (5000, 1100, 900, [0, 0, 4000, 5000])])
def test_nan_in_a_training_step(mx, M, K, N, off, dtype):
    import torch
    E = len(off) - 1 if off else 0
    plan = mx.LinearPlan(M, K, N, dtype=getattr(torch, dtype), experts=E, train=True)
    r, c, n = M - 3, K - 1, N // 2          # in the last expert
    x = _spoil(_held(0, M, K, dtype=dtype), [((r, c), float("nan"))])
    dy = _spoil(_held(1, M, N, dtype=dtype), [((r - 1, n), float("inf"))])
    w = _held(2, *((E, N, K) if E else (N, K)), dtype=dtype)
    plan.quantize_weight(w)
    y = plan.forward(x, offsets=_offsets(off) if E else None)
    dx, dw = plan.backward(dy)
    want = [torch.zeros(t.shape, dtype=torch.bool, device="cuda") for t in (y, dx, dw)]
    want[0][r] = True                       # the block of X's row
    want[1][r - 1] = True                   # of dY's row
    last = want[2][-1] if E else want[2]
    last[:, c] = True                       # of X's and of dY's column
    last[n] = True
    for got, bad in zip((y, dx, dw), want):
        assert torch.equal(got.isnan(), bad)
    # a NaN weight: the column of Y for its row, of dX for its column
    w.view(-1, N, K)[-1, 2, 1] = float("nan")
    x, dy = _held(0, M, K, dtype=dtype), _held(1, M, N, dtype=dtype)
    plan.quantize_weight(w)
    y = plan.forward(x, offsets=_offsets(off) if E else None)
    dx, dw = plan.backward(dy)
    first = off[-2] if E else 0
    want = [torch.zeros(t.shape, dtype=torch.bool, device="cuda") for t in (y, dx)]
    want[0][first:, 2] = True
    want[1][first:, 1] = True
    assert torch.equal(y.isnan(), want[0]) and torch.equal(dx.isnan(), want[1]) and not dw.isnan().any()
