"""Microscaled 4-bit products over a long inner axis, with sums that are exact in
fp32 (tests/mx_exact.py): every output has to equal the sum in 64 bits, fp32 as
it is and bf16 rounded once."""
import pytest

from tests import mx_exact

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2411_10948_amd import mx, shiftquant
    shiftquant.load()
    return mx


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("M,N,K", mx_exact.LONG)
def test_gemm_of_a_long_inner_axis(mx, M, N, K, dtype):
    import torch
    a, b = (torch.from_numpy(v).cuda() for v in mx_exact.operands(M, N, K))
    ca, cb = mx.quantize(a)[0], mx.quantize(b)[0]
    need = mx.sq_mx_gemm_workspace_size(M, N, K)
    assert (need > 0) == (K >= 2 * 40 * 128)      # parts of 40 steps of 128 at least
    C = torch.full((M, N + 3), 7.0, dtype=getattr(torch, dtype), device="cuda")
    mx.sq_mx_gemm(ca.codes, ca.scales, cb.codes, cb.scales, K, C[:, :N], mx._workspace(need, "cuda"))
    mx_exact.equal(C[:, :N].contiguous(), a, b)
    assert (C[:, N:] == 7.0).all()
