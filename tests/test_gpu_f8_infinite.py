"""Products of 8-bit values past fp32's range, which are Inf: few rows give what the
quantizer and the product give, whatever tiles of the inner axis a wave has."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [100, 128, 384, 1000, 1024, 1152, 1280, 4224])
@pytest.mark.parametrize("M", [1, 5, 40])
@pytest.mark.parametrize("types", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
def test_few_rows(types, M, K):
    import torch
    from paper_2411_10948_amd import f8
    dt, out = ({"bf16": torch.bfloat16, "f32": torch.float32}[t] for t in types)
    N, g = 48, torch.Generator(device="cuda").manual_seed(K)
    x = (1 + torch.rand(M, K, generator=g, device="cuda")).to(dt)
    w = torch.randn(N, K, generator=g, device="cuda")
    last = (K - 1) // 128 * 128
    w[3, last:] = 3.4e38            # 2^128 in 8 bits
    w[20, :K % 128 or 128] = -3.4e38
    codes = f8.quantize(w, square=True)[0]
    a = f8.quantize(x)[0]
    want, got = torch.empty(M, N, dtype=out, device="cuda"), torch.empty(M, N, dtype=out, device="cuda")
    ws = torch.empty(max(16, f8.sq_f8_gemm_workspace_size(M, N, K)), dtype=torch.uint8, device="cuda")
    f8.sq_f8_gemm(a.codes, a.scales, codes.codes, codes.scales, K, want, ws)
    ws = torch.empty(max(16, f8.sq_f8_linear_workspace_size(M, K, N)), dtype=torch.uint8, device="cuda")
    f8.sq_f8_linear(x, codes.codes, codes.scales, got, ws)
    assert (want[:, 3] == float("inf")).all() and (want[:, 20] == -float("inf")).all()
    assert (got[:, 3] == float("inf")).all() and (got[:, 20] == -float("inf")).all()
    # the others: weights in the same block of 128 x 128 are zeros in 8 bits next to 3.4e38, sums of the rest in another order
    rest = [i for i in range(N) if i not in (3, 20)]
    assert got[:, rest].isfinite().all() and want[:, rest].isfinite().all()
