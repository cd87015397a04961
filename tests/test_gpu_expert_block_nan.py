"""A token of the block of experts whose logits hold NaN shows it in its output and
gradients, with a shared MLP and without, and leaves the others alone."""
import pytest

pytestmark = pytest.mark.gpu


def _layer(shared, dtype, train=True, T=20, **rule):
    import torch
    from paper_2411_10948_amd import experts
    D, H, E, k = 64, 32, 4, 2
    g = torch.Generator(device="cuda").manual_seed(shared)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    w = [1 + 0.2 * r(D), 0.1 * r(D), r(E, D) / 8, r(E, 2 * H, D).to(dtype), r(E, D, H).to(dtype)]
    w += [r(2 * shared, D).to(dtype), r(D, shared).to(dtype)] if shared else [None, None]
    layer = experts.ExpertBlock(T, D, H, E, k, shared, dtype=dtype, train=train, **rule)
    layer.set_weights(*w)
    return layer, w, r(T, D).to(dtype), r(T, D).to(dtype), r(T, D).to(dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shared", [0, 48])
@pytest.mark.parametrize("rule", [dict(), dict(score="sigmoid", scale=2.5)])
def test_a_row_with_nan(shared, dtype, rule):
    import torch
    layer, _, x, res, dout = _layer(shared, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype], **rule)
    clean = layer.forward(x, res)[0].clone()
    assert clean.isfinite().all()
    x[3, 5], x[11, 0] = float("nan"), float("inf")
    out, h = layer.forward(x, res)
    rest = [t for t in range(20) if t not in (3, 11)]
    assert out[[3, 11]].isnan().all() and out[rest].isfinite().all() and h[3, 5].isnan() and h[rest].isfinite().all()
    dx = layer.backward(dout)["x"]
    assert dx[[3, 11]].isnan().all() and dx[rest].isfinite().all()
    x[3, 5] = x[11, 0] = 0.0        # nothing of it stays
    assert layer.forward(x, res)[0].isfinite().all()


@pytest.mark.parametrize("shared", [0, 48])
@pytest.mark.parametrize("train", [True, False])
def test_a_router_that_is_nan(shared, train):
    import torch
    layer, w, x, res, _ = _layer(shared, torch.bfloat16, train)
    w[2][1, 7] = float("nan")       # kept, not copied
    assert layer.forward(x, res)[0].isnan().all()


@pytest.mark.parametrize("shared", [0, 48])
def test_one_token(shared):
    import torch
    layer, _, x, res, _ = _layer(shared, torch.bfloat16, False, 1)
    assert layer.forward(x, res)[0].isfinite().all()
    x[0, 63] = float("nan")
    assert layer.forward(x, res)[0].isnan().all()
