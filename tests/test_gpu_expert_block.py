"""The block of experts that puts layer norm, router, exchange, the products by
expert in 4 bits and the dense ones in 8 together: its stages against the plain
implementations in 64 bits, its gradients through the norm against differences, a
captured training step, and the example that trains and serves one."""
import numpy as np
import pytest

from tests import block_reference as block
from tests import f8_reference as f8_ref
from tests import mx_reference as mx_ref

pytestmark = pytest.mark.gpu
U = block.U


@pytest.fixture(scope="module")
def block_cls():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2411_10948_amd import experts, shiftquant
    shiftquant.load()
    return experts.ExpertBlock


def _np(t):
    return t.detach().double().cpu().numpy()


def _near(got, want, mag, terms):
    """An fp32 sum of `terms` products, `mag` the sum of their magnitudes."""
    assert (np.abs(got - want) <= mag * (terms + 2) * 2.0 ** -23 + 1e-30).all()


def _weights(r, dim, hidden, E, shared, dtype):
    import torch
    w = [1 + 0.2 * r(dim), 0.1 * r(dim), r(E, dim) / dim ** 0.5, r(E, 2 * hidden, dim).to(dtype), r(E, dim, hidden).to(dtype)]
    w += [r(2 * shared, dim).to(dtype), r(dim, shared).to(dtype)] if shared else [None, None]
    return w + [0.05 * r(E)]


RULE = dict(score="sigmoid", groups=2, top_groups=1, renormalize=True, scale=2.5)


@pytest.mark.parametrize("tokens,dim,hidden,E,k,shared", [(1, 64, 32, 4, 2, 48), (40, 96, 64, 6, 2, 0), (200, 128, 100, 8, 3, 70)])
def test_stages(block_cls, tokens, dim, hidden, E, k, shared):
    # each stage from the stage before as the GPU computed it
    import torch
    g = torch.Generator(device="cuda").manual_seed(tokens)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    layer = block_cls(tokens, dim, hidden, E, k, shared, dtype=torch.float32, **RULE)
    w = _weights(r, dim, hidden, E, shared, torch.float32)
    gamma, beta, router, w1, w2, s1, s2, bias = w
    layer.set_weights(*w)
    x, res, dout, dh = r(tokens, dim), r(tokens, dim), r(tokens, dim), r(tokens, dim)
    out, h = layer.forward(x, res)
    assert (h == x + res).all()
    y, logits, share, place, z = (_np(t) for t in layer._saved)
    gu, a = _np(layer.up.Y), _np(layer.act.H)
    grads = {n: _np(t) for n, t in layer.backward(dout, dh).items()}
    want, xh, _ = block.norm(_np(h), _np(gamma), _np(beta), 1e-5)
    assert np.abs(y - want).max() <= 100 * U * (1 + np.abs(xh).max()) * (1 + np.abs(want).max())
    _near(logits, *mx_ref.mx_product(y, _np(router)), dim)
    ws, wc, wp, wo = block.route(logits, k, "sigmoid", _np(bias), 2, 1, True, 2.5)
    assert (layer.router.chosen.cpu().numpy() == wc).all() and (place == wp).all()
    assert (np.abs(share - ws) <= 32 * U * ws).all() and (layer.router.offsets.cpu().numpy() == wo).all()
    place, rows = place.astype(int), block.dispatch(y, wp, np.zeros((tokens * k, dim)))
    dz, dshare, mag = block.combine_backward(_np(dout), z, place, share, np.zeros_like(z))
    assert (np.abs(_np(layer.exchange.dR) - dz) <= 2 * U * np.abs(dz)).all()
    dz, v = _np(layer.exchange.dR), mx_ref.mx_values
    da, dgu, drows = _np(layer.down.dX), _np(layer.act.dX), _np(layer.up.dX)
    for e, (lo, hi) in enumerate(mx_ref.segments(wo.tolist())):
        s = slice(lo, hi)
        if hi == lo:
            assert not grads["w1"][e].any() and not grads["w2"][e].any()
            continue
        _near(gu[s], *mx_ref.mx_product(v(rows[s]), v(_np(w1[e]))), dim)
        _near(z[s], *mx_ref.mx_product(v(a[s]), v(_np(w2[e]))), hidden)
        _near(da[s], *mx_ref.mx_product(v(dz[s]), v(_np(w2[e]).T)), dim)
        _near(drows[s], *mx_ref.mx_product(v(dgu[s]), v(_np(w1[e]).T)), 2 * hidden)
        _near(grads["w2"][e], *mx_ref.mx_product(v(dz[s].T), v(a[s].T)), hi - lo)
        _near(grads["w1"][e], *mx_ref.mx_product(v(dgu[s].T), v(rows[s].T)), hi - lo)
    dlogits, lmag = block.route_backward(logits, wc, _np(layer.exchange.dshare), "sigmoid", True, 2.5)
    assert (np.abs(_np(layer.router.dlogits) - dlogits) <= 64 * U * lmag + 1e-30).all()
    dlogits = _np(layer.router.dlogits)
    _near(grads["router"], *mx_ref.mx_product(dlogits.T, y.T), tokens)
    dy, dmag = mx_ref.mx_product(dlogits, _np(router).T)
    dense = 0.0
    if shared:
        q, sq = f8_ref.f8_values, lambda m: f8_ref.f8_values(m, True)
        sgu, sa, dense = _np(layer.shared_up.Y), _np(layer.shared_act.H), _np(layer.shared_down.Y)
        dsgu, ds = _np(layer.shared_act.dX), _np(layer.shared_up.dX)
        _near(sgu, *mx_ref.mx_product(q(y), sq(_np(s1))), dim)
        _near(dense, *mx_ref.mx_product(q(sa), sq(_np(s2))), shared)
        _near(ds, *mx_ref.mx_product(q(dsgu), sq(_np(s1)).T), 2 * shared)
        _near(grads["s2"], *mx_ref.mx_product(q(_np(dout).T), q(sa.T)), tokens)
        _near(grads["s1"], *mx_ref.mx_product(q(dsgu.T), q(y.T)), tokens)
        dy, dmag = dy + ds, dmag + np.abs(ds)
    total, tmag = block.combine(z, place, share, dense)
    assert (np.abs(_np(out) - total) <= (k + 2) * U * tmag + 1e-30).all()
    back, bmag = block.combine(drows, place, None, dy)
    assert (np.abs(_np(layer.exchange.dX) - back) <= (dim + k + 4) * 2.0 ** -23 * (bmag + dmag)).all()
    wx, wg, wb = block.norm_backward(_np(h), _np(gamma), 1e-5, _np(layer.exchange.dX), _np(dh))
    scale = np.abs(_np(layer.exchange.dX)).max() * (1 + np.abs(xh).max()) ** 2 * (1 + np.abs(_np(gamma)).max())
    assert np.abs(grads["x"] - wx).max() <= 400 * U * scale * np.abs(block.norm(_np(h), 1, 0, 1e-5)[2]).max() + U * np.abs(_np(dh)).max()
    for name, want in (("gamma", wg), ("beta", wb)):
        assert np.abs(grads[name] - want).max() <= (100 + tokens / 64) * U * tokens * scale


def test_router_gradient_against_differences(block_cls):
    # with the experts' outputs and y held, d sum(dout out) / d router in 64 bits
    import torch
    g = torch.Generator(device="cuda").manual_seed(7)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    T, D, H, E, k = 24, 64, 32, 4, 2
    layer = block_cls(T, D, H, E, k, dtype=torch.float32, score="sigmoid", scale=2.5)
    w = _weights(r, D, H, E, 0, torch.float32)
    layer.set_weights(*w)
    dout = r(T, D)
    layer.forward(r(T, D), r(T, D))
    y, _, _, place, z = (_np(t) for t in layer._saved)
    chosen = layer.router.chosen.cpu().numpy()
    got = _np(layer.backward(dout)["router"])

    def loss(router):
        share = block.shares(y @ router.T, chosen, "sigmoid", True, 2.5)
        return (block.combine(z, place.astype(int), share)[0] * _np(dout)).sum()
    router, eps = _np(w[2]), 1e-5
    rng = np.random.default_rng(0)
    for _ in range(12):
        at = int(rng.integers(E)), int(rng.integers(D))
        up, down = router.copy(), router.copy()
        up[at] += eps
        down[at] -= eps
        diff = (loss(up) - loss(down)) / (2 * eps)
        # fp32 terms of the gradient 1e-5 of its size at most, the difference's rounding 1e-16 / eps of the loss
        assert abs(got[at] - diff) <= 1e-4 * (np.abs(got).max() + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_training_step_in_a_graph(block_cls, dtype):
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    T, D, H, E, k, S = 150, 128, 96, 8, 2, 64
    w = _weights(r, D, H, E, S, dt)
    x, res, dout = r(T, D).to(dt), r(T, D).to(dt), r(T, D).to(dt)
    make = lambda: block_cls(T, D, H, E, k, S, dtype=dt, **RULE)

    def step(layer):
        layer.set_weights(*w)
        out, h = layer.forward(x, res)
        grads = layer.backward(dout, h)
        return [out, h] + [grads[n] for n in sorted(grads)]
    mine = make()
    step(mine)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):      # torch's matrix products set themselves up outside of the graph
        step(mine)
    s.synchronize()
    with torch.cuda.graph(graph, stream=s):
        out = step(mine)
    for i in range(3):
        x.copy_(r(T, D))
        w[3].copy_(r(*w[3].shape))
        if i == 1:
            w[2][3] += 2.0          # another split of the rows
        want = [t.clone() for t in step(make())]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), i


def test_serving_gives_what_training_gives(block_cls):
    import torch
    g = torch.Generator(device="cuda").manual_seed(6)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    w = _weights(r, 128, 96, 8, 64, torch.bfloat16)
    x, res = r(300, 128).bfloat16(), r(300, 128).bfloat16()
    train, serve = block_cls(300, 128, 96, 8, 2, 64, **RULE), block_cls(300, 128, 96, 8, 2, 64, train=False, **RULE)
    for layer in (train, serve):
        layer.set_weights(*w)
    a, b = train.forward(x, res), serve.forward(x, res)
    # the same codes; sums of the experts' few rows are made in another order: an fp32 rounding may move one to bf16
    assert (a[1] == b[1]).all() and (a[0].float() - b[0].float()).abs().max() <= 2.0 ** -7 * a[0].float().abs().max()
    with pytest.raises(ValueError):
        serve.backward(x)


def test_example_trains_and_serves():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "expert_block.py")
    spec = importlib.util.spec_from_file_location("expert_block", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    losses, grads, far = mod.run(steps=5, tokens=96, dim=128, hidden=64, experts=4, shared=64, log=lambda *a, **k: None)
    assert len(losses) == 5 and all(np.isfinite(losses))
    for name, t in grads.items():
        assert t.isfinite().all() and t.any(), name
    # a token alone takes other sums and the same codes but where a bf16 rounding falls the other way
    assert far < 0.05
