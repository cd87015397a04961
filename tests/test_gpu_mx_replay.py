"""Captured steps of the microscaled 4-bit layers: every replay takes the inputs,
weights and offsets that its buffers then hold."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2411_10948_amd import mx, shiftquant
    shiftquant.load()
    return mx


def _inputs(seed, M, K, N, E):
    """(x, dy, w, offsets or None)"""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: (torch.randn(*s, generator=g, device="cuda") * (1 + seed)).bfloat16()  # noqa: E731
    o = None
    if E:       # another split every time, experts without rows and rows without experts among them
        cut = torch.randint(0, M + 1, (E + 1,), generator=g, device="cuda").sort().values
        if seed % 2:
            cut[0], cut[-1] = 0, M
        if seed == 3:
            cut[:] = M // 3
        o = cut.to(torch.int32)
    return r(M, K), r(M, N), r(*((E, N, K) if E else (N, K))), o


@pytest.mark.parametrize("M,K,N,E,train", [
    (1, 512, 256, 0, False), (4096, 512, 512, 0, False), (128, 12288, 1024, 0, False),     # few rows; two launches; three
    (30, 700, 650, 6, False), (2000, 520, 700, 3, False),
    (600, 300, 64, 0, True), (14000, 65, 70, 0, True), (700, 200, 100, 5, True), (5000, 1100, 900, 4, True)])
def test_replays_follow_their_inputs(mx, M, K, N, E, train):
    import torch
    held = _inputs(0, M, K, N, E)
    x, dy, w, o = held
    plan, eager = (mx.LinearPlan(M, K, N, experts=E, train=train) for _ in range(2))
    codes = None if train else mx.quantize(w)[0]

    def step(plan, x, dy, w, o, codes):
        if not train:
            return (plan.forward(x, codes, o),)
        plan.quantize_weight(w)
        y = plan.forward(x, offsets=o)
        return (y, *plan.backward(dy))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(plan, *held, codes)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = step(plan, *held, codes)
    for seed in (1, 2, 3, 4, 1):
        new = _inputs(seed, M, K, N, E)
        for a, b in zip(held, new):
            if a is not None:
                a.copy_(b)
        if not train:
            fresh = mx.quantize(new[2])[0]
            codes.codes.copy_(fresh.codes)
            codes.scales.copy_(fresh.scales)
        for t in out:
            t.fill_(7.0)
        want = step(eager, *new, None if train else fresh)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        rows = slice(int(new[3][0]), int(new[3][-1])) if E else slice(0, M)
        for i, (a, b) in enumerate(zip(out, want)):
            assert torch.equal(a[rows], b[rows]) if i < 2 else torch.equal(a, b)
            if i < 2:
                assert (a[:rows.start] == 7.0).all() and (a[rows.stop:] == 7.0).all()
