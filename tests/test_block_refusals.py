"""Refusals of layer norm, router and exchange (no GPU: every call is refused, or
has nothing to do, before a launch; no pointer is read)."""
import ctypes as ct
import os

import pytest

INVALID, UNSUPPORTED, SMALL = 1, 3, 4
P, ODD = ct.c_void_p(0x100000), ct.c_void_p(0x100001)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    from paper_2411_10948_amd import shiftquant
    if not os.path.exists(shiftquant.LIB_PATH):
        from paper_2411_10948_amd import build
        build.build()
    return shiftquant.load()


def _call(f, names, defaults, **given):
    assert set(given) <= set(names)
    return f(*[given.get(n, d) for n, d in zip(names, defaults)])


def _size(f, *args):
    n = ct.c_size_t(0)
    return f(*args, ct.byref(n)), n.value


def test_norm_forward(L):
    names = "x res type M C ld_x ld_r gamma beta ptype eps h ld_h y ld_y stats stream".split()
    ok = [P, None, 1, 4, 64, 64, 64, P, P, 0, 1e-5, None, 64, P, 64, P, None]

    def f(**k):
        return _call(L.sq_norm_forward, names, ok, **k)
    for bad in (dict(x=None), dict(y=None), dict(gamma=None), dict(beta=None), dict(type=2), dict(ptype=-1), dict(M=-1),
                dict(M=1 << 31), dict(C=1 << 20), dict(ld_x=63), dict(ld_y=63), dict(x=ODD), dict(gamma=ODD), dict(eps=-1e-5),
                dict(eps=NAN), dict(eps=INF), dict(res=P), dict(h=P), dict(res=P, h=P, ld_r=63), dict(res=P, h=P, ld_h=63),
                dict(stats=ct.c_void_p(0x100004))):
        assert f(**bad) == INVALID, bad
    assert f(M=0, x=None, y=None) == 0 and f(C=0, x=None, y=None, gamma=None, beta=None) == 0


def test_norm_backward(L):
    status, need = _size(L.sq_norm_backward_workspace_size, 4, 64)
    assert status == 0 and need >= 2 * 64 * 4
    assert _size(L.sq_norm_backward_workspace_size, -1, 64)[0] == INVALID
    assert _size(L.sq_norm_backward_workspace_size, 4, 1 << 20)[0] == INVALID
    assert L.sq_norm_backward_workspace_size(4, 64, None) == INVALID
    # never more than the rows of a thread block each
    assert _size(L.sq_norm_backward_workspace_size, 1 << 30, 4096)[1] <= 1 << 26
    names = "dy h dh type M C ld_dy ld_h ld_dh gamma ptype stats dx ld_dx dgamma dbeta ws nws stream".split()
    ok = [P, P, None, 1, 4, 64, 64, 64, 64, P, 0, P, P, 64, P, P, P, need, None]

    def f(**k):
        return _call(L.sq_norm_backward, names, ok, **k)
    for bad in (dict(dy=None), dict(h=None), dict(dx=None), dict(stats=None), dict(stats=ct.c_void_p(0x100008)), dict(dgamma=None),
                dict(dbeta=ODD), dict(gamma=None), dict(type=3), dict(ld_dy=63), dict(ld_h=1), dict(ld_dx=63),
                dict(dh=P, ld_dh=63), dict(ws=None), dict(ws=ct.c_void_p(0x100008)), dict(C=1 << 20)):
        assert f(**bad) == INVALID, bad
    assert f(nws=2 * 64 * 4 - 1, M=1) == SMALL
    assert f(C=0, gamma=None, dgamma=None, dbeta=None) == 0


def test_router(L):
    names = "l type T E ld bias score k groups top renorm scale share chosen place off ws nws stream".split()
    ok = [P, 0, 100, 64, 64, None, 0, 8, 1, 1, 0, 1.0, P, P, P, P, P, 1 << 30, None]

    def f(**k):
        return _call(L.sq_route_forward, names, ok, **k)
    for bad in (dict(l=None), dict(l=ODD), dict(type=7), dict(T=-1), dict(E=0), dict(k=0), dict(k=65), dict(ld=63), dict(bias=ODD),
                dict(score=2), dict(renorm=2), dict(groups=0), dict(groups=7), dict(groups=8, top=0), dict(groups=8, top=9),
                dict(groups=16, top=1), dict(scale=NAN), dict(scale=INF), dict(share=None), dict(chosen=ODD), dict(place=None),
                dict(off=None), dict(ws=None), dict(ws=ct.c_void_p(0x100008))):
        assert f(**bad) == INVALID, bad
    assert f(E=1025, ld=1025) == f(E=512, ld=512, k=65) == f(E=1000, ld=1000, groups=100, top=100) == UNSUPPORTED
    assert f(T=1 << 26) == f(T=(1 << 31) - 1) == f(T=1 << 25, k=64) == UNSUPPORTED
    status, need = _size(L.sq_route_workspace_size, 100, 64)
    assert status == 0 and need > 0 and f(nws=need - 1) == SMALL
    assert _size(L.sq_route_workspace_size, 64, 64) == (0, 0)       # one launch
    assert _size(L.sq_route_workspace_size, 64, 0)[0] == _size(L.sq_route_workspace_size, 64, 1025)[0] == INVALID
    assert _size(L.sq_route_workspace_size, 1 << 26, 64)[0] == UNSUPPORTED
    assert _size(L.sq_route_workspace_size, (1 << 26) - 3, 64)[0] == UNSUPPORTED       # a launch of 2^32 threads
    assert _size(L.sq_route_workspace_size, (1 << 26) - 4, 64)[0] == 0

    names = "d l type T E ld score k renorm scale share chosen dl ld_d stream".split()
    ok = [P, P, 0, 100, 64, 64, 0, 8, 0, 1.0, P, P, P, 64, None]

    def g(**k):
        return _call(L.sq_route_backward, names, ok, **k)
    for bad in (dict(d=None), dict(l=None), dict(share=ODD), dict(chosen=None), dict(dl=None), dict(ld_d=63), dict(ld=63),
                dict(score=-1), dict(renorm=-1), dict(k=0), dict(k=65), dict(scale=NAN), dict(type=2)):
        assert g(**bad) == INVALID, bad
    assert g(T=1 << 26) == UNSUPPORTED and g(T=0, d=None, l=None, dl=None) == 0


def test_exchange(L):
    d = [P, 0, 10, 64, 64, P, 2, P, 20, 64, None]
    for i, bad in ((0, None), (1, 2), (2, -1), (2, 1 << 31), (3, 1 << 20), (4, 63), (5, None), (5, ODD), (6, 0), (7, None), (8, -1),
                   (8, 1 << 31), (9, 63)):
        assert L.sq_exchange_dispatch(*d[:i], bad, *d[i + 1:]) == INVALID, (i, bad)
    assert L.sq_exchange_dispatch(*d[:6], 65, *d[7:]) == L.sq_exchange_dispatch(*d[:2], 1 << 30, *d[3:]) == UNSUPPORTED
    assert L.sq_exchange_dispatch(*d[:2], 0, *d[3:]) == L.sq_exchange_dispatch(*d[:8], 0, *d[9:]) == 0
    c = [P, 0, 20, 64, 64, P, P, 10, 2, None, 64, P, 64, None]
    for i, bad in ((0, None), (1, -1), (2, -1), (3, -1), (4, 63), (5, None), (6, ODD), (7, -1), (8, 0), (11, None), (12, 63)):
        assert L.sq_exchange_combine(*c[:i], bad, *c[i + 1:]) == INVALID, (i, bad)
    assert L.sq_exchange_combine(*c[:9], P, 63, *c[11:]) == INVALID         # add and its row stride
    assert L.sq_exchange_combine(*c[:7], 0, *c[8:]) == 0
    b = [P, P, 0, 20, 64, 64, 64, P, P, 10, 2, P, 64, P, None]
    for i, bad in ((0, None), (1, None), (2, 2), (3, -1), (4, 1 << 20), (5, 63), (6, 63), (7, ODD), (8, None), (9, -1), (10, 0),
                   (11, None), (12, 63), (13, None)):
        assert L.sq_exchange_combine_backward(*b[:i], bad, *b[i + 1:]) == INVALID, (i, bad)
    assert L.sq_exchange_combine_backward(*b[:9], 0, *b[10:]) == 0


def test_plans():
    import torch
    from paper_2411_10948_amd import norm, route
    kw = dict(device="cpu")     # buffers alone: no call reaches a launch
    for bad in (dict(score="tanh"), dict(groups=3), dict(groups=0), dict(groups=4, top_groups=5), dict(groups=8, top_groups=1, k=3)):
        with pytest.raises(ValueError):
            route.RouterPlan(4, 16, **{"k": 2, **bad}, **kw)
    with pytest.raises(TypeError):
        route.RouterPlan(4, 16, 2, dtype=torch.float16, **kw)
    for bad in ((4, 0, 8), (4, 65, 8), (-1, 2, 8), (4, 2, 1 << 20)):
        with pytest.raises(ValueError):
            route.ExchangePlan(*bad, **kw)
    with pytest.raises(TypeError):
        norm.NormPlan(4, 8, param_dtype=torch.float16, **kw)
    plan, x, g = norm.NormPlan(4, 8, residual=True, **kw), torch.zeros(4, 8, dtype=torch.bfloat16), torch.ones(8)
    with pytest.raises(ValueError, match="residual"):
        plan.forward(x, g, g)
    with pytest.raises(ValueError, match="x: expected a tensor on the plan's GPU"):
        plan.forward(x, g, g, x)
    with pytest.raises(ValueError, match="train"):
        plan.backward(x, x, g)
    with pytest.raises(ValueError, match="train"):
        route.ExchangePlan(4, 2, 8, **kw).dispatch_backward(x, g)
    with pytest.raises(ValueError, match="forward"):
        route.RouterPlan(4, 8, 2, **kw).backward(torch.zeros(4, 2), x)
