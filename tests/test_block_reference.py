"""The plain forms of layer norm, router and exchange (tests/block_reference.py):
gradients against differences, and hand-made choices."""
import numpy as np
import pytest

from tests import block_reference as ref

rng = np.random.default_rng(0)


def _difference(f, x, at, eps=1e-6):
    up, down = x.copy(), x.copy()
    up[at] += eps
    down[at] -= eps
    return (f(up) - f(down)) / (2 * eps)


def test_norm_gradients_are_differences():
    h, g, b, dy = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    dx, dg, db = ref.norm_backward(h, g, 1e-5, dy)
    for i in range(7):
        assert abs(dx[1, i] - _difference(lambda v: (ref.norm(v, g, b, 1e-5)[0] * dy).sum(), h, (1, i))) < 1e-7
        assert abs(dg[i] - _difference(lambda v: (ref.norm(h, v, b, 1e-5)[0] * dy).sum(), g, i)) < 1e-7
        assert abs(db[i] - _difference(lambda v: (ref.norm(h, g, v, 1e-5)[0] * dy).sum(), b, i)) < 1e-7


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_router_gradients_are_differences(score, renorm):
    l, d = rng.standard_normal((2, 6)), rng.standard_normal((2, 3))
    l[1, 2] = -np.inf
    chosen = ref.route(l, 3, score)[1]
    grad, _ = ref.route_backward(l, chosen, d, score, renorm, 2.5)
    for t in range(2):
        for e in range(6):
            if l[t, e] > -np.inf:
                diff = _difference(lambda v: (ref.shares(v, chosen, score, renorm, 2.5) * d).sum(), l, (t, e))
                assert abs(grad[t, e] - diff) < 1e-8
    assert grad[1, 2] == 0


def test_exchange_gradients_are_differences():
    x, share, dout = rng.standard_normal((4, 5)), rng.standard_normal((4, 2)), rng.standard_normal((4, 5))
    y, place = rng.standard_normal((8, 5)), rng.permutation(8).reshape(4, 2)
    place[2, 1] = -1
    dy, dshare, _ = ref.combine_backward(dout, y, place, share, np.zeros((8, 5)))
    f = lambda y, s: (ref.combine(y, place, s)[0] * dout).sum()
    for i in range(8):
        assert abs(dy[i, 3] - _difference(lambda v: f(v, share), y, (i, 3))) < 1e-8
    for at in np.ndindex(4, 2):
        assert abs(dshare[at] - _difference(lambda v: f(y, v), share, at)) < 1e-8
    dx = ref.combine(y, place, None)[0]
    for i in range(4):
        assert abs(dx[i, 2] - _difference(lambda v: (ref.dispatch(v, place, np.zeros((8, 5))) * np.where(
            np.isin(np.arange(8), place)[:, None], y, 0.0)).sum(), x, (i, 2))) < 1e-8


def test_choices_by_hand():
    inf = np.inf
    l = np.array([[1.0, 3.0, 3.0, 2.0], [-inf, 0.0, -inf, -inf], [-inf] * 4, [0.0, np.nan, 1.0, 2.0]])
    share, chosen, place, offsets = ref.route(l, 2)
    assert chosen.tolist() == [[1, 2], [1, -1], [-1, -1], [-1, -1]]
    assert place.tolist() == [[0, 2], [1, -1], [-1, -1], [-1, -1]] and offsets.tolist() == [0, 0, 2, 3, 3]
    assert share[1].tolist() == [1.0, 0.0] and (share[2] == 0).all() and np.isnan(share[3]).all()
    # two groups: {0, 1} has the highest expert, {2, 3} the higher sum of two
    l = np.array([[5.0, -9.0, 4.0, 3.0]])
    assert ref.route(l, 2, "sigmoid", groups=2, top_groups=1)[1].tolist() == [[2, 3]]
    assert ref.route(l, 2, "sigmoid", bias=np.array([0.0, 2.0, 0.0, 0.0]), groups=2, top_groups=1)[1].tolist() == [[1, 0]]
