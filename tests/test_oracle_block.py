"""The float64 definitions of the operators around the layer, pinned by hand-worked values,
identities and central differences."""
import math

import numpy as np
import pytest

from oracle import block


def _rand(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


def test_norm_forward_by_hand():
    X, Y = np.array([[1.0, -2.0]]), np.array([[3.0, 4.0]])
    (Xo, _), (N, _) = block.norm_forward(X, Y, pre=True, post=True, w_pre=np.array([2.0, 1.0]),
                                         gate_c=np.array([1.0, 0.5]), gate_t=np.array([2.0]), res_scale=0.5, eps=0.0)
    r = 1 / math.sqrt(12.5)
    want = np.array([0.5 + 2 * 3 * r, -1.0 + 2 * 0.5 * 4 * r])
    np.testing.assert_allclose(Xo[0], want, rtol=1e-14)
    np.testing.assert_allclose(N[0], want / math.sqrt((want ** 2).mean()) * [2.0, 1.0], rtol=1e-14)
    (Xo, _), none = block.norm_forward(X, None, pre=False, post=False, res_scale=3.0)
    assert none is None
    np.testing.assert_array_equal(Xo, 3 * X)


@pytest.mark.parametrize("pre,post", [(True, True), (True, False), (False, True)])
def test_norm_gradient_is_that_of_the_forward(pre, post):
    T, d = 3, 7
    a = dict(X=_rand(1, T, d), Y=_rand(2, T, d), w_pre=_rand(3, d) if pre else None,
             w_post=_rand(4, d) if post else None, gate_c=_rand(5, d), gate_t=_rand(6, T))
    dX_out, dN = _rand(7, T, d), _rand(8, T, d)
    kw = dict(pre=pre, post=post, res_scale=0.7, eps=1e-3)

    def f(v):
        (Xo, _), n = block.norm_forward(v["X"], v["Y"], w_pre=v["w_pre"], w_post=v["w_post"], gate_c=v["gate_c"],
                                        gate_t=v["gate_t"], **kw)
        return (dX_out * Xo).sum() + ((dN * n[0]).sum() if pre else 0.0)

    (Xo, _), _ = block.norm_forward(a["X"], a["Y"], w_pre=a["w_pre"], w_post=a["w_post"], gate_c=a["gate_c"],
                                    gate_t=a["gate_t"], **kw)
    g = block.norm_backward(Xo, a["Y"], dX_out, dN if pre else None, w_pre=a["w_pre"], w_post=a["w_post"],
                            gate_c=a["gate_c"], gate_t=a["gate_t"], **kw)
    h = 1e-5
    for name, v in a.items():
        if v is None:
            continue
        got = g["d" + name][0]
        assert (np.abs(got) <= g["d" + name][1] * (1 + 1e-12)).all()
        for i in np.ndindex(v.shape):
            up, down = dict(a), dict(a)
            up[name], down[name] = v.copy(), v.copy()
            up[name][i] += h
            down[name][i] -= h
            assert abs((f(up) - f(down)) / (2 * h) - got[i]) < 1e-7, (name, i)


def test_route_choice_ties_and_masks():
    inf = math.inf
    l = np.array([[1.0, 3.0, 3.0, -inf], [-inf, -inf, -inf, -inf], [0.0, -0.0, math.nan, -5.0], [-inf, 2.0, -inf, math.nan]])
    e, w = block.route_forward(l, 2)
    np.testing.assert_array_equal(e, [[1, 2], [-1, -1], [0, 1], [1, -1]])
    np.testing.assert_allclose(w, [[0.5, 0.5], [0, 0], [0.5, 0.5], [1, 0]])
    e, w = block.route_forward(l, 2, normalise=False, scale=2.0)
    np.testing.assert_allclose(w[0, 0], 2 / (2 + math.exp(-2)), rtol=1e-14)


@pytest.mark.parametrize("normalise", [True, False])
def test_route_gradient_is_that_of_the_forward(normalise):
    l = _rand(11, 4, 6)
    l[1, 2] = -math.inf
    l[2] = -math.inf
    l[3, 1:] = math.nan
    dw = _rand(12, 4, 3)
    e, _ = block.route_forward(l, 3, normalise, 1.5)
    g, sc = block.route_backward(l, e, dw, normalise, 1.5)
    h = 1e-6
    for i in np.ndindex(l.shape):
        if not np.isfinite(l[i]):
            assert g[i] == 0
            continue
        up, down = l.copy(), l.copy()
        up[i] += h
        down[i] -= h
        (eu, wu), (ed, wd) = block.route_forward(up, 3, normalise, 1.5), block.route_forward(down, 3, normalise, 1.5)
        assert (eu == e).all() and (ed == e).all()
        assert abs(((wu - wd) * dw).sum() / (2 * h) - g[i]) < 1e-8
        assert abs(g[i]) <= sc[i] * (1 + 1e-12)


def test_expert_order_is_a_stable_sort():
    expert = np.array([[2, 0], [0, -1], [2, 1], [9, 0]], dtype=np.int32)
    pos, offsets = block.expert_order(expert, 4)
    np.testing.assert_array_equal(offsets, [0, 3, 4, 6, 6])
    np.testing.assert_array_equal(pos, [[4, 0], [1, -1], [5, 3], [-1, 2]])


def test_combine_and_its_gradient():
    expert = np.array([[1, 0], [-1, -1], [0, 1]], dtype=np.int32)
    pos, _ = block.expert_order(expert, 2)
    Ys, w, dY = _rand(21, 4, 3), _rand(22, 3, 2), _rand(23, 3, 3)
    Y, _ = block.expert_combine(Ys, pos, w)
    np.testing.assert_array_equal(Y[1], 0)
    np.testing.assert_allclose(Y[0], w[0, 0] * Ys[2] + w[0, 1] * Ys[0], rtol=1e-14)
    dYs, (dw, _) = block.expert_combine_backward(dY, Ys, pos, w)
    # linear in each: the gradients reproduce the inner product with any change
    for seed in (1, 2):
        E, v = _rand(30 + seed, 4, 3), _rand(40 + seed, 3, 2)
        np.testing.assert_allclose((block.expert_combine(E, pos, w)[0] * dY).sum(), (dYs * E).sum(), rtol=1e-12)
        np.testing.assert_allclose((block.expert_combine(Ys, pos, v)[0] * dY).sum(), (dw * v).sum(), rtol=1e-12)


def test_clip():
    norm, g = block.clip([np.array([3.0]), np.array([[0.0, -4.0]])], 1.0)
    assert norm == 5.0
    np.testing.assert_allclose(g[1], [[0.0, -0.8]])
    assert block.clip([np.array([3.0])], 3.0)[1][0][0] == 3.0
    assert math.isnan(block.clip([np.array([math.nan, 1.0])], 1.0)[0])
    assert block.clip([np.array([math.inf, 2.0])], 1.0)[1][0][1] == 2.0
