"""Pins of the float64 definitions in oracle/routed.py: hand-worked values, torch's conversion to
e4m3, central differences."""
import numpy as np
import pytest
import torch

from oracle import routed as o


def test_e4m3_is_torchs():
    x = np.concatenate([np.linspace(-448, 448, 20001), o.e4m3_values(), -o.e4m3_values(),
                        (o.e4m3_values()[1:] + o.e4m3_values()[:-1]) / 2, [np.nan]]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = o.to_e4m3(x.astype(np.float64))
    nan = np.isnan(x)
    np.testing.assert_array_equal(got[~nan], want[~nan])
    assert (got[nan] & 127 == 127).all()
    codes = np.arange(256, dtype=np.uint8)
    np.testing.assert_array_equal(o.from_e4m3(codes), torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy())


def test_scale_exponents():
    for amax, e in ((448, 0), (448.001, 1), (224, -1), (224.001, 0), (1, -8), (1.75, -8), (1.7500001, -7), (0, 0),
                    (2.0 ** -149, -127), (2.0 ** 127, 119)):
        assert o.scale_exponent(amax) == e, amax


def test_router_by_hand():
    l = np.log(np.array([[0.5, 0.25, 0.2, 0.8]]) / (1 - np.array([[0.5, 0.25, 0.2, 0.8]])))
    e, w = o.route_groups(l, 2)
    assert e.tolist() == [[3, 0]] and np.allclose(w, [[0.8 / 1.3, 0.5 / 1.3]])
    # the bias moves the choice, not the weights
    e, w = o.route_groups(l, 2, bias=[0, 0.6, 0, 0], normalise=False, scale=2)
    assert e.tolist() == [[1, 3]] and np.allclose(w, [[0.5, 1.6]])
    # groups (0, 1) and (2, 3): by the best expert the second, by the two best the second too; with a
    # bias on expert 1 the first by two
    assert o.route_groups(l, 1, groups=2)[0].tolist() == [[3]]
    assert o.route_groups(l, 1, groups=2, group_top=2, bias=[0, 0.3, 0, 0])[0].tolist() == [[1]]
    # an unavailable group leaves slots empty
    l[0, 2:] = -np.inf
    e, w = o.route_groups(l, 4, groups=2, group_k=2)
    assert e.tolist() == [[0, 1, -1, -1]] and np.allclose(w[0], [2 / 3, 1 / 3, 0, 0])
    assert o.route_groups(np.full((1, 4), -np.inf), 2, score="softmax")[0].tolist() == [[-1, -1]]


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("normalise", [True, False])
def test_router_gradient_by_differences(score, normalise):
    rng = np.random.default_rng(3)
    l, dw = rng.normal(size=(3, 7)), rng.normal(size=(3, 3))
    l[1, 2] = -np.inf
    kw = dict(score=score, normalise=normalise, scale=1.7)
    expert, _ = o.route_groups(l, 3, **kw)
    d = o.route_groups_backward(l, expert, dw, **kw)
    for t in range(3):
        for e in range(7):
            if l[t, e] == -np.inf:
                assert d[t, e] == 0
                continue
            f = []
            for by in (1e-6, -1e-6):
                x = l.copy()
                x[t, e] += by
                got = o.route_groups(x, 3, **kw)
                assert (got[0] == expert).all()
                f.append((got[1] * dw).sum())
            assert abs(d[t, e] - (f[0] - f[1]) / 2e-6) < 1e-8


def test_quotients_of_small_sigmoids():
    w = o.route_groups(np.array([[-2000.0, -2001.0]]), 2)[1]
    assert np.allclose(w, [[1 / (1 + np.exp(-1)), 1 / (1 + np.e)]], rtol=1e-12)


def test_columns_take_whole_blocks():
    x = np.arange(1.0, 7.0).reshape(3, 2)
    q, e = o.quant_columns(x, [0, 2, 2, 3])
    assert q.shape == (2, 256) and e.shape == (2, 2)
    np.testing.assert_array_equal(o.held(q, e)[:, [0, 1, 128]], x.T)
    assert not q[:, 2:128].any()


def test_adamw_is_torchs():
    rng = np.random.default_rng(5)
    p, g = torch.tensor(rng.normal(size=50)), torch.tensor(rng.normal(size=50))
    ref = p.clone().requires_grad_()
    opt = torch.optim.AdamW([ref], lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    q, m, v = p.numpy(), np.zeros(50), np.zeros(50)
    for t in range(1, 4):
        ref.grad = g * t
        opt.step()
        q, m, v = o.adamw(q, g.numpy() * t, m, v, t, lr=1e-2, beta1=0.8, beta2=0.95, eps=1e-6, weight_decay=0.1)
    np.testing.assert_allclose(q, ref.detach().numpy(), rtol=1e-12)


def test_drawn_rounding_keeps_values_on_average():
    bits = np.arange(0, 65536, 16)
    for x in (300.0, 17.3, 2.0 ** -7, 1.9 * 2.0 ** -9):
        got, _ = o.drawn(np.full(bits.size, x), bits, 0, False)
        assert np.isin(got, o.e4m3_values()).all() and abs(got.mean() / x - 1) < 1e-3
    assert (o.drawn(np.full(bits.size, 2.0 ** -12), bits, 0, True)[0] == 2.0 ** -9).all()


def test_noise_bits_are_even():
    for t in (1, 2):
        for bits in o.noise(np.arange(1 << 16), t, 7):
            assert abs(bits.mean() / 32767.5 - 1) < 0.02  # five standard deviations are 0.011
    a, b = o.noise(np.arange(1000), 1, 7)[0], o.noise(np.arange(1000), 2, 7)[0]
    assert (a != b).mean() > 0.99
    assert o.mix(0) == 0 and int(o.mix(1)) == 0x514e28b7  # MurmurHash3's published finaliser
