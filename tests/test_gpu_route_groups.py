"""The router with groups against its float64 definition: choices exactly, weights and gradients
within what fp32 roundings add up to."""
import numpy as np
import pytest
import torch

from block_util import DT, Out, assert_rounded, f32, same_bits, shifted, stored
from oracle import routed as o
from paper_2603_23198_amd import binding as b

pytestmark = pytest.mark.gpu

# E, k, groups, group_k, group_top
LAYOUTS = [(1, 1, 1, 1, 1), (7, 3, 1, 1, 1), (8, 8, 2, 2, 2), (60, 6, 6, 3, 2), (64, 8, 8, 4, 2), (64, 8, 64, 64, 1),
           (65, 5, 5, 2, 2), (128, 1, 1, 1, 2), (160, 8, 8, 3, 1), (256, 8, 8, 4, 2), (256, 64, 4, 1, 2), (255, 9, 3, 2, 2),
           (257, 2, 1, 1, 1), (512, 8, 16, 2, 2), (1000, 10, 100, 7, 2), (1024, 64, 32, 4, 1), (1024, 8, 512, 200, 2)]


def logits_of(rng, T, E, masked):
    l = rng.normal(size=(T, E)) * 2
    if masked:
        l[rng.random((T, E)) < 0.3] = -np.inf
        l[rng.random((T, E)) < 0.02] = np.nan
        l[T // 2] = -np.inf
        l[T // 3] = np.nan
        if T > 4:
            l[4] = -np.inf
            l[4, E - 1] = 0.5
    return l


def both(l, dt, k, bias=None, normalise=True, score="sigmoid", scale=1.0, dweight=None, by=0, **kw):
    """(outputs, expected) of forward and backward; by: the alignment of every buffer, in elements."""
    (L, held), (B, bv), T = stored(l, dt), f32(bias), l.shape[0]
    expert, weight = Out((T, k), torch.int32, by), Out((T, k), torch.float32, by)
    same = dict(score=score, normalise=normalise, scale=scale)
    L = shifted(L, by)
    b.sfl_route_groups_forward(L, expert.t, weight.t, bias=shifted(B, by), **same, **kw)
    want = o.route_groups(held, k, bias=bv, **same, **kw)
    got = (expert.values(), weight.values())
    if dweight is None:
        return got, want
    D, dv = f32(dweight)
    d = Out(l.shape, DT[dt], by)
    b.sfl_route_groups_backward(L, expert.t, shifted(D, by), d.t, **same)
    return got + (d.values(),), want + (o.route_groups_backward(held, want[0], dv, **same), held, dv)


def check(got, want, k, scale, dt="f32", normalise=True):
    np.testing.assert_array_equal(got[0], want[0])
    # exp, the sum's k + 1 terms, a quotient and the scale: each term's error is relative to it, of
    # library functions of at most two units (their argument's rounding is relative to the logits, which
    # are below 16: 16 half units)
    terms = 2 * (16 + 4) + want[0].shape[1] + 6
    assert_rounded(got[1], want[1], np.abs(want[1]), "f32", terms, "weight")
    if len(got) > 2:
        held, dw = want[3], want[4]
        G = scale * np.abs(np.where(want[0] >= 0, dw, 0)).sum(1, keepdims=True)
        # every term is at most |G| in all, scores and shares are at most 1
        assert_rounded(got[2], want[2], np.broadcast_to(G, want[2].shape), dt, terms + held.shape[1], "dlogits")


@pytest.mark.parametrize("E,k,groups,group_k,group_top", LAYOUTS)
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_layouts(E, k, groups, group_k, group_top, score):
    rng = np.random.default_rng(E + k)
    for dt, masked, normalise, T in (("f32", False, True, 9), ("bf16", True, False, 33), ("f32", True, True, 70)):
        bias = rng.normal(size=E) * (0.3 if score == "sigmoid" else 0.3 / E)
        got, want = both(logits_of(rng, T, E, masked), dt, k, bias, normalise, score, 2.5, rng.normal(size=(T, k)),
                         groups=groups, group_k=group_k, group_top=group_top)
        check(got, want, k, 2.5, dt)


@pytest.mark.parametrize("T", [1, 2, 3, 63, 1025])
def test_tokens_and_alignments(T):
    rng = np.random.default_rng(T)
    for by in (0, 1, 3):
        got, want = both(rng.normal(size=(T, 30)), "bf16", 4, rng.normal(size=30) * 0.1, by=by,
                         dweight=rng.normal(size=(T, 4)), groups=5, group_k=2, group_top=2)
        check(got, want, 4, 1.0, "bf16")


def test_no_tokens():
    e = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    b.sfl_route_groups_forward(torch.empty((0, 8), device="cuda"), e, torch.empty((0, 2), device="cuda"))


def test_equal_scores_go_by_index():
    """Equal logits, logits of one sigmoid in fp32 (all above 17 are 1), equal worths, +0 and -0."""
    l = np.zeros((5, 12))
    l[1] = np.linspace(20, 60, 12)[::-1]
    l[2] = [1, 0, 0, 1, 0, 0, 1, 0, 0, 1, 0, 0]
    l[3] = -1e30  # scores of zero
    l[4] = np.where(np.arange(12) % 2, 0.0, -0.0)
    for score in ("sigmoid", "softmax"):
        for kw in (dict(), dict(groups=4, group_k=2, group_top=2)):
            got, want = both(l, "f32", 4, score=score, **kw)
            np.testing.assert_array_equal(got[0], want[0])
    assert both(l, "f32", 4)[0][0][1].tolist() == [0, 1, 2, 3]
    bias = np.zeros(12)
    bias[[5, 7]] = -0.0, 0.0
    assert both(l[4:], "f32", 3, bias)[0][0].tolist() == [[0, 1, 2]]


def test_scores_that_fp32_cannot_tell_apart():
    """The choice is that of scores in 64 bits, rounded once: pairs of logits whose sigmoids lie within
    few last places of one another, with a bias that moves them to where fp32 rounds coarsely."""
    rng = np.random.default_rng(11)
    base = rng.normal(size=(400, 1)) * 2
    l = (base + rng.integers(-3, 4, size=(400, 32)) * 2.0 ** -22).astype(np.float32).astype(np.float64)
    bias = rng.integers(0, 2, size=32) * 2.0 ** -24
    for score in ("sigmoid", "softmax"):
        got, want = both(l, "f32", 8, bias, score=score)
        np.testing.assert_array_equal(got[0], want[0])
        got, want = both(l, "f32", 8, bias, score=score, groups=4, group_k=2, group_top=2)
        np.testing.assert_array_equal(got[0], want[0])


def test_infinite_logits_and_biases():
    inf, nan = np.inf, np.nan
    l = np.array([[0.0, inf, 1.0, inf], [inf, inf, inf, inf], [-inf, nan, inf, 0.0]])
    for score in ("sigmoid", "softmax"):
        for normalise in (True, False):
            got, want = both(l, "f32", 3, None, normalise, score, dweight=np.ones((3, 3)))
            check(got, want, 3, 1.0)
    bias = np.array([0.0, -inf, nan, inf])
    got, want = both(np.zeros((1, 4)), "f32", 4, bias)
    np.testing.assert_array_equal(got[0], [[3, 0, -1, -1]])
    check(got, want, 4, 1.0)


def test_quotients_of_scores_that_underflow():
    l = np.array([[-200.0, -201.0, -300.0, -1e30], [-1e30, -1e30, -2e30, -3e30], [90.0, 100.0, -200.0, 0.0]])
    got, want = both(l, "f32", 3, dweight=np.array([[1.0, 2.0, 3.0]] * 3))
    np.testing.assert_array_equal(got[0], want[0])
    # exp of arguments up to 300: 300 half units of it
    assert_rounded(got[1], want[1], want[1], "f32", 700, "weight")
    assert_rounded(got[2], want[2], np.full((3, 4), 6.0), "f32", 700, "dlogits")


def test_repeats_and_graphs():
    """The same bits again, also from a captured call on changed logits."""
    T, E, k = 200, 64, 8
    kw = dict(score="sigmoid", scale=2.5)
    L = torch.randn((T, E), device="cuda")
    bias, dw = torch.randn(E, device="cuda") * 0.1, torch.randn((T, k), device="cuda")
    outs = [torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda"), torch.empty_like(L)]

    def call():
        b.sfl_route_groups_forward(L, outs[0], outs[1], bias=bias, groups=8, group_k=4, group_top=2, **kw)
        b.sfl_route_groups_backward(L, outs[0], dw, outs[2], **kw)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(3):
        L.copy_(torch.randn((T, E), device="cuda"))
        call()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(same_bits(a, w) for a, w in zip(outs, want))


LOWEST = -float(np.finfo(np.float32).max)


@pytest.mark.parametrize("E,groups", [(60, 6), (10, 5), (64, 8), (256, 8), (12, 3)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_groups_whose_worth_is_below_every_number(E, groups, score):
    """Biases of the lowest number switch experts off until no others are left. The sum of two of them is -inf:
    a group of such is the last that is taken, but before a group without any expert, whatever their places."""
    size = E // groups
    l = np.random.default_rng(E).normal(size=(5, E))
    l[1, :size] = -np.inf  # a group without any, before the others and behind them
    l[2, -size:] = np.nan
    l[3, size:2 * size] = -np.inf
    l[4, 1:] = -np.inf
    kept = np.arange(E) >= E - size // 2 - 1  # some experts of the last group
    for bias in (np.full(E, LOWEST), np.where(kept, 0.0, LOWEST), np.where(np.arange(E) % size, LOWEST, -3e38)):
        for group_k in (1, groups - 1, groups):
            k = min(8, group_k * size)
            for top in (1, 2):
                got, want = both(l, "f32", k, bias, score=score, groups=groups, group_k=group_k, group_top=top)
                check(got, want, k, 1.0)


def test_experts_switched_off_by_the_lowest_bias_are_still_there():
    bias = np.full(60, LOWEST)
    got, _ = both(np.zeros((1, 60)), "f32", 8, bias, groups=6, group_k=6, group_top=2)
    assert got[0].tolist() == [list(range(8))]
