"""The router on the GPU against the float64 definition: choices exactly, weights and gradients
within a few fp32 roundings (an exp of a difference of logits below 64 in magnitude carries at
most 64 units of rounding of its argument, sums of E terms E / 16 + 16 more)."""
import math

import numpy as np
import pytest
import torch

from oracle import block
from tests.block_util import DT, Out, assert_rounded, f32, same_bits, shifted, stored

pytestmark = pytest.mark.gpu

b = pytest.importorskip("paper_2603_23198_amd.binding")

SIZES = [(1, 1, 1), (7, 2, 2), (33, 5, 3), (64, 8, 2), (64, 8, 8), (5, 16, 1), (130, 60, 6), (257, 64, 8), (3, 64, 64),
         (9, 65, 64), (40, 128, 8), (31, 160, 6), (17, 200, 33), (20, 256, 8), (6, 512, 10), (4, 1000, 7), (5, 1024, 64)]


def make(T, E, dt, seed, kind):
    r = np.random.default_rng(seed)
    l = 1.5 * r.standard_normal((T, E))
    if kind == "ties":
        l = np.round(l * 2) / 2 * r.choice([1.0, -1.0, 0.0, -0.0], size=(T, E))
    if kind == "masked":
        l[r.uniform(size=(T, E)) < 0.4] = -math.inf
        l[r.uniform(size=(T, E)) < 0.05] = math.nan
        l[::3] = np.where(r.uniform(size=l[::3].shape) < 0.9, -math.inf, l[::3])
        l[T // 2] = -math.inf
    return stored(l, dt)


def check(T, E, k, dt, kind, normalise, scale, seed=0, by=0):
    logits, val = make(T, E, dt, seed, kind)
    if by:
        logits = shifted(logits, by)
    expert, weight = Out((T, k), torch.int32, by), Out((T, k), torch.float32, by)
    kw = dict(normalise=normalise, scale=scale)
    b.sfl_route_forward(logits, expert.t, weight.t, **kw)
    we, ww = block.route_forward(val, k, normalise, scale)
    np.testing.assert_array_equal(expert.values(), we)
    terms = 64 + E / 16 + 16
    assert_rounded(weight.values(), ww, np.abs(ww), "f32", terms, "weight")
    dwt, dw = f32(np.where(we < 0, math.nan, np.random.default_rng(seed + 1).standard_normal((T, k))))
    dl = Out((T, E), DT[dt], by)
    b.sfl_route_backward(logits, expert.t, shifted(dwt, by) if by else dwt, dl.t, **kw)
    want, sc = block.route_backward(val, we, np.nan_to_num(dw), normalise, scale)
    assert_rounded(dl.values(), want, sc, dt, 3 * terms, "dlogits")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,k", SIZES)
def test_route(T, E, k, dt):
    check(T, E, k, dt, "plain", True, 1.0, seed=T + E)
    check(T, E, k, dt, "ties", False, 2.5, seed=T + E)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,k", [(33, 5, 3), (64, 8, 8), (130, 60, 6), (65, 64, 8), (31, 160, 6), (12, 1024, 40)])
def test_masked_experts_and_empty_rows(T, E, k, dt):
    for normalise in (True, False):
        check(T, E, k, dt, "masked", normalise, 1.0, seed=E)


def test_element_alignment():
    for by in (1, 3):
        check(21, 64, 8, "bf16", "plain", False, 1.0, by=by)
        check(21, 37, 5, "f32", "masked", True, 1.0, by=by)


def test_infinite_and_extreme_logits():
    inf = math.inf
    l = torch.tensor([[inf, 1.0, 2.0, -inf], [3e38, -3e38, 1e38, 0.0], [-3e38, -3.1e38, -inf, -inf], [1.0, 2.0, 3.0, 4.0]],
                     device="cuda")
    e, w = torch.empty((4, 2), dtype=torch.int32, device="cuda"), torch.empty((4, 2), device="cuda")
    for normalise in (True, False):
        b.sfl_route_forward(l, e, w, normalise=normalise)
        np.testing.assert_array_equal(e.cpu().numpy(), [[0, 2], [0, 2], [0, 1], [3, 2]])
        assert w[0].isnan().all()
        np.testing.assert_array_equal(w[1:3].cpu().numpy(), [[1, 0], [1, 0]])
        assert w[3].isfinite().all()


def test_long_batch_matches_its_parts():
    T, E, k = 40003, 64, 8
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    l = torch.randn((T, E), generator=g, device="cuda")
    dw = torch.randn((T, k), generator=g, device="cuda")
    e, w, dl = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda"), torch.empty_like(l)
    b.sfl_route_forward(l, e, w)
    b.sfl_route_backward(l, e, dw, dl)
    for a, z in ((0, 7), (20000, 20001), (39990, T)):
        pe, pw, pdl = e[a:z].clone(), w[a:z].clone(), dl[a:z].clone()
        b.sfl_route_forward(l[a:z], pe, pw)
        b.sfl_route_backward(l[a:z], pe, dw[a:z], pdl)
        assert torch.equal(pe, e[a:z]) and same_bits(pw, w[a:z]) and same_bits(pdl, dl[a:z])
    top = l.topk(k, dim=1)
    assert torch.equal(top.indices.int(), e)


@pytest.mark.parametrize("normalise", [True, False])
def test_gradient_against_differences(normalise):
    """fp32 gradient against central differences (h = 1e-5, error about 1e-10) of the float64
    forward, logits far enough apart that the choice does not change."""
    r = np.random.default_rng(7)
    l = np.stack([r.permutation(12) * 0.3 + r.uniform(0, 0.1, 12) for _ in range(5)])
    lt, lv = stored(l, "f32")
    dwt, dw = f32(r.standard_normal((5, 4)))
    e, w, dl = torch.empty((5, 4), dtype=torch.int32, device="cuda"), torch.empty((5, 4), device="cuda"), torch.empty_like(lt)
    b.sfl_route_forward(lt, e, w, normalise=normalise, scale=1.5)
    b.sfl_route_backward(lt, e, dwt, dl, normalise=normalise, scale=1.5)
    got, h = dl.cpu().double().numpy(), 1e-5
    for i in np.ndindex(l.shape):
        up, down = lv.copy(), lv.copy()
        up[i] += h
        down[i] -= h
        q = ((block.route_forward(up, 4, normalise, 1.5)[1] - block.route_forward(down, 4, normalise, 1.5)[1]) * dw).sum()
        assert abs(q / (2 * h) - got[i]) < 1e-5
