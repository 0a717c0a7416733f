"""Global gradient norm and clipping on the GPU. Squares are summed in fp64 (n terms: relative
error below n 2^-53), the norm is rounded once to fp32; a clipped value is one fp32 product of the
rounded coefficient (two roundings), and one to the stored type."""
import math

import numpy as np
import pytest
import torch

from oracle import block
from tests.block_util import DT, Out, assert_rounded, same_bits, stored

pytestmark = pytest.mark.gpu

b = pytest.importorskip("paper_2603_23198_amd.binding")


def total(grads, workspace=None):
    q = torch.full((1,), -1.0, dtype=torch.float64, device="cuda")
    ws = torch.empty(b.sfl_grad_workspace_size(grads), dtype=torch.uint8, device="cuda")
    b.sfl_grad_sumsq(grads, q, workspace=ws)
    return q


def check(sizes, kinds, max_norm, seed=0, std=1.0, in_place=False, by=0):
    r = np.random.default_rng(seed)
    vals, src, dst = [], [], []
    for n, dt in zip(sizes, kinds):
        t, v = stored(std * r.standard_normal(n), dt)
        o = Out((n,), DT[dt], by)
        o.t.copy_(t)
        vals.append(v)
        src.append(o)
        dst.append(o if in_place else Out((n,), DT[dt], by))
    grads = b.grad_list([o.t for o in src], None if in_place else [o.t for o in dst])
    q, norm = total(grads), Out((1,), torch.float32)
    want, scaled = block.clip(vals, max_norm)
    assert abs(q.item() - want * want) <= 1e-12 * want * want
    b.sfl_grad_clip(grads, q, max_norm, norm.t)
    assert_rounded(norm.values(), np.array([want]), want, "f32", 2)
    for o, w, v, dt in zip(dst, scaled, vals, kinds):
        if want <= max_norm:
            np.testing.assert_array_equal(o.values(), v)
        else:
            assert_rounded(o.values(), w, np.abs(w), dt, 4)
    for o, v in zip(src, vals):
        if not in_place:
            np.testing.assert_array_equal(o.values(), v)


LISTS = [([1], ["f32"]), ([0, 5, 0], ["bf16", "f32", "f32"]), ([7, 4096, 300001], ["f32", "bf16", "bf16"]),
         ([262144, 1024, 262144, 256], ["f32"] * 4), ([16384, 16385, 16383, 3, 65537], ["bf16", "f32", "bf16", "f32", "bf16"]),
         ([1 + 131 * i % 997 for i in range(400)], ["bf16" if i % 3 else "f32" for i in range(400)])]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sizes,kinds", LISTS, ids=range(len(LISTS)))
def test_clip(sizes, kinds, in_place):
    check(sizes, kinds, 1e-3, in_place=in_place)     # far above the largest norm
    check(sizes, kinds, 1e9, in_place=in_place)      # below it: nothing changes
    check(sizes, kinds, 0.5, by=1, in_place=in_place)
    check(sizes, kinds, 0.0, by=3, in_place=in_place)


def test_views_of_one_bucket():
    """Tensors that lie end to end go as one range: with gaps, other types and empty tensors among
    them, in order and not, in place and to buckets laid out alike and otherwise."""
    r = np.random.default_rng(3)
    flat = {"f32": torch.empty(40000, device="cuda"), "bf16": torch.empty(40000, device="cuda", dtype=torch.bfloat16)}
    vals = {n: stored(r.standard_normal(40000), n) for n in flat}
    for lens, order, skip in [([5000] * 8, range(8), 0), ([1, 4095, 4097, 0, 3, 20000, 7], range(7), 0),
                              ([5000] * 8, [3, 4, 5, 0, 1, 7, 6, 2], 0), ([999] * 20, range(20), 1)]:
        for n in flat:
            flat[n].copy_(vals[n][0])
        at = np.concatenate([[0], np.cumsum([l + skip for l in lens])])
        src = [flat["bf16" if i % 3 == 2 else "f32"][at[i]:at[i] + lens[i]] for i in order]
        want = torch.cat([t.double() for t in src])
        out = torch.empty(2 * sum(lens) + 64, device="cuda")
        halves = torch.empty(2 * sum(lens) + 64, device="cuda", dtype=torch.bfloat16)
        dst, a = [], 0
        for i, t in zip(order, src):
            dst.append((out if t.dtype == torch.float32 else halves)[a:a + t.numel()])
            a += t.numel() + (16 if i % 2 else 0)
        norm = torch.empty(1, device="cuda")
        q = total(b.grad_list(src))
        assert abs(q.item() - want.square().sum().item()) <= 1e-12 * q.item()
        b.sfl_grad_clip(b.grad_list(src, dst), q, 1.0, norm)
        b.sfl_grad_clip(b.grad_list(src), q, 1.0)
        by = 1.0 / math.sqrt(q.item())
        for got in (dst, src):
            for g, w in zip(got, want.split([t.numel() for t in src])):
                w = (w * by).cpu().numpy()
                assert_rounded(g.cpu().double().numpy(), w, np.abs(w), "f32" if g.dtype == torch.float32 else "bf16", 4)


@pytest.mark.parametrize("std", [1e-30, 1e-22, 1e18, 1e30])
def test_squares_outside_the_fp32_range(std):
    check([5000, 333], ["f32", "bf16"], std, std=std)


def test_empty_lists():
    for grads in (b.grad_list([]), b.grad_list([torch.empty(0, device="cuda")])):
        q, norm = total(grads), torch.full((1,), -1.0, device="cuda")
        b.sfl_grad_clip(grads, q, 1.0, norm)
        assert q.item() == 0 and norm.item() == 0


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_norm_that_is_not_finite_scales_nothing(bad, in_place):
    a, c = torch.randn(40000, device="cuda"), torch.randn(777, device="cuda").bfloat16()
    a[39999] = bad
    out = [torch.empty_like(a), torch.empty_like(c)]
    a0, c0 = a.clone(), c.clone()
    grads = b.grad_list([a, c], None if in_place else out)
    q, norm = total(grads), torch.zeros(1, device="cuda")
    b.sfl_grad_clip(grads, q, 1.0, norm)
    assert not norm.isfinite().item()
    assert same_bits(a, a0) and same_bits(c, c0)
    if not in_place:
        assert same_bits(out[0], a0) and same_bits(out[1], c0)


def test_a_norm_that_fp32_cannot_hold_is_infinite():
    a = torch.full((10000,), 3e37, device="cuda")  # norm 3e39
    grads = b.grad_list([a])
    q, norm = total(grads), torch.zeros(1, device="cuda")
    b.sfl_grad_clip(grads, q, 1.0, norm)
    assert math.isinf(norm.item()) and (a == 3e37).all() and abs(q.item() / (1e4 * a[0].item() ** 2) - 1) < 1e-12


def test_ranks_add_their_sums():
    """Two shards of one list, clipped by the sum of their squares as two ranks would."""
    g = [torch.randn(30000, device="cuda"), torch.randn(12345, device="cuda")]
    whole = b.grad_list(g, [torch.empty_like(t) for t in g])
    parts = [b.grad_list([t], [torch.empty_like(t)]) for t in g]
    q = sum(total(p) for p in parts)
    assert abs(q.item() - total(whole).item()) <= 1e-12 * q.item()
    norm = torch.empty(1, device="cuda")
    b.sfl_grad_clip(parts[0], q, 1.0, norm)
    assert abs(norm.item() - math.sqrt(sum(t.double().square().sum().item() for t in g))) <= 1e-6 * norm.item()


def test_results_are_the_same_from_call_to_call():
    g = [torch.randn(1_000_003, device="cuda"), torch.randn(99_999, device="cuda").bfloat16()]
    grads = b.grad_list(g)
    first = total(grads)
    assert all(same_bits(first, total(grads)) for _ in range(3))


def test_more_elements_than_32_bits():
    n = (1 << 31) + 77
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[n // 2], g[n - 1] = 2.0, 3.0, 6.0
    grads = b.grad_list([g])
    q = total(grads)
    assert q.item() == 49.0
    b.sfl_grad_clip(grads, q, 3.5)
    assert [g[i].item() for i in (0, n // 2, n - 1)] == [1.0, 1.5, 3.0] and g[1].item() == 0


@pytest.mark.parametrize("std,max_norm", [(1e36, 1e-3), (1e36, 1.0), (1e18, 1e-30), (3e-5, 1e-25), (1e30, 1e-12)])
@pytest.mark.parametrize("in_place", [False, True])
def test_coefficients_below_the_fp32_range(std, max_norm, in_place):
    """max_norm / norm may be subnormal or zero in fp32 where the scaled gradients are ordinary numbers."""
    check([5000, 333], ["f32", "bf16"], max_norm, std=std, in_place=in_place)
