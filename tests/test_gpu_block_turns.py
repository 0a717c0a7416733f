"""Batches of which every workgroup takes several rows in turn (and long expert rows and gradient
shares): the loops over rows, against the float64 definition.

Bounds. Rows as for single turns: sums of d terms in at least 64 partial sums, d / 64 + 64 fp32
roundings. A parameter's gradient is added over a thread's rows (one rounding each), over the R rows
that a workgroup has at a time, over every 32nd workgroup and over 32 such sums: about 1e-5 of the
magnitudes' sum in all, less than one row's part of it in batches of up to 80000 rows."""
import numpy as np
import pytest
import torch

from oracle import block
from tests import test_gpu_block_norm as norms
from tests import test_gpu_experts as experts
from tests import test_gpu_gradients as gradients
from tests.block_util import DT, Out, assert_rounded

pytestmark = pytest.mark.gpu

b = pytest.importorskip("paper_2603_23198_amd.binding")

WIDTHS = [9, 100, 136, 300, 513, 640, 1032, 2048, 4096]
WIDE = [8192, 8200, 16384]


def rows_at_a_time(d):
    """R: rows of up to 512 columns share a workgroup of 256 threads."""
    lanes = 8
    while lanes < -(-d // 8):
        lanes *= 2
    return 256 // lanes if lanes <= 64 else 1


def check_backward(T, d, dt, form, eps=1e-6):
    dev, val, bits = norms.setup(T, d, dt, form, T + d)
    blocks = b.sfl_norm_workspace_size(T, d, dt) // (8 * d)
    R = rows_at_a_time(d)
    turns = -(-T // (blocks * R))
    outs = {"dX": Out((T, d), DT[dt]), "dY": Out((T, d), DT[dt]), "dgate_c": Out((d,), torch.float32),
            "dgate_t": Out((T,), torch.float32)}
    if form["pre"]:
        outs["dw_pre"] = Out((d,), torch.float32)
    if form["post"]:
        outs["dw_post"] = Out((d,), torch.float32)
    ws = torch.empty(b.sfl_norm_workspace_size(T, d, dt), dtype=torch.uint8, device="cuda")
    kw = dict(res_scale=0.75, eps=eps)
    b.sfl_norm_backward(dev["X"], dev["Y"], dev["dX_out"], dev["dN"], norms=bits, workspace=ws, **kw,
                        **{n: dev[n] for n in norms.PARAMS}, **{n: o.t for n, o in outs.items()})
    want = block.norm_backward(val["X"], val["Y"], val["dX_out"], val["dN"], pre=form["pre"], post=form["post"], **kw,
                               **{n: val[n] for n in norms.PARAMS})
    row = d / 64 + 64
    for n, o in outs.items():
        rows = n in ("dX", "dY")
        sums = 0 if rows or n == "dgate_t" else turns + R + -(-blocks // 32) + 32
        assert_rounded(o.values(), *want[n], dt if rows else "f32", row + sums, n)
    return turns


def batch(d, dt, turns):
    """Tokens of so many turns of every workgroup and a part of one more, not a multiple of R."""
    T = 1
    while True:  # the workspace holds 8 d bytes per workgroup and stops growing at the most of them
        most = b.sfl_norm_workspace_size(T, d, dt) // (8 * d)
        if T > 2 * most * rows_at_a_time(d):
            return int((turns + 0.4) * most * rows_at_a_time(d)) | 1
        T *= 2


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS + WIDE)
def test_norm_backward(d, dt):
    assert check_backward(batch(d, dt, 2 if d < 8192 else 1), d, dt, norms.FORMS[0]) >= 2


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("form", [norms.FORMS[3], norms.FORMS[4], norms.FORMS[6]],
                         ids=lambda f: "-".join(k for k, v in f.items() if v))
def test_norm_backward_forms(form, dt):
    for d in (100, 640):
        assert check_backward(batch(d, dt, 1), d, dt, form) == 2


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_norm_backward_groups_past_the_last_row(dt):
    """They add nothing, without an eps either."""
    for d in (9, 100, 136, 300):
        for T in (1, 3, 65, 1001):
            check_backward(T, d, dt, norms.FORMS[0], eps=0.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS + WIDE)
def test_norm_forward(d, dt):
    threads = 256 if d <= 512 else min(1024, -(-d // 512) * 64)
    most = 256 * (4096 // threads) * rows_at_a_time(d)
    norms.forward(int(1.15 * most) | 1, d, dt, norms.FORMS[0], seed=d)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_expert_rows(dt):
    """Over 2048 slots (the rows in a launch of their own) of every number of threads per row."""
    for d in (64, 100, 513, 1025, 2047, 4100):
        experts.test_rows_there_and_back(1100, d, 2, 4, "holes", dt)
    experts.test_rows_there_and_back(700, 2056, 3, 60, "skew", dt)


LONG = [([5_000_003], ["f32"]), ([3_000_001, 4097, 8193, 70_001], ["f32", "f32", "bf16", "f32"]),
        ([9_000_007, 2_000_000, 123], ["bf16", "f32", "f32"]), ([40_961] * 120, ["f32"] * 120)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sizes,kinds", LONG, ids=range(len(LONG)))
def test_gradient_shares(sizes, kinds, in_place):
    """Lists long enough for every length of a workgroup's share."""
    gradients.check(sizes, kinds, 0.5, in_place=in_place)
    gradients.check(sizes, kinds, 1e9, in_place=in_place)
    gradients.check(sizes, kinds, 3.0, by=1, in_place=in_place)
