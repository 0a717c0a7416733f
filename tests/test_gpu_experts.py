"""Tokens into expert order and back on the GPU: the order exactly, rows moved bit for bit, sums
of k products within k fp32 roundings and one to the stored type, dot products of d terms held in
at least 64 partial sums."""
import numpy as np
import pytest
import torch

from oracle import block
from tests.block_util import DT, Out, assert_rounded, f32, same_bits, shifted, stored

pytestmark = pytest.mark.gpu

b = pytest.importorskip("paper_2603_23198_amd.binding")


def choices(T, k, E, seed, kind="uniform"):
    r = np.random.default_rng(seed)
    if kind == "one":
        return np.full((T, k), E - 1, dtype=np.int32)
    if kind == "none":
        return np.full((T, k), -1, dtype=np.int32)
    e = r.integers(0, E, (T, k)) if kind != "skew" else np.minimum((E * r.uniform(size=(T, k)) ** 4), E - 1)
    e = e.astype(np.int32)
    if kind == "holes":
        e[r.uniform(size=(T, k)) < 0.3] = -1
        e[r.uniform(size=(T, k)) < 0.05] = E + 3
        e[r.uniform(size=(T, k)) < 0.02] = -(1 << 31)
        e[T // 2] = -1
    return e


def space(T, k, E):
    return torch.empty(b.sfl_expert_workspace_size(T, k, E), dtype=torch.uint8, device="cuda")


def order(e, E, by=0):
    T, k = e.shape
    pos, off = Out((T, k), torch.int32, by), Out((E + 1,), torch.int32, by)
    et = torch.from_numpy(e).cuda()
    b.sfl_expert_dispatch(shifted(et, by) if by else et, E, pos.t, off.t, workspace=space(T, k, E))
    return pos, off


ORDERS = [(1, 1, 1, "uniform"), (1, 2, 8, "uniform"), (5, 3, 2, "holes"), (32, 2, 8, "uniform"), (64, 1, 64, "one"),
          (100, 8, 64, "skew"), (257, 4, 60, "holes"), (33, 64, 100, "uniform"), (2048, 2, 8, "uniform"),
          (2049, 2, 8, "skew"), (513, 8, 256, "holes"), (4001, 3, 65, "holes"), (9000, 2, 1024, "skew"),
          (20000, 8, 64, "uniform"), (70000, 2, 8, "skew"), (3000, 2, 16, "one"), (5000, 1, 7, "none"), (40, 1, 1000, "none")]


@pytest.mark.parametrize("T,k,E,kind", ORDERS)
def test_order(T, k, E, kind):
    e = choices(T, k, E, T + E, kind)
    pos, off = order(e, E)
    want, offsets = block.expert_order(e, E)
    np.testing.assert_array_equal(off.values(), offsets)
    np.testing.assert_array_equal(pos.values(), want)


@pytest.mark.parametrize("T,d,k,E,kind", [(1, 1, 1, 1, "uniform"), (1, 2048, 2, 8, "uniform"), (32, 4096, 2, 8, "uniform"),
                                          (33, 7, 3, 5, "holes"), (65, 1003, 8, 60, "holes"), (3000, 96, 2, 8, "skew"),
                                          (50, 256, 64, 80, "holes"), (700, 520, 1, 16, "one"), (10, 8200, 2, 4, "holes"),
                                          (3, 33000, 2, 4, "uniform"), (2100, 264, 4, 256, "holes"), (9, 64, 2, 4, "none")])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rows_there_and_back(T, d, k, E, kind, dt, by=0):
    r = np.random.default_rng(T + d)
    e = choices(T, k, E, T + d, kind)
    pos, offsets = block.expert_order(e, E)
    n = int(offsets[-1])
    move = lambda t: shifted(t, by) if by else t  # noqa: E731
    X, Xv = stored(r.standard_normal((T, d)), dt)
    Ys, Yv = stored(r.standard_normal((n, d)), dt)
    dY, dYv = stored(r.standard_normal((T, d)), dt)
    w, wv = f32(r.uniform(-1, 1, (T, k)))
    X, Ys, dY, w = move(X), move(Ys), move(dY), move(w)
    got_pos, got_off = Out((T, k), torch.int32, by), Out((E + 1,), torch.int32, by)
    Xs, Y, Y1 = Out((n, d), DT[dt], by), Out((T, d), DT[dt], by), Out((T, d), DT[dt], by)
    b.sfl_expert_dispatch(move(torch.from_numpy(e).cuda()), E, got_pos.t, got_off.t, X=X, Xs=Xs.t, workspace=space(T, k, E))
    np.testing.assert_array_equal(got_pos.values(), pos)
    np.testing.assert_array_equal(got_off.values(), offsets)
    want = np.zeros((n, d))
    for j in range(k):
        t = pos[:, j] >= 0
        want[pos[t, j]] = Xv[t]
    np.testing.assert_array_equal(Xs.values(), want)
    b.sfl_expert_combine(Ys, got_pos.t, Y.t, weight=w)
    assert_rounded(Y.values(), *block.expert_combine(Yv, pos, wv), dt, k + 1, "Y")
    b.sfl_expert_combine(Ys, got_pos.t, Y1.t)
    assert_rounded(Y1.values(), *block.expert_combine(Yv, pos), dt, k + 1, "Y of ones")
    dYs, dw = Out((n, d), DT[dt], by), Out((T, k), torch.float32, by)
    b.sfl_expert_combine_backward(dY, Ys, got_pos.t, w, dYs=dYs.t, dweight=dw.t)
    want, want_w = block.expert_combine_backward(dYv, Yv, pos, wv)
    assert_rounded(dYs.values(), want, np.abs(want), dt, 2, "dYs")
    assert_rounded(dw.values(), *want_w, "f32", d / 64 + 32, "dweight")
    # one of the two alone, and weights of ones
    dYs2, dw2 = Out((n, d), DT[dt], by), Out((T, k), torch.float32, by)
    b.sfl_expert_combine_backward(dY, None, got_pos.t, w, dYs=dYs2.t)
    b.sfl_expert_combine_backward(dY, Ys, got_pos.t, w, dweight=dw2.t)
    assert same_bits(dYs.t, dYs2.t) and same_bits(dw.t, dw2.t)
    b.sfl_expert_combine_backward(dY, None, got_pos.t, None, dYs=dYs2.t)
    np.testing.assert_array_equal(dYs2.values(), block.expert_combine_backward(dYv, Yv, pos)[0])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_element_alignment(dt):
    for by in (1, 3):
        for d in (64, 1001):
            test_rows_there_and_back(40, d, 2, 6, "holes", dt, by)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("widths", [range(1, 20), (63, 65, 127, 129, 255, 511, 513, 1023, 1025, 2047, 2049, 4097)],
                         ids=lambda w: f"{min(w)}-{max(w)}")
def test_widths_around_the_kernels_units(widths, dt):
    """Rows that end anywhere in a thread's or a workgroup's columns; one and several launches."""
    for d in widths:
        test_rows_there_and_back(9, d, 3, 4, "holes", dt)
        test_rows_there_and_back(1100 if d < 600 else 5, d, 2, 4, "holes", dt)


def test_fewer_rows_than_slots_and_foreign_positions():
    """Rows beyond the buffer are not written; positions outside it add nothing."""
    T, k, E, d, rows = 50, 2, 4, 72, 60
    e = choices(T, k, E, 1)
    pos, _ = block.expert_order(e, E)
    X, Xv = stored(np.random.default_rng(2).standard_normal((T, d)), "bf16")
    p, off, Xs = Out((T, k), torch.int32), Out((E + 1,), torch.int32), Out((rows, d), torch.bfloat16)
    b.sfl_expert_dispatch(torch.from_numpy(e).cuda(), E, p.t, off.t, X=X, Xs=Xs.t, workspace=space(T, k, E))
    want = np.zeros((rows, d))
    for j in range(k):
        t = pos[:, j] < rows
        want[pos[t, j]] = Xv[t]
    np.testing.assert_array_equal(Xs.values(), want)
    np.testing.assert_array_equal(p.values(), pos)
    wild = pos.copy()
    wild[0, 0], wild[1, 1], wild[2] = 1 << 30, -(1 << 31), rows
    wt = torch.from_numpy(wild).cuda()
    Y, dYs, dw = Out((T, d), torch.bfloat16), Out((rows, d), torch.bfloat16), Out((T, k), torch.float32)
    b.sfl_expert_combine(Xs.t, wt, Y.t)
    assert_rounded(Y.values(), *block.expert_combine(want, wild), "bf16", k + 1)
    b.sfl_expert_combine_backward(X, Xs.t, wt, None, dYs=dYs.t, dweight=dw.t)
    wd, (ww, ws) = block.expert_combine_backward(Xv, want, wild)
    named = np.zeros(rows, dtype=bool)
    named[wild[(wild >= 0) & (wild < rows)]] = True
    np.testing.assert_array_equal(dYs.values()[named], wd[named])
    assert (dYs.values()[~named] == -77).all()
    assert_rounded(dw.values(), ww, ws, "f32", d / 64 + 32)


def test_slots_without_a_row_read_nothing():
    """NaN in rows and weights that no valid slot uses stays out of the sums."""
    pos = torch.tensor([[0, -1], [-1, -1]], dtype=torch.int32, device="cuda")
    Ys = torch.full((2, 40), float("nan"), device="cuda")
    Ys[0] = 2.0
    w = torch.tensor([[0.5, float("nan")], [float("nan"), float("inf")]], device="cuda")
    Y = torch.empty((2, 40), device="cuda")
    b.sfl_expert_combine(Ys, pos, Y, weight=w)
    assert (Y[0] == 1).all() and (Y[1] == 0).all()
    dY, dYs, dw = torch.ones((2, 40), device="cuda"), torch.zeros((2, 40), device="cuda"), torch.full((2, 2), 9.0, device="cuda")
    b.sfl_expert_combine_backward(dY, Ys, pos, w, dYs=dYs, dweight=dw)
    assert (dYs[0] == 0.5).all() and (dYs[1] == 0).all()
    np.testing.assert_array_equal(dw.cpu().numpy(), [[80, 0], [0, 0]])


def test_no_tokens():
    z = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    off = torch.full((9,), 7, dtype=torch.int32, device="cuda")
    b.sfl_expert_dispatch(z, 8, z, off, workspace=space(0, 2, 8))
    assert (off == 0).all()


def test_rows_beyond_32_bit_offsets():
    d, k, E = 16384, 2, 3
    T = (1 << 31) // (d * k) + 7
    e = choices(T, k, E, 3)
    pos, offsets = block.expert_order(e, E)
    X = torch.arange(T, device="cuda")[:, None].expand(T, d).bfloat16().contiguous()  # exact up to 256
    X += (torch.arange(d, device="cuda") % 64)[None, :].bfloat16()
    p, off = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty(E + 1, dtype=torch.int32, device="cuda")
    Xs = torch.empty((T * k, d), dtype=torch.bfloat16, device="cuda")
    b.sfl_expert_dispatch(torch.from_numpy(e).cuda(), E, p, off, X=X, Xs=Xs, workspace=space(T, k, E))
    np.testing.assert_array_equal(p.cpu().numpy(), pos)
    last = np.nonzero(pos[:, 0] == T * k - 1)[0]
    t = int(last[0]) if len(last) else int(np.nonzero(pos[:, 1] == T * k - 1)[0][0])
    assert same_bits(Xs[T * k - 1], X[t])
    Y = torch.empty_like(X)
    w = torch.full((T, k), 0.5, device="cuda")
    b.sfl_expert_combine(Xs, p, Y, weight=w)
    assert same_bits(Y, X)
    Xs.zero_()
    b.sfl_expert_combine_backward(X, None, p, None, dYs=Xs)
    assert same_bits(Xs[T * k - 1], X[t])


def test_on_another_stream():
    T, k, E, d = 4000, 2, 8, 512
    e = torch.from_numpy(choices(T, k, E, 4)).cuda()
    X = torch.randn((T, d), device="cuda").bfloat16()
    p, off, Xs = torch.empty_like(e), torch.empty(E + 1, dtype=torch.int32, device="cuda"), X.new_empty((T * k, d))
    ws = space(T, k, E)
    b.sfl_expert_dispatch(e, E, p, off, X=X, Xs=Xs, workspace=ws)
    torch.cuda.synchronize()
    side, late, Xs2 = torch.cuda.Stream(), torch.empty_like(e), torch.zeros_like(Xs)
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        late.copy_(e)
        b.sfl_expert_dispatch(late, E, p, off, X=X, Xs=Xs2, workspace=ws)
    side.synchronize()
    assert same_bits(Xs, Xs2)
