"""Numbers in 8 bits: codes and scales bit for bit against the float64 definition, both layouts."""
import numpy as np
import pytest
import torch

from block_util import DT, shifted, stored
from oracle import routed as o
from paper_2603_23198_amd import binding as b
from routed_util import Bytes, F8, column_outputs, row_outputs, run_offsets, same_codes, up

pytestmark = pytest.mark.gpu


def spread(rng, T, d):
    """Rows of different magnitude with channels that stand out."""
    return rng.normal(size=(T, d)) * np.exp(rng.normal(size=(T, 1)) * 2) * np.where(rng.random(d) < 0.05, 30, 1)


def check_rows(Q, S, x, rows=None):
    T, d = x.shape
    q, e = o.quant(x)
    rows = np.arange(T) if rows is None else rows
    got, s = Q.values(), S.values()
    same_codes(got[rows], q[rows])
    np.testing.assert_array_equal(s[rows, :e.shape[1]], e[rows] + 127)
    assert (s[rows, e.shape[1]:] == 127).all()
    rest = np.setdiff1d(np.arange(T), rows)
    assert (got[rest] == Q.fill).all() and (s[rest] == S.fill).all(), "rows of no run"


def check_columns(Qt, St, x, offsets):
    q, e = o.quant_columns(x, offsets)
    got, s = Qt.values(), St.values()
    same_codes(got[:, :q.shape[1]], q)
    np.testing.assert_array_equal(s[:, :e.shape[1]], e + 127)
    assert (got[:, q.shape[1]:] == Qt.fill).all() and (s[:, e.shape[1]:] == St.fill).all(), "behind the last run"


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 1), (1, 8), (3, 7), (2, 127), (5, 128), (4, 129), (3, 511), (2, 512), (7, 520), (9, 1003),
                                 (300, 2048)])
def test_rows(dt, T, d):
    rng = np.random.default_rng(T * 1000 + d)
    for by in (0, 1, 2):  # rows of element alignment
        X, x = stored(spread(rng, T, d), dt)
        Q, S = row_outputs(T, d)
        b.sfl_quant_rows(shifted(X, by), Q.t, S.t)
        check_rows(Q, S, x)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1, 64, 129, 264, 1003])
@pytest.mark.parametrize("loads", [[1], [127, 1, 128, 129], [0, 0, 5, 0], [0, 300, 0, 0, 257, 0], [0, 0]])
def test_rows_and_columns(dt, d, loads):
    rng = np.random.default_rng(d)
    T = sum(loads)
    X, x = stored(spread(rng, max(T, 1), d)[:T], dt)
    of, offsets = run_offsets(loads)
    for rows in (True, False):
        Q, S = row_outputs(T, d)
        Qt, St = column_outputs(d, b.sfl_quant_columns(T, len(loads)))
        b.sfl_quant_rows(X, Q.t if rows else None, S.t if rows else None, Qt=Qt.t, St=St.t, offsets=offsets)
        check_columns(Qt, St, x, of)
        if rows:
            check_rows(Q, S, x)


def test_one_run_without_offsets():
    rng = np.random.default_rng(2)
    X, x = stored(spread(rng, 200, 140), "bf16")
    Q, S = row_outputs(200, 140)
    Qt, St = column_outputs(140, b.sfl_quant_columns(200, 1) + 512)  # wider than need be
    b.sfl_quant_rows(X, Q.t, S.t, Qt=Qt.t, St=St.t)
    check_rows(Q, S, x)
    check_columns(Qt, St, x, [0, 200])


@pytest.mark.parametrize("columns", [True, False])
def test_rows_of_no_run_are_left(columns):
    """Runs that begin behind the first row and end before the last, as in a batch of fixed room."""
    rng = np.random.default_rng(4)
    X, x = stored(spread(rng, 300, 200), "f32")
    of, offsets = run_offsets([100, 0, 91], first=7)
    Q, S = row_outputs(300, 200)
    Qt, St = column_outputs(200, b.sfl_quant_columns(300, 3))
    b.sfl_quant_rows(X, Q.t, S.t, Qt=Qt.t if columns else None, St=St.t if columns else None, offsets=offsets)
    check_rows(Q, S, x, np.arange(7, 198))
    if columns:
        check_columns(Qt, St, x, of)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_where(dt):
    """Elements where another batch is not above zero (zeros, NaN) are zeros; the batch may be X."""
    rng = np.random.default_rng(6)
    x0, w0 = spread(rng, 150, 300), rng.normal(size=(150, 300))
    w0[rng.random(w0.shape) < 0.1] = 0
    w0[rng.random(w0.shape) < 0.05] = np.nan
    w0[3], w0[:, 7] = -1, -1  # a block without any
    X, x = stored(x0, dt)
    W, w = stored(np.nan_to_num(w0), dt)
    W[torch.from_numpy(np.isnan(w0)).cuda()] = float("nan")
    x0 = np.where(w0 > 0, x, 0)
    Q, S = row_outputs(150, 300)
    Qt, St = column_outputs(300, 512)
    b.sfl_quant_rows(X, Q.t, S.t, Qt=Qt.t, St=St.t, where=W)
    check_rows(Q, S, x0)
    check_columns(Qt, St, x0, [0, 150])
    Q, S = row_outputs(150, 300)
    b.sfl_quant_rows(X, Q.t, S.t, where=X)
    check_rows(Q, S, np.where(x > 0, x, 0))


def borders(dt):
    """Rows of 128 whose largest element lies where a scale changes, with halves between codes, zeros of
    both signs, subnormal numbers, and elements that are not finite."""
    rng = np.random.default_rng(8)
    top = np.array([448, 449, 450, 224, 225, 1, 1.75, 1.7578125, 2.0 ** 120, 2.0 ** -100, 2.0 ** -118, 2.0 ** -119,
                    2.0 ** -125, 2.0 ** -126, 0, 2.0 ** 127, 3.38e38, -448, -2.0 ** -126])
    x = rng.choice(np.append(o.e4m3_values(), (o.e4m3_values()[1:] + o.e4m3_values()[:-1]) / 2), size=(top.size, 128)) / 448
    x = x * np.where(rng.random(x.shape) < 0.5, -1, 1) * np.abs(top)[:, None]
    x[:, 0] = top
    x[:, 1:3] = 0.0, -0.0
    special = x[[0, 5, 14]].copy()
    special[0, [3, 50]], special[1, 9], special[2, [0, 127]] = (np.nan, np.inf), -np.inf, (np.inf, np.nan)
    return np.concatenate([x, special])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_borders(dt):
    with np.errstate(over="ignore"):
        x = borders(dt)
    X = torch.from_numpy(x.astype(np.float32)).cuda().to(DT[dt])
    x = X.float().cpu().numpy().astype(np.float64)
    Q, S = row_outputs(*x.shape)
    b.sfl_quant_rows(X, Q.t, S.t)
    check_rows(Q, S, x)
    turned = np.ascontiguousarray(x.T)
    Qt, St = column_outputs(x.shape[0], 512)
    b.sfl_quant_rows(X.t().contiguous(), Qt=Qt.t, St=St.t)
    check_columns(Qt, St, turned, [0, 128])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("E,R,C", [(1, 1, 1), (1, 128, 128), (2, 129, 127), (3, 200, 333), (1, 513, 260), (2, 64, 1100)])
def test_weights(dt, E, R, C):
    rng = np.random.default_rng(E * R + C)
    W, w = stored(rng.normal(size=(E, R, C)) * np.exp(rng.normal(size=(E, R, 1))), dt)
    for which in ((True, True), (True, False), (False, True)):
        Q, S = Bytes((E, R, up(C)), F8), Bytes((E, up(R) // 128, up(up(C) // 128, 4)))
        Qt, St = Bytes((E, C, up(R)), F8), Bytes((E, up(C) // 128, up(up(R) // 128, 4)))
        b.sfl_quant_weights(W, *((Q.t, S.t) if which[0] else ()), **(dict(Qt=Qt.t, St=St.t) if which[1] else {}))
        for e in range(E):
            for use, codes, scales, m in ((which[0], Q, S, w[e]), (which[1], Qt, St, np.ascontiguousarray(w[e].T))):
                got, s = codes.values()[e], scales.values()[e]
                if not use:
                    assert (got == codes.fill).all() and (s == scales.fill).all()
                    continue
                q, ex = o.quant_square(m)
                same_codes(got, q)
                np.testing.assert_array_equal(s[:, :ex.shape[1]], ex + 127)
                assert (s[:, ex.shape[1]:] == 127).all()


def test_offsets_without_meaning_stay_in_bounds():
    """Descending offsets, ones below zero and past the batch: what is written is no one's, and lies
    within the buffers."""
    X, _ = stored(np.ones((100, 140)), "bf16")
    for of in ([50, 20, 90, 10], [-5, 300, 7, 1000], [0, 100, 0, 100], [1 << 30, -(1 << 30), 5, 100]):
        Q, S = row_outputs(100, 140)
        Qt, St = column_outputs(140, b.sfl_quant_columns(100, 3))
        b.sfl_quant_rows(X, Q.t, S.t, Qt=Qt.t, St=St.t, offsets=torch.tensor(of, dtype=torch.int32, device="cuda"))
        for t in (Q, S, Qt, St):
            t.values()


def test_no_rows():
    X = torch.empty((0, 64), device="cuda")
    Q, S = torch.empty((0, 128), dtype=F8, device="cuda"), torch.empty((0, 4), dtype=torch.uint8, device="cuda")
    b.sfl_quant_rows(X, Q, S)
