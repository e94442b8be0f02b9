"""GPU: layer norms of more rows than one launch takes (HIP counts a launch's
threads along x in 32 bits; 64 to 1024 threads work on a row)."""
import pytest

import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch

pytestmark = pytest.mark.gpu

T = torch()


def spots(rows, step):
    """The first and last rows and those on both sides of every multiple of step."""
    at = {0, 1, rows - 2, rows - 1}
    for b in range(step, rows, step):
        at |= {b - 1, b}
    return T.tensor(sorted(at), device=DEV)


def check(rows, cols, step):
    """Every row alone gives the row's result; most rows are all zeros, whose
    results are known: Y = beta, mean 0, dX = dR."""
    g = T.Generator(device=DEV).manual_seed(rows)
    at = spots(rows, step)
    X = T.zeros(rows, cols, dtype=T.bfloat16, device=DEV)
    X[at] = T.randn(len(at), cols, generator=g, device=DEV).bfloat16()
    gamma, beta = (T.randn(cols, generator=g, device=DEV) for _ in range(2))
    few = X[at].clone()
    want, wm, ws = sa.layer_norm_fwd(few, gamma, beta)
    Y, mean, rstd = sa.layer_norm_fwd(X, gamma, beta)
    assert T.equal(Y[at], want) and T.equal(mean[at], wm) and T.equal(rstd[at], ws)
    other = T.ones(rows, dtype=T.bool, device=DEV)
    other[at] = False
    assert not mean[other].any()
    assert int((rstd == rstd[other][0]).sum()) >= rows - len(at)
    for i in range(0, rows, 1 << 22):  # every row was written
        keep = other[i:i + (1 << 22)]
        assert (Y[i:i + (1 << 22)][keep] == beta.bfloat16()).all()
    dY = Y  # the gradient takes dY's place
    dY.zero_()
    dY[at] = T.randn(len(at), cols, generator=g, device=DEV).bfloat16()
    dy = dY[at].clone()
    wx, wg, wb = sa.layer_norm_bwd(dy, few, wm, ws, gamma)
    dX, dg, db = sa.layer_norm_bwd(dY, X, mean, rstd, gamma, dX=dY)
    assert T.equal(dX[at], wx)
    for i in range(0, rows, 1 << 22):
        assert not dX[i:i + (1 << 22)][other[i:i + (1 << 22)]].any()
    # the rows of zeros add exactly; len(at) terms in binary32, in two orders
    x = (few.double() - wm.double()[:, None]) * ws.double()[:, None]
    e = 2 * (len(at) + 16) * 2.0 ** -24
    assert ((dg - wg).abs().double() <= e * (dy.double() * x).abs().sum(0)).all()
    assert ((db - wb).abs().double() <= e * dy.double().abs().sum(0)).all()


def test_more_rows_than_a_launch_takes():
    check((1 << 26) + 3, 8, 1 << 22)


def test_more_long_rows_than_a_launch_takes():
    check((1 << 18) + 3, 16392, 1 << 18)
