"""The root-mean-square norm over the whole range of its types: rows whose squares leave
binary32 on either side, beside ordinary ones.

Bounds as in test_parity_nn8: a sum of cols squares is good to (cols + 16) E, half of which
comes through the root.  rstd below 2^-126 is rounded to a multiple of 2^-149.
"""
import pytest

import nn8_reference as ref8
import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch
from test_parity_nn import E, check, gen, rounded, vec
from test_parity_nn8 import same_bits

pytestmark = pytest.mark.gpu

T = torch()

COLS = [1, 5, 64, 300, 1000, 1229, 2458, 4096, 9830, 16385, 20000]  # every layout of rows


def rows_of(g, cols, dtype):
    """Ordinary rows between others whose sums of squares overflow or underflow."""
    x = T.randn(11, cols, generator=g, device=DEV)
    x[1, cols // 2] = 1e20
    x[2] *= 1e20
    x[3] = 3e38 * x[3].sign()
    x[5] *= 1e-25
    x[6] = x[6].sign() * 2.0 ** -131  # below the normal numbers
    x[7] = 0.0
    x[8, ::2] *= 1e20
    x[8, 1::2] *= 1e-30
    x[9] = 4e18 * x[9].sign()  # only their sum overflows, and not everywhere
    x[10, 1:] = 0.0
    x[10, 0] = 1e-30
    return x.to(dtype)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-5, 3e38])
@pytest.mark.parametrize("residual", [False, True])
def test_rms_norm_of_any_finite_row(cols, dtype, eps, residual):
    dt = {"bf16": T.bfloat16, "f32": T.float32}[dtype]
    g = gen(cols)
    X, gamma = rows_of(g, cols, dt), vec(g, cols, 0.2, 1.0)
    R = (X.double() * T.rand(11, 1, generator=g, device=DEV).double() * -0.5).to(dt) if residual else None
    if eps == 0.0:
        X[7] = 1.0  # 0 / 0 otherwise
    Y, S, rstd, Q = sa.rms_norm_fwd(X, gamma, R=R, eps=eps, out="ysrq")
    s = X if R is None else (X.float() + R.float()).to(dt)
    assert T.equal(S, s)
    # eps as the descriptor holds it
    y, r = ref8.rms_fwd(s.double(), gamma.double(), T.tensor(eps, dtype=T.float32).double().item())
    er = (cols + 16) * E
    top = T.finfo(T.float32).max
    assert T.equal(rstd.isinf(), r > top)  # a norm below 2^-128: its reciprocal leaves binary32, Y does not
    kept = ~rstd.isinf()
    check(rstd[kept], r[kept], er * r[kept] + 2.0 ** -150, "rstd")
    tol = (er + 8 * E) * y.abs()
    check(Y, y, tol + rounded(y, dt) + 2.0 ** -150, "Y")
    ref8.check_codes(Q, y, tol + 2.0 ** -149, "Q")
    # alone, in a launch without the other rows, and in the inputs' place
    for i in (0, 2, 5, 9):
        one = sa.rms_norm_fwd(X[i:i + 1], gamma, R=None if R is None else R[i:i + 1], eps=eps, out="yrq")
        assert T.equal(one[0], Y[i:i + 1]) and T.equal(one[2], rstd[i:i + 1])
        assert same_bits(one[3].codes, Q.codes[i:i + 1]) and T.equal(one[3].scales, Q.scales[i:i + 1])
    x2, r2 = X.clone(), None if R is None else R.clone()
    sa.rms_norm_fwd(x2, gamma, R=r2, eps=eps, S=x2, Y=r2, out="r")
    assert T.equal(x2, S) and (R is None or T.equal(r2, Y))


@pytest.mark.parametrize("cols", [300, 4096, 20000])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_infinities_and_nan_stay_in_their_rows(cols, eps):
    g = gen(cols)
    X = rows_of(g, cols, T.float32)
    X[7] = 1.0
    want = sa.rms_norm_fwd(X, eps=eps)
    X[3, 1], X[8, 2] = float("inf"), float("nan")
    Y, _, rstd, _ = sa.rms_norm_fwd(X, eps=eps)
    keep = [0, 1, 2, 4, 5, 6, 7, 9, 10]
    assert T.equal(Y[keep], want[0][keep]) and T.equal(rstd[keep], want[2][keep])
    # 1 / infinity: the infinity's own result is NaN, the others 0
    assert rstd[3] == 0 and Y[3, 1].isnan() and (Y[3, 2:] == 0).all()
    assert rstd[8].isnan() and Y[8].isnan().all()
