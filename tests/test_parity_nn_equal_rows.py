"""GPU: layer norm over rows of equal values, whose binary32 sum is not a multiple of
the value.

With d = x - m for the rounded mean m, d is the same few units of x in every column, so
sums of d are exact and the corrected mean is x itself: Y = beta to the bit.  The sum of a
row of up to 16384 columns is off by at most 46 roundings (32 values a thread, six
steps in a wavefront, eight wavefronts), so |d| <= 46 * 2^-23 |x|; the variance is the
difference of two squares of that, off by 4 E d^2, E = 2^-24."""
import pytest

import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch

pytestmark = pytest.mark.gpu

T = torch()
E = 2.0 ** -24
VALUES = [1000.1, 0.1, -3.3, 77777.7, 1.0 / 3, 1e6 + 0.3, -1e-3]


@pytest.mark.parametrize("dtype", [T.float32, T.bfloat16, T.float16])
@pytest.mark.parametrize("cols", [1, 7, 77, 500, 513, 1000, 1029, 2047, 2458, 4096, 4099, 8190, 8193, 10007, 16384])
def test_equal_values(cols, dtype):
    x = T.tensor(VALUES, device=DEV).to(dtype)
    x = x[T.isfinite(x)]
    g = T.Generator(device=DEV).manual_seed(cols)
    gamma, beta = T.randn(cols, generator=g, device=DEV), T.randn(cols, generator=g, device=DEV)
    X, eps = x[:, None].expand(-1, cols).contiguous(), 1e-5
    Y, mean, rstd = sa.layer_norm_fwd(X, gamma, beta, eps)
    assert T.equal(mean, x.float())
    assert T.equal(Y, beta.to(dtype).expand_as(Y))
    var = 4 * E * (46 * 2.0 ** -23 * x.double()) ** 2
    want = eps ** -0.5
    assert ((rstd.double() - want).abs() <= want * (6 * E + 0.5 * var / eps)).all()
    # dX = rstd * (t - mean t), xn = 0; t = dy gamma
    dY = T.randn(len(x), cols, generator=g, device=DEV).to(dtype)
    dX, dg, db = sa.layer_norm_bwd(dY, X, mean, rstd, gamma)
    assert not dg.any()


@pytest.mark.parametrize("cols", [16385, 20000, 40007])
def test_equal_values_of_long_rows(cols):
    """A thread adds cols / 1024 values and those of a row are off by as many
    roundings more; the sum of d by (cols / 1024 + 30) E of itself."""
    x = T.tensor(VALUES, device=DEV)
    X, eps = x[:, None].expand(-1, cols).contiguous(), 1e-5
    Y, mean, rstd = sa.layer_norm_fwd(X, eps=eps)
    n = cols / 1024 + 30
    d = n * 2.0 ** -23 * x.double().abs()
    assert ((mean.double() - x.double()).abs() <= E * x.double().abs() + n * E * d).all()
    assert (Y.double().abs() <= (eps ** -0.5 * 1.01 * n * E * d)[:, None]).all()


@pytest.mark.parametrize("cols", [300, 4096, 20000])
def test_a_mean_far_from_zero(cols):
    """Rows of mean 1000 and deviation 2^-6: x is exact, so the statistics are known."""
    g = T.Generator(device=DEV).manual_seed(cols)
    k = T.randint(-2, 3, (6, cols), generator=g, device=DEV).float()
    X = 1000.0 + k * 2.0 ** -6
    Y, mean, rstd = sa.layer_norm_fwd(X, eps=1e-12)
    x = X.double()
    m, d = x.mean(1), x - x.mean(1, keepdim=True)
    s = (d.square().mean(1) + 1e-12).rsqrt()
    n = cols / 1024 + 46
    first = n * E * 1000.0  # of the first mean; what is left of it after the correction:
    left = n * E * (first + d.abs().mean(1))
    assert ((mean.double() - m).abs() <= 1000.0 * E + left).all()
    er = n * E * (1 + (first * s) ** 2) + (left * s) ** 2 + 8 * E
    assert ((rstd.double() - s).abs() <= s * er).all()
    tol = d.abs() * s[:, None] * (er + 8 * E)[:, None] + (left * s)[:, None]
    assert ((Y.double() - d * s[:, None]).abs() <= 1.01 * tol + E).all()
