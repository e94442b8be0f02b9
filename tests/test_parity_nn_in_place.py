"""GPU: layer norm gradients written over the residual path's gradient, in rows whose last
vector overlaps the one before it."""
import pytest

import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch

pytestmark = pytest.mark.gpu

T = torch()


@pytest.mark.parametrize("dtype", [T.bfloat16, T.float16, T.float32])
@pytest.mark.parametrize("rows,cols", [(1, 5), (700, 77), (1500, 513), (1500, 1025), (2000, 1537), (2000, 2458), (1200, 4099),
                                       (600, 8190), (300, 12291), (40, 16391)])
def test_gradient_in_the_residuals_place(rows, cols, dtype):
    g = T.Generator(device=DEV).manual_seed(cols)
    X, dY, dR = (T.randn(rows, cols, generator=g, device=DEV).to(dtype) for _ in range(3))
    gamma = T.randn(cols, generator=g, device=DEV)
    _, mean, rstd = sa.layer_norm_fwd(X, gamma)
    want = sa.layer_norm_bwd(dY, X, mean, rstd, gamma, dR=dR)
    got = sa.layer_norm_bwd(dY, X, mean, rstd, gamma, dR=dR, dX=dR)
    for a, b in zip(got, want):
        assert T.equal(a, b)
    Y = sa.layer_norm_fwd(X, gamma)[0]
    assert T.equal(sa.layer_norm_fwd(X, gamma, Y=X)[0], Y)
