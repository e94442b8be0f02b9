"""GPU: a weight gradient summed over as many rows as the operators take."""
import pytest

import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch

pytestmark = pytest.mark.gpu

T = torch()


def test_sum_over_the_most_rows():
    """2^31 - 1 rows of one element, 4 GiB each; all but a few are zeros, and the
    products of the others are whole numbers, so the sums are exact."""
    M = (1 << 31) - 1
    at = T.tensor([0, 1, 63, 64, 1 << 20, (1 << 30) + 5, (1 << 31) - 66, (1 << 31) - 65, (1 << 31) - 64, M - 2, M - 1],
                  device=DEV)
    dY, X = (T.zeros(M, 1, dtype=T.bfloat16, device=DEV) for _ in range(2))
    dY[at, 0] = T.arange(1, len(at) + 1, device=DEV).bfloat16()
    X[at, 0] = T.arange(3, len(at) + 3, device=DEV).bfloat16()
    W = T.ones(1, 1, dtype=T.bfloat16, device=DEV)
    _, dW, db = sa.linear_bwd(dY, X, W, grads="wb")
    assert dW.item() == sum((i + 1) * (i + 3) for i in range(len(at)))
    assert db.item() == sum(range(1, len(at) + 1))
    del dY, X
    T.cuda.empty_cache()
