"""GPU: values and slopes of the activations by themselves, relative to their own size.

A product of one term is exact, so z is exact and what is left is the activation's
own arithmetic, written to binary32.  E = 2^-24.  An exponential exp(-y) is off by
(5 y + 4) E: the rounding of y, of its product with log2 e and of that constant, one
unit of the hardware's 2^t.  What a formula multiplies it with adds a few E."""
import math

import pytest

import nn_reference as ref
import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch

pytestmark = pytest.mark.gpu

T = torch()
E = 2.0 ** -24
TINY = 2.0 ** -126  # below the smallest normal number nothing is promised


def grid(dtype, largest):
    """Every value of a 16-bit type from 2^-12 to `largest` in size, and 0."""
    z = T.arange(-32768, 32768, device=DEV).to(T.int16).view(dtype)
    z = z[(z.float().abs() >= 2.0 ** -12) & (z.float().abs() <= largest)]
    return T.cat([z, T.zeros(1, dtype=dtype, device=DEV)])


def values(z, a):
    """act(z) in binary32: of single rows, and of the tiles that more rows take."""
    one, wide = T.ones(1, 1, dtype=z.dtype, device=DEV), T.ones(640, 1, dtype=z.dtype, device=DEV)
    row = sa.linear_fwd(one, z[:, None], act=sa.ACTS[a], out_dtype=T.float32)[0]
    tiles = sa.linear_fwd(z[:, None].contiguous(), wide, act=sa.ACTS[a], out_dtype=T.float32)
    # the gated pair's du = act(g) for dh = 1: its column sum over one row, in binary32
    G, n = z[None], len(z)
    w = T.ones(n, 1, dtype=z.dtype, device=DEV)
    pair = sa.glu_bwd(T.ones_like(G), one, w, w, G, T.ones_like(G), act=sa.ACTS[a], grads="b")
    assert T.equal(tiles, tiles[:, :1].expand_as(tiles))
    return {"row": row, "tiles": tiles[:, 0], "pair": pair[4]}, {"pair": pair[3]}


def slopes(z, a):
    """act'(z) in binary32: the bias gradient of one row with dY = 1."""
    one, w = T.ones(1, 1, dtype=z.dtype, device=DEV), T.ones(len(z), 1, dtype=z.dtype, device=DEV)
    return sa.linear_bwd(T.ones_like(z)[None], one, w, Z=z[None], act=sa.ACTS[a], grads="b")[2]


def check(got, want, tol, z, what):
    bad = ~((got.double() - want).abs() <= tol + TINY)
    i = int(bad.nonzero()[0]) if bad.any() else 0
    assert not bad.any(), (what, int(bad.sum()), float(z[i]), float(got[i]), float(want[i]), float(tol[i]))


@pytest.mark.parametrize("dtype", [T.bfloat16, T.float16])
def test_gelu(dtype):
    """z Phi(z) without the cancellation of 1 + erf in the lower tail.  exp(-z^2/2)
    is the square of an exponential of z^2/4: (2.5 z^2 + 8) / 2 E each, twice; the
    polynomial of the tail is off by 7 E, five products and sums follow."""
    z = grid(dtype, 13.0)
    x = z.double()
    want, slope = ref.act("gelu", x), ref.dact("gelu", x)
    rel = (2.5 * x * x + 24) * E
    got, pair = values(z, "gelu")
    for k, v in got.items():
        check(v, want, rel * want.abs(), z, k)
    # two terms, of opposite signs below 0
    size = 0.5 * T.erfc(-x / math.sqrt(2)) + x.abs() * T.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    check(slopes(z, "gelu"), slope, rel * size, z, "slope")
    check(pair["pair"], slope, rel * size, z, "slope of the pair")
