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
    assert T.allclose(tiles, tiles[:, :1].expand_as(tiles), rtol=0, atol=0, equal_nan=True)
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


def exact(name, z):
    """Value, slope, the sum of the slope's terms' sizes and the exponent, in binary64
    and without differences."""
    c, k = math.sqrt(8 / math.pi), 0.044715
    s = T.sigmoid
    if name == "sigmoid":
        return s(z), s(z) * s(-z), s(z) * s(-z), z.abs()
    if name == "silu":
        d = s(z) * s(-z)
        return z * s(z), s(z) + z * d, s(z) + z.abs() * d, z.abs()
    y, dy = c * (z + k * z ** 3), c * (1 + 3 * k * z * z)
    d = s(y) * s(-y) * dy
    return z * s(y), s(y) + z * d, s(y) + z.abs() * d, y.abs()


@pytest.mark.parametrize("dtype", [T.bfloat16, T.float16])
@pytest.mark.parametrize("name,largest,own", [("sigmoid", 91.0, 0), ("silu", 91.0, 0), ("gelu_tanh", 10.2, 6)])
def test_logistic(name, largest, own, dtype):
    """Both tails of the activations made of s(y) = 1 / (1 + exp(-y)): factors
    exp(-|y| / 2), (2.5 |y| + 4) E each, two of them in the tail; y itself is off by
    `own` E; the reciprocal, products and sums add fewer than 24 E (slopes: 30 E)."""
    z = grid(dtype, largest)
    want, slope, size, y = exact(name, z.double())
    got, pair = values(z, name)
    for k, v in got.items():
        check(v, want, ((5 + own) * y + 24) * E * want.abs(), z, (name, k))
    tol = ((7 + own) * y + 30) * E * size
    check(slopes(z, name), slope, tol, z, (name, "slope"))
    check(pair["pair"], slope, tol, z, (name, "slope of the pair"))


def test_results_next_to_the_smallest_normal_numbers():
    """silu(-88 .. -91) and the others' last values are normal bfloat16 numbers."""
    for name, z in (("silu", [-87.5, -88.0, -89.0, -90.0, -91.0]), ("gelu_tanh", [-10.0, -10.0625]),
                    ("gelu", [-12.875, -13.0])):
        z = T.tensor(z, dtype=T.bfloat16, device=DEV)
        Y = sa.linear_fwd(T.ones(1, 1, dtype=T.bfloat16, device=DEV), z[:, None], act=sa.ACTS[name])[0]
        x = z.double()
        want = ref.act("gelu", x) if name == "gelu" else exact(name, x)[0]
        assert (want.abs() > TINY).all()
        # u of the result, and the exponential's (5 y + 24) E, y at most 100
        assert ((Y.double() - want).abs() <= (2.0 ** -8 + 600 * E) * want.abs()).all(), (name, Y, want)


def test_infinite_and_missing_values():
    """+infinity and NaN through every activation."""
    z = T.tensor([float("inf"), float("nan")], dtype=T.bfloat16, device=DEV)
    for name in ref.ACTS:
        got, _ = values(z, name)
        for v in got.values():
            assert float(v[0]) == (1.0 if name == "sigmoid" else float("inf")) and T.isnan(v[1])
        d = slopes(z, name)
        assert float(d[0]) == (0.0 if name == "sigmoid" else 1.0) and T.isnan(d[1]) == (name != "none")
