"""What 16-bit results of the 8-bit products promise: with exact=True whole products and
binary32 sums, without it at most the stated cut, on operands made to show it.

The cut: of 8 neighbouring k each product is cut at 2^-13 of 2^(largest sum of two codes'
exponents among them), so a sum loses less than 8 * 2^-13 of that for each eight
(nn8_reference.product, exact=False).
"""
import math

import pytest

import nn8_reference as ref8
import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch
from test_parity_nn import E, check, gen, matrix, out_matrix, rounded, vec
from test_parity_nn8 import check_out, operand

pytestmark = pytest.mark.gpu

T = torch()

# one row, few, many; k in one part and in several; whole and cut blocks
SIZES = [(1, 40, 256), (1, 4096, 9000), (16, 300, 520), (40, 200, 1000), (64, 128, 4096), (130, 140, 1000), (300, 520, 264),
         (700, 640, 96), (1000, 1024, 1229), (1024, 4100, 700)]


def eight(codes, block, scale):
    """An operand with these codes and one scale."""
    m = sa.matrix8(*codes.shape, block)
    m.codes.view(T.uint8).copy_(codes.to(T.float8_e4m3fn).view(T.uint8))
    m.scales.fill_(scale)
    return m


def loud_rows(M, N, K, case):
    """x, w: in each eight of k one loud product and seven that the cut loses ("loud"), or two
    loud ones that cancel and six that remain ("cancel")."""
    x, w = T.full((M, K), 15 * 2.0 ** -9, device=DEV), T.ones(N, K, device=DEV)
    x[:, ::8] = 256.0
    if case == "cancel":
        x = T.full((M, K), 2.0 ** -7, device=DEV)
        w = T.full((N, K), 2.0 ** -7, device=DEV)
        x[:, ::8], w[:, ::8] = 1.0, 1.0
        x[:, 1::8], w[:, 1::8] = 1.0, -1.0
    return x, w


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("case", ["loud", "cancel"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_loud_products_beside_small_ones(M, N, K, case, dtype):
    dt = {"bf16": T.bfloat16, "f16": T.float16}[dtype]
    x, w = loud_rows(M, N, K, case)
    X, W = eight(x, 1, 2.0 ** -6), eight(w, 128, 1.0)
    want = ref8.product(X, W)[0]
    assert T.equal(want, x.double() @ w.double().t() * 2.0 ** -6)  # every value is a code
    assert want.abs().max() < 60000
    for exact in (True, False):
        y, _ = sa.linear8_fwd(X, W, out_dtype=dt, exact=exact)
        bound = ref8.product(X, W, exact)[1]
        check(y, want, bound + rounded(want, dt), exact)
        h, _ = sa.glu8_fwd(X, W, W, act=sa.ACT_NONE, dtype=T.bfloat16, out="h", exact=exact)
        check(h, want * want, 2 * bound * want.abs() + bound * bound + 2 * E * want * want + rounded(want * want, T.bfloat16), exact)


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_exact_products_with_16_bit_results(M, N, K, dtype):
    """The binary32 result, rounded: every output and addend, gated and not."""
    dt, g = {"bf16": T.bfloat16, "f16": T.float16}[dtype], gen(M + N + K)
    X, W, V = operand(g, M, K, 1), operand(g, N, K, 128, 1 / math.sqrt(K)), operand(g, N, K, 128, 1 / math.sqrt(K))
    bias, R = vec(g, N), matrix(g, M, N, dt, "odd")[0]
    plain, _ = sa.linear8_fwd(X, W, bias, act=sa.ACT_SILU, out_dtype=T.float32)
    y, _ = sa.linear8_fwd(X, W, bias, act=sa.ACT_SILU, out_dtype=dt, exact=True)
    assert T.equal(y, plain.to(dt))  # the same kernel and split
    (Y, buf), (Z, zbuf) = out_matrix(M, N, dt, "odd"), out_matrix(M, N, dt, "padded")
    sa.linear8_fwd(X, W, bias, R, sa.ACT_GELU, Y=Y, Z=Z, out="", exact=True)
    want, tol, z, tz = ref8.linear8(X, W, bias, R, "gelu")
    check_out(Y, want, tol, dt, buf, "Y")
    check_out(Z, z, tz, dt, zbuf, "Z")
    (H, hbuf), (G, gbuf), (U, ubuf) = (out_matrix(M, N, dt, "packed") for _ in range(3))
    sa.glu8_fwd(X, W, V, bias, None, H=H, G=G, U=U, out="", exact=True)
    h, th, gg, tg, u, tu = ref8.glu8(X, W, V, bias, None, "silu")
    check_out(H, h, th, dt, hbuf, "H")
    check_out(G, gg, tg, dt, gbuf, "G")
    check_out(U, u, tu, dt, ubuf, "U")
