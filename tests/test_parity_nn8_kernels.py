"""GPU parity of every kernel of the 8-bit products, by name, against the binary64 reference:
with bias, activation, residual, kept pre-activations and results on odd and aligned rows."""
import math

import pytest

import nn8_reference as ref8
import paper_1807_11091_amd as sa
from gpu_helpers import torch
from nn8_kernel_cases import CASES, case_id, kernel_of
from test_parity_nn import gen, matrix, out_matrix, vec
from test_parity_nn8 import check_out, operand, out8, same_bits, untouched8

pytestmark = pytest.mark.gpu

T = torch()


@pytest.mark.parametrize("dtype,layout", [("bf16", "odd"), ("f16", "packed")])
@pytest.mark.parametrize("case", CASES, ids=case_id)
def test_every_kernel(case, dtype, layout):
    (M, N, K), gated, out, f32, kernel, split = case
    p = sa.product8_plan(M, N, K, gated, out, f32)
    assert (kernel_of(p), p["split"] > 1) == (kernel, split)
    g, dt = gen(M + N + K), {"bf16": T.bfloat16, "f16": T.float16}[dtype]
    to, exact = T.float32 if f32 else dt, f32 or "q" in out
    X = operand(g, M, K, 1)
    W = [operand(g, N, K, 128, 1 / math.sqrt(K)) for _ in range(2 if gated else 1)]
    bias = vec(g, N)
    Y, ybuf = out_matrix(M, N, to, layout) if out != "q" else (None, None)
    Q, qbufs = out8(M, N) if "q" in out else (None, None)
    (Z, zbuf), (U, ubuf) = out_matrix(M, N, dt, layout), out_matrix(M, N, dt, layout)
    if gated:
        sa.glu8_fwd(X, *W, bias, None, H=Y, Q=Q, G=Z, U=U, out="")
        y, ty, z, tz, u, tu = ref8.glu8(X, *W, bias, None, "silu", exact)
        check_out(U, u, tu, dt, ubuf, "U")
    else:
        R = matrix(g, M, N, to, layout)[0]
        sa.linear8_fwd(X, *W, bias, R, sa.ACT_GELU, Y=Y, Z=Z, Q=Q, out="")
        y, ty, z, tz = ref8.linear8(X, *W, bias, R, "gelu", exact)
    check_out(Z, z, tz, dt, zbuf, "Z")
    if Y is not None:
        check_out(Y, y, ty, to, ybuf, "Y")
    if Q is not None:
        ref8.check_codes(Q, y, ty, "Q")
        assert untouched8(Q, qbufs)
    # results alone, in the residual's place
    if not gated:
        again = sa.linear8_fwd(X, *W, bias, R, sa.ACT_GELU, Y=R if Y is not None else None, out="q" if Q is not None else "")
        assert Y is None or T.equal(R, Y)
        assert Q is None or same_bits(again[1].codes, Q.codes) and T.equal(again[1].scales, Q.scales)
