"""From a pruned matrix to the block in 8 bits: projected, compacted and quantised as they are
called one after the other, then run and, for its weights' gradients, turned round.  Each
step against binary64 on what it was given."""
import os
import sys

import pytest

import nn8_reference as ref8
import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch
from test_parity_nn import E, check, gen, rounded
from test_parity_nn8 import same_bits

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu

T = torch()


@pytest.mark.parametrize("width,neurons,keep,rows", [(64, 256, 128, 64), (96, 250, 151, 70), (77, 300, 33, 1), (256, 1024, 614, 300),
                                                     (512, 4096, 2458, 16)])
def test_pruned_block_in_8_bits(width, neurons, keep, rows):
    import pruned_ffn
    g = gen(width + rows)
    randn = lambda *s: T.randn(*s, generator=g, device=DEV)
    Wgu, Wd = randn(neurons, 2 * width) / width ** 0.5, randn(width, neurons) / neurons ** 0.5
    gu, down, _ = pruned_ffn.prune(Wgu, Wd, keep)
    want = T.topk(Wgu.double().norm(dim=1), keep).indices.sort().values
    # halves of a compacted matrix's rows, and rows cut by the kept neurons, quantised where they lie
    parts = (gu[:, :width], Wgu[want, :width]), (gu[:, width:], Wgu[want, width:]), (down, Wd[:, want])
    q = [sa.quantize8(view, 128, out="qt") for view, _ in parts]
    for (m, mt), (_, w) in zip(q, parts):
        for got, v in ((m, w.bfloat16()), (mt, w.bfloat16().t())):
            codes, scales = ref8.quantise(v, 128)
            assert T.equal(got.scales, scales) and same_bits(got.codes, codes)
    (qg, _), (qu, _), (qd, qdt) = q

    x, dy = randn(rows, width).bfloat16(), randn(rows, width).bfloat16()
    n8 = sa.rms_norm_fwd(x, out="q")[3]
    yn, _ = ref8.rms_fwd(x.double(), None, 1e-5)
    ref8.check_codes(n8, yn, (width + 24) * E * yn.abs(), "norm")
    h, h8 = sa.glu8_fwd(n8, qg, qu, out="hq")
    hr, th = ref8.glu8(n8, qg, qu, None, None, "silu")[:2]
    check(h, hr, th + rounded(hr, T.bfloat16), "h")
    ref8.check_codes(h8, hr, th, "h8")
    y, _ = sa.linear8_fwd(h8, qd, R=x)
    yr, ty = ref8.linear8(h8, qd, None, x, "none", exact=False)[:2]
    check(y, yr, ty + rounded(yr, T.bfloat16), "y")
    # the down projection's gradients, the operands turned round
    dy8, dyt = sa.quantize8(dy, out="qt")
    dh, _ = sa.linear8_fwd(dy8, qdt)
    z, tz = ref8.product(dy8, qdt, exact=False)
    check(dh, z, tz + rounded(z, T.bfloat16), "dh")
    ht = sa.quantize8(h, 128, out="t")[1]
    dwd, _ = sa.linear8_fwd(dyt, ht, out_dtype=T.float32)
    z, tz = ref8.product(dyt, ht)
    check(dwd, z, tz + rounded(z, T.float32), "dWd")
    assert dwd.shape == down.shape
