"""The 8-bit feed-forward operators as they are called: one after another in a block and its
gradients, on streams and in graphs, with NaN and infinities, shared scales, empty sizes, and
matrices of more than 2^32 bytes."""
import math

import pytest

import nn8_reference as ref8
import nn_reference as ref
import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch
from test_parity_nn import E, U, check, gen, matrix, out_matrix, rounded, vec
from test_parity_nn8 import check_out, operand, out8, same_bits, untouched8

pytestmark = pytest.mark.gpu

T = torch()


# ------------------------------------------------------------------- a block
@pytest.mark.parametrize("M,K,N", [(1, 256, 600), (40, 200, 300), (300, 512, 1230), (1000, 640, 614)])
def test_block_and_its_gradients(M, K, N):
    """A pre-norm gated block in 8 bits from the norm to the down projection, its gradients by
    8-bit products of both orientations; each step against binary64 on what it was given."""
    g = gen(M + K)
    x, r = matrix(g, M, K, T.bfloat16, "packed")[0], matrix(g, M, K, T.bfloat16, "packed")[0]
    gamma = vec(g, K, 0.2, 1.0)
    wg, wu, wd = (matrix(g, a, b, T.bfloat16, "padded", 1 / math.sqrt(b))[0] for a, b in ((N, K), (N, K), (K, N)))
    (qg, _), (qu, _), (qd, qdt) = (sa.quantize8(w, 128, out="qt") for w in (wg, wu, wd))
    _, s, rstd, n8 = sa.rms_norm_fwd(x, gamma, R=r, out="srq")
    G, U_ = (T.empty(M, N, dtype=T.bfloat16, device=DEV) for _ in range(2))
    h, h8 = sa.glu8_fwd(n8, qg, qu, G=G, U=U_, out="hq")
    y, none = sa.linear8_fwd(h8, qd, R=s)
    assert none is None

    yn, rs = ref8.rms_fwd(s.double(), gamma.double(), 1e-5)
    ref8.check_codes(n8, yn, (K + 24) * E * yn.abs(), "norm")
    hr, th, gr, tg, ur, tu = ref8.glu8(n8, qg, qu, None, None, "silu")
    check_out_(h, hr, th, "h")
    check_out_(G, gr, tg, "g")
    check_out_(U_, ur, tu, "u")
    ref8.check_codes(h8, hr, th, "h8")
    yr, ty, _, _ = ref8.linear8(h8, qd, None, s, "none", exact=False)
    check_out_(y, yr, ty, "y")

    dy = matrix(g, M, K, T.bfloat16, "packed")[0]
    dy8, dyt = sa.quantize8(dy, out="qt")
    dh, _ = sa.linear8_fwd(dy8, qdt)
    dwd, _ = sa.linear8_fwd(dyt, sa.quantize8(h, 128, out="t")[1], out_dtype=T.float32)
    assert dh.shape == (M, N) and dwd.shape == (K, N) and dwd.dtype == T.float32
    z, tz = ref8.product(dy8, qdt, exact=False)
    check_out_(dh, z, tz, "dh")
    z, tz = ref8.product(dyt, sa.quantize8(h, 128, out="t")[1])
    check_out_(dwd, z, tz, "dWd")
    # and the formulas themselves: each product has two quantised operands, each off by at most 2^-4
    # of its value or 2^-10 of its block's scale, which is at most the largest value / 448; the
    # result's rounding and the products' cut are below 2^-6 of the sum of magnitudes
    def near(got, a, b):
        a, b = a.double(), b.double()
        small = 2.0 ** -18 * (a.abs().amax() * b.abs().sum(0) + b.abs().amax() * a.abs().sum(1, keepdim=True))
        assert ((got.double() - a @ b).abs() <= (2 * 2.0 ** -4 + 2.0 ** -6) * (a.abs() @ b.abs()) + 1.1 * small).all()
    near(dh, dy, wd)
    near(dwd, dy.t(), h)
    dn, _, _, _, _ = sa.glu_bwd(dh, yn.bfloat16(), wg, wu, G, U_)
    dx, dgamma = sa.rms_norm_bwd(dn, s, rstd, gamma, dR=dy)
    want, wgm = ref8.rms_bwd(dn.double(), s.double(), rstd.double(), gamma.double(), dy.double())
    t = (dn.double() * gamma.double()).abs()
    xn = (s.double() * rstd.double()[:, None]).abs()
    tol = rstd.double()[:, None] * (8 * E * t + xn * (t * xn).mean(1, keepdim=True) * (K + 16) * E) + 4 * E * dy.double().abs()
    check(dx, want, tol + rounded(want, T.bfloat16), "dx")
    check(dgamma, wgm, (M + 16) * E * (dn.double().abs() * xn).sum(0) + 1e-30, "dgamma")


def check_out_(got, want, tol, what):
    check(got, want, tol + rounded(want, got.dtype), what)


# ------------------------------------------- further sizes: every kernel and split
@pytest.mark.parametrize("M,N,K", [(1024, 4100, 700), (2100, 2050, 300), (300, 8200, 130), (600, 512, 9000),
                                   (130, 130, 16000), (17, 1000, 12000), (4096, 300, 513), (2048, 4096, 1100),
                                   (64, 16000, 70), (250, 200, 64)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("eight", [False, True])
def test_more_sizes(M, N, K, gated, eight):
    g = gen(M + N + K)
    X, W, V = operand(g, M, K, 1), operand(g, N, K, 128, 1 / math.sqrt(K)), operand(g, N, K, 128, 1 / math.sqrt(K))
    Y, buf = (None, None) if eight else out_matrix(M, N, T.bfloat16, "odd")
    Q, bufs = out8(M, N) if eight else (None, None)
    if gated:
        sa.glu8_fwd(X, W, V, act=sa.ACT_GELU, H=Y, Q=Q, out="")
        want, tol = ref8.glu8(X, W, V, None, None, "gelu", exact=eight)[:2]
    else:
        sa.linear8_fwd(X, W, act=sa.ACT_SILU, Y=Y, Q=Q, out="")
        want, tol = ref8.linear8(X, W, None, None, "silu", exact=eight)[:2]
    if eight:
        ref8.check_codes(Q, want, tol, "Q")
        assert untouched8(Q, bufs)
    else:
        check_out(Y, want, tol, T.bfloat16, buf, "Y")


@pytest.mark.parametrize("M,N,K,layout", [(8192, 4096, 200, "packed"), (5120, 6080, 84, "packed"), (8300, 4100, 130, "odd"),
                                          (8200, 8190, 128, "odd")])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_large_results_with_residual_and_preactivations(M, N, K, layout, dtype):
    """Results of 48 MB and more, which tiles store past the caches, on aligned and odd rows."""
    g = gen(M + N)
    t = {"bf16": T.bfloat16, "f16": T.float16, "f32": T.float32}[dtype]
    X, W = operand(g, M, K, 1), operand(g, N, K, 128, 1 / math.sqrt(K))
    bias, R = vec(g, N), matrix(g, M, N, t, layout)[0]
    (Y, buf), (Z, zbuf) = out_matrix(M, N, t, layout), out_matrix(M, N, T.bfloat16 if dtype == "f32" else t, layout)
    sa.linear8_fwd(X, W, bias, R, sa.ACT_RELU, Y=Y, Z=Z, out="")
    want, tol, z, tz = ref8.linear8(X, W, bias, R, "relu", exact=dtype == "f32")
    check_out(Y, want, tol, t, buf, "Y")
    check_out(Z, z, tz, Z.dtype, zbuf, "Z")


def test_empty_sums_and_sizes():
    g = gen(2)
    X, W = sa.matrix8(5, 0), sa.matrix8(200, 0, 128)
    bias, R = vec(g, 200), matrix(g, 5, 200, T.float16, "packed")[0]
    y, _ = sa.linear8_fwd(X, W, bias, R=R, act=sa.ACT_RELU)
    assert T.equal(y, (bias.clamp(min=0) + R.float()).half())
    X = sa.matrix8(100, 0)
    y, q = sa.linear8_fwd(X, W, bias, out="yq")
    assert T.equal(y, bias.bfloat16().expand(100, 200))
    c, s = ref8.quantise(bias.expand(100, 200), 1)
    assert T.equal(q.scales, s) and same_bits(q.codes, c)
    h, q = sa.glu8_fwd(X, W, W, bias, None, out="hq")
    assert (h == 0).all() and (q.codes.float() == 0).all()
    for M, N in ((0, 30), (30, 0)):
        X, W = sa.matrix8(M, 64), sa.matrix8(N, 64, 128)  # nothing reads what they hold
        y, q = sa.linear8_fwd(X, W, out="yq")
        assert y.shape == q.codes.shape == (M, N)
        h, q = sa.glu8_fwd(X, W, W, out="hq")
        assert h.shape == q.codes.shape == (M, N)


@pytest.mark.parametrize("M,N,K", [(3, 300, 400), (50, 300, 400), (400, 300, 400), (1500, 1300, 700)])
@pytest.mark.parametrize("out", ["y", "q"])
def test_nan_and_infinities_stay_in_their_rows(M, N, K, out):
    g = gen(M)
    X, W = operand(g, M, K, 1), operand(g, N, K, 128, 0.1)
    clean = sa.linear8_fwd(X, W, out=out)
    x, w = sa.matrix8(M, K), sa.Matrix8(W.codes, W.scales.clone())  # a clone has packed rows
    x.codes.view(T.uint8).copy_(X.codes.view(T.uint8))
    x.scales.copy_(X.scales)
    row = M // 2
    x.codes.view(T.uint8)[row, K - 1] = 0xff  # a NaN beside the padding
    dirty = sa.linear8_fwd(x, W, out=out)
    keep = T.arange(M, device=DEV) != row
    if out == "y":
        assert dirty[0][row].isnan().all() and T.equal(dirty[0][keep], clean[0][keep])
    else:
        assert dirty[1].codes.float()[row].isnan().all()
        assert same_bits(dirty[1].codes[keep], clean[1].codes[keep]) and T.equal(dirty[1].scales[keep], clean[1].scales[keep])
    w.scales[1, 0] = float("inf")  # neurons 128 .. 255
    dirty = sa.linear8_fwd(X, w)[0]
    other = T.cat([T.arange(128), T.arange(256, N)]).to(DEV)
    assert not dirty[:, 128:256].isfinite().any() and T.equal(dirty[:, other], sa.linear8_fwd(X, W)[0][:, other])


@pytest.mark.parametrize("M", [7, 60, 500])
def test_one_scale_for_many_blocks(M):
    """Scales with strides of 0: one for a whole matrix, or for each row."""
    g = gen(M)
    X, W = operand(g, M, 500, 1), operand(g, 300, 500, 128, 0.1)
    one, row = T.full((1, 1), 0.25, device=DEV), T.rand(M, 1, generator=g, device=DEV) + 0.5
    for sx, sw in ((one.expand(M, 4), one.expand(3, 4)), (row.expand(M, 4), W.scales), (X.scales, one.expand(3, 4))):
        got = sa.linear8_fwd(sa.Matrix8(X.codes, sx), sa.Matrix8(W.codes, sw))[0]
        assert T.equal(got, sa.linear8_fwd(sa.Matrix8(X.codes, sx.contiguous()), sa.Matrix8(W.codes, sw.contiguous()))[0])
    with pytest.raises(sa.StructAdmmError, match="share one"):
        sa.quantize8(matrix(g, M, 500, T.float16, "packed")[0], Q=sa.Matrix8(X.codes, one.expand(M, 4)), out="")


@pytest.mark.parametrize("M", [5, 90, 600])
@pytest.mark.parametrize("power", [-60, -64, 50])
def test_small_and_large_scales(M, power):
    """Both operands times 2^power: the scales' product rounds to binary32, below 2^-126 by
    up to 2^-150, once for the block's sum of products of codes."""
    g = gen(M + power)
    X, W = operand(g, M, 700, 1), operand(g, 300, 700, 128)
    X, W = (sa.Matrix8(m.codes, m.scales * 2.0 ** power) for m in (X, W))
    Y = sa.linear8_fwd(X, W, out_dtype=T.float32)[0]
    want, tol = ref8.product(X, W)
    tol = tol + 2.0 ** -150 * (X.codes.double().abs() @ W.codes.double().abs().t())
    # sums below 2^-126 are rounded by up to 2^-150 at each of their additions
    assert ((Y.double() - want).abs() <= tol + 64 * 2.0 ** -150).all()


# --------------------------------------------------------- streams and graphs
def chain(x, gamma, r, qg, qu, qd, bufs):
    s, n8, rstd, G, U_, h8, y, ws1, ws2 = bufs
    sa.rms_norm_fwd(x, gamma, R=r, S=s, Q=n8, rstd=rstd, out="")
    sa.glu8_fwd(n8, qg, qu, Q=h8, G=G, U=U_, ws=ws1, out="")
    sa.linear8_fwd(h8, qd, R=s, Y=y, ws=ws2, out="")


def chain_buffers(M, K, N):
    new = lambda *s: T.zeros(*s, dtype=T.bfloat16, device=DEV)
    return (new(M, K), sa.matrix8(M, K), T.zeros(M, device=DEV), new(M, N), new(M, N), sa.matrix8(M, N), new(M, K),
            T.empty(64 << 20, dtype=T.uint8, device=DEV), T.empty(64 << 20, dtype=T.uint8, device=DEV))


def chain_inputs(M, K, N, seed):
    g = gen(seed)
    w = [sa.quantize8(matrix(g, a, b, T.bfloat16, "packed", 1 / math.sqrt(b))[0], 128)[0] for a, b in ((N, K), (N, K), (K, N))]
    return matrix(g, M, K, T.bfloat16, "packed")[0], vec(g, K, 0.1, 1.0), matrix(g, M, K, T.bfloat16, "packed")[0], *w


@pytest.mark.parametrize("M,K,N", [(1, 512, 1229), (16, 1024, 2458), (300, 256, 700)])
def test_captured_and_replayed(M, K, N):
    a, b = chain_inputs(M, K, N, 1), chain_inputs(M, K, N, 2)
    x, r = a[0].clone(), a[2].clone()
    bufs = chain_buffers(M, K, N)
    chain(x, a[1], r, *a[3:], bufs)  # every kernel's first launch is before the capture
    first = bufs[6].clone()
    graph = T.cuda.CUDAGraph()
    with T.cuda.graph(graph):
        chain(x, a[1], r, *a[3:], bufs)
    for k in range(4):
        x.copy_((a, b)[k % 2][0])
        r.copy_((a, b)[k % 2][2])
        graph.replay()
        T.cuda.synchronize()
        other = chain_buffers(M, K, N)
        chain(x, a[1], r, *a[3:], other)
        assert T.equal(bufs[6], other[6]) and T.equal(bufs[3], other[3]) and T.equal(bufs[5].scales, other[5].scales)
        assert same_bits(bufs[5].codes, other[5].codes) and T.equal(bufs[6], first) == (k % 2 == 0)


def test_training_step_captured_beside_an_eager_graph():
    """The gradients of a captured step equal the eager ones, replay after replay, while torch
    keeps an eager graph of the same tensors."""
    g = gen(9)
    x, dy = matrix(g, 200, 300, T.bfloat16, "packed")[0], matrix(g, 200, 300, T.bfloat16, "packed")[0]
    gamma = vec(g, 300, 0.2, 1.0).requires_grad_()
    eager = (x.float() * gamma).square().sum()  # alive over the capture
    W = sa.quantize8(matrix(g, 400, 300, T.bfloat16, "packed")[0], 128, out="t")[1]
    dz = matrix(g, 200, 400, T.bfloat16, "packed")[0]

    def step():
        _, s, rstd, _ = sa.rms_norm_fwd(x, gamma.detach(), out="sr")
        q, qt = sa.quantize8(dz, out="qt")
        dn, _ = sa.linear8_fwd(q, W)
        dw, _ = sa.linear8_fwd(qt, sa.quantize8(x, 128, out="t")[1], out_dtype=T.float32)
        return *sa.rms_norm_bwd(dn, s, rstd, gamma.detach(), dR=dy), dw
    want = step()
    graph = T.cuda.CUDAGraph()
    with T.cuda.graph(graph):
        got = step()
    for _ in range(3):
        graph.replay()
        T.cuda.synchronize()
        assert all(T.equal(a, b) for a, b in zip(got, want))
        assert all(T.equal(a, b) for a, b in zip(step(), want))
    eager.backward()
    assert gamma.grad.isfinite().all()


def test_two_streams_at_once():
    streams = [T.cuda.Stream() for _ in range(2)]
    inputs = [chain_inputs(200, 512, 1300, i) for i in (3, 4)]
    want, bufs = [], [chain_buffers(200, 512, 1300) for _ in range(2)]
    for i in inputs:
        b = chain_buffers(200, 512, 1300)
        chain(*i, b)
        want.append(b[6].clone())
    T.cuda.synchronize()
    for _ in range(5):
        for s, i, b in zip(streams, inputs, bufs):
            with T.cuda.stream(s):
                chain(*i, b)
    T.cuda.synchronize()
    for b, w in zip(bufs, want):
        assert T.equal(b[6], w)


def test_results_do_not_depend_on_the_run():
    """No result depends on the order of workgroups."""
    g = gen(6)
    X, W = operand(g, 40, 9000, 1), operand(g, 500, 9000, 128, 0.02)
    first = sa.linear8_fwd(X, W, out="yq")
    for _ in range(5):
        again = sa.linear8_fwd(X, W, out="yq")
        assert T.equal(first[0], again[0]) and same_bits(first[1].codes, again[1].codes) and T.equal(first[1].scales, again[1].scales)


# ----------------------------------------------------------------- large ones
def test_codes_of_more_than_2_32_bytes():
    """Rows of X, of results and of quantised matrices past 2^32 bytes."""
    M, K, N, ld = (1 << 21) + 300, 200, 40, 2064
    codes = T.zeros(M * ld, dtype=T.uint8, device=DEV).view(M, ld)[:, :K]
    scales = T.full((2, M), 0.5, device=DEV).t()
    g = gen(4)
    W = operand(g, N, K, 128, 0.1)
    some = T.tensor([0, 1, (1 << 21) - 1, 1 << 21, M - 257, M - 1], device=DEV)
    part = operand(g, len(some), K, 1)
    codes[some] = part.codes.view(T.uint8)
    scales[some] = part.scales
    y, _ = sa.linear8_fwd(sa.Matrix8(codes, scales), W)
    want, tol, _, _ = ref8.linear8(part, W, None, None, "none", exact=False)
    check(y[some].contiguous(), want, tol + rounded(want, T.bfloat16), "Y")
    assert y.count_nonzero() == y[some].count_nonzero()
    del y, codes
    rows, cols = (1 << 20) + 130, 2200
    X = T.zeros(rows, cols, dtype=T.bfloat16, device=DEV)
    some = T.tensor([0, (1 << 20) - 1, 1 << 20, rows - 1], device=DEV)
    X[some] = T.randn(4, cols, generator=g, device=DEV).bfloat16()
    for norm in (False, True):
        Q = sa.matrix8(rows, cols)
        if norm:
            sa.rms_norm_fwd(X, Q=Q, out="")
            y, _ = ref8.rms_fwd(X[some].double(), None, 1e-5)
            ref8.check_codes(sa.Matrix8(Q.codes[some], Q.scales[some]), y, (cols + 24) * E * y.abs(), "Q")
        else:
            sa.quantize8(X, Q=Q, out="")
            q, s = ref8.quantise(X[some], 1)
            assert same_bits(Q.codes[some], q) and T.equal(Q.scales[some], s)
        assert (Q.scales[2:1000] == 2.0 ** -126).all() and (Q.codes.view(T.uint8)[2:1000] == 0).all()


def test_more_rows_than_a_launch_takes():
    rows, cols = (1 << 24) + 40, 8
    X = T.zeros(rows, cols, dtype=T.float16, device=DEV)
    some = T.tensor([0, 5, (1 << 22) + 3, 1 << 24, rows - 1], device=DEV)
    X[some] = T.randn(5, cols, generator=gen(1), device=DEV).half()
    codes, scales = T.zeros(rows, 16, dtype=T.uint8, device=DEV)[:, :cols], T.zeros(1, rows, device=DEV).t()
    q, s = ref8.quantise(X[some], 1)
    sa.quantize8(X, Q=sa.Matrix8(codes, scales), out="")
    assert same_bits(codes[some].view(T.float8_e4m3fn), q) and T.equal(scales[some], s) and (scales > 0).all()
    scales.zero_()
    Y, _, rstd, _ = sa.rms_norm_fwd(X, Q=sa.Matrix8(codes, scales), out="yr")
    y, r = ref8.rms_fwd(X[some].double(), None, 1e-5)
    check(Y[some], y, (cols + 24) * E * y.abs() + rounded(y, T.float16), "Y")
    assert (scales > 0).all() and (rstd > 0).all()
