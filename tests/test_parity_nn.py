"""GPU parity of the feed-forward operators against the binary64 reference.

Tolerances follow from the arithmetic.  u is the unit roundoff of a type
(2^-8 bfloat16, 2^-11 binary16, 2^-24 binary32) and e = 2^-24.  A result rounded
once from binary32 is off by u |y|; a binary32 sum of n products, in any order,
by at most n e times the sum of the products' magnitudes (and each product of
16-bit operands is exact); bias, activation and residual add a few e of their
own operands, the exponential of z about (2 + |z|) e of its value.  Where an
operand of a product is itself rounded (dz, dg, du), u times the sum of the
magnitudes is added.  All bounds are per element.
"""
import math

import pytest

import nn_reference as ref
import paper_1807_11091_amd as sa
from gpu_helpers import DEV, torch

pytestmark = pytest.mark.gpu

T = torch()
TYPES = {"bf16": T.bfloat16, "f16": T.float16, "f32": T.float32}
U = {T.bfloat16: 2.0 ** -8, T.float16: 2.0 ** -11, T.float32: 2.0 ** -24}
TINY = {T.bfloat16: 2.0 ** -126, T.float16: 2.0 ** -24, T.float32: 2.0 ** -126}
E = 2.0 ** -24


def gen(seed):
    return T.Generator(device=DEV).manual_seed(seed)


def matrix(g, rows, cols, dtype, pitch, scale=1.0, fill=None):
    """A [rows, cols] matrix of normals inside a buffer of NaN: "packed" rows,
    rows "padded" to 64, or an "odd" pitch and start."""
    ld = {"packed": cols, "padded": (cols + 63) // 64 * 64, "odd": (cols + 2) // 2 * 2 + 1}[pitch]
    at = 3 if pitch == "odd" else 0
    buf = T.full((at + rows * ld + 64,), float("nan"), dtype=dtype, device=DEV)
    m = buf[at:at + rows * ld].view(rows, ld)[:, :cols]
    m.copy_(T.randn(rows, cols, generator=g, device=DEV) * scale if fill is None else T.full((rows, cols), fill))
    return m, buf


def out_matrix(rows, cols, dtype, pitch):
    return matrix(gen(0), rows, cols, dtype, pitch, fill=float("nan"))


def padding_untouched(m, buf):
    """Everything of buf outside m still holds NaN."""
    n = T.isnan(buf.float()).sum().item() - T.isnan(m.float()).sum().item()
    return n == buf.numel() - m.numel()


def vec(g, n, scale=0.1, shift=0.0):
    return T.randn(n, generator=g, device=DEV) * scale + shift


def check(got, want, tol, what):
    got = got.double()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((got - want).abs().max()), float(tol.min()))


def rounded(y, dtype):
    return U[dtype] * y.abs() + TINY[dtype]


PITCHES = ["packed", "padded", "odd"]

# ---------------------------------------------------------------- layer norm
LN_SIZES = [(1, 1), (1, 64), (3, 7), (5, 8), (2, 63), (130, 512), (33, 513), (9, 1000), (6, 1025), (4, 2047), (7, 2458),
            (3, 4096), (5, 4099), (3, 8192), (2, 8200), (2, 16385), (3, 32768), (2, 32771), (700, 96), (3000, 130)]


@pytest.mark.parametrize("rows,cols", LN_SIZES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("pitch", PITCHES)
def test_layer_norm(rows, cols, dtype, pitch):
    dt, g, eps = TYPES[dtype], gen(rows * 7 + cols), 1e-5
    X, _ = matrix(g, rows, cols, dt, pitch, 2.0)
    X.add_(0.5)
    gamma, beta = (None, None) if (rows + cols) % 3 == 0 else (vec(g, cols, 0.2, 1.0), vec(g, cols))
    Y, buf = out_matrix(rows, cols, dt, pitch)
    _, mean, rstd = sa.layer_norm_fwd(X, gamma, beta, eps, Y=Y)
    x = X.double()
    d = lambda t: None if t is None else t.double()
    y, m, s = ref.ln_fwd(x, d(gamma), d(beta), eps)
    mag = x.abs().mean(1)
    # mean: a sum of cols values; rstd: a sum of squares of differences, each off by the mean's error
    em = (cols + 8) * E * mag
    check(mean, m, em + 1e-30, "mean")
    er = s * ((cols + 16) * E + em * s * math.sqrt(cols) * 2 + (em * s) ** 2)
    check(rstd, s, er, "rstd")
    gm = 1.0 if gamma is None else gamma.double().abs()
    b = 0.0 if beta is None else beta.double().abs()
    xn = (x - m[:, None]).abs() * s[:, None]
    tol = gm * (xn * (er / s)[:, None] + (em * s)[:, None] * 1.01 + 8 * E * xn) + 4 * E * b
    check(Y, y, tol * 1.01 + rounded(y, dt), "Y")
    assert padding_untouched(Y, buf)
    no_stats = sa.layer_norm_fwd(X, gamma, beta, eps, stats=False)
    assert no_stats[1] is None and T.equal(no_stats[0], Y)
    in_place = X.clone()
    sa.layer_norm_fwd(in_place, gamma, beta, eps, Y=in_place)
    assert T.equal(in_place, Y)

    dY, _ = matrix(g, rows, cols, dt, pitch)
    dR = matrix(g, rows, cols, dt, pitch)[0] if cols % 2 else None
    dX, buf = out_matrix(rows, cols, dt, pitch)
    dg, db = T.full((cols,), 7.0, device=DEV), T.full((cols,), 7.0, device=DEV)
    sa.layer_norm_bwd(dY, X, mean, rstd, gamma, dR=dR, dX=dX, dgamma=dg, dbeta=db)
    dy, m, s = dY.double(), mean.double(), rstd.double()
    rx, rg, rb = ref.ln_bwd(dy, x, m, s, d(gamma), d(dR))
    xn = (x - m[:, None]).abs() * s[:, None]
    t = dy.abs() * gm
    # each xn and t is off by a few e; two row sums of cols terms
    tol = s[:, None] * (t * 8 * E + (t.mean(1, keepdim=True) + xn * (t * xn).mean(1, keepdim=True)) * (cols + 16) * E)
    r = 0.0 if dR is None else dR.double().abs()
    check(dX, rx, tol * 1.01 + 4 * E * r + rounded(rx, dt), "dX")
    assert padding_untouched(dX, buf)
    check(dg, rg, (rows + 16) * E * (dy.abs() * xn).sum(0) + 1e-30, "dgamma")
    check(db, rb, (rows + 16) * E * dy.abs().sum(0) + 1e-30, "dbeta")
    only = sa.layer_norm_bwd(dY, X, mean, rstd, gamma, dR=dR, params=False)
    assert only[1] is None and T.equal(only[0], dX)
    over = dY.clone()  # dX in dY's place
    dg2 = sa.layer_norm_bwd(over, X, mean, rstd, gamma, dR=dR, dX=over)[1]
    assert T.equal(over, dX) and T.equal(dg2, dg)


def test_layer_norm_equal_values_and_no_rows():
    X = T.full((3, 100), 2.5, dtype=T.bfloat16, device=DEV)
    beta = vec(gen(1), 100)
    Y, mean, rstd = sa.layer_norm_fwd(X, None, beta, 1e-5)
    assert T.equal(Y, beta.to(T.bfloat16).expand(3, 100)) and (mean == 2.5).all()
    assert ((rstd - 1e-5 ** -0.5).abs() <= 4 * E * 1e-5 ** -0.5).all()
    none = X[:0]
    Y, mean, rstd = sa.layer_norm_fwd(none, None, beta)
    assert Y.shape == (0, 100)
    dX, dg, db = sa.layer_norm_bwd(none, none, mean, rstd)
    assert (dg == 0).all() and (db == 0).all()


def test_layer_norm_keeps_rows_apart():
    """A row with an infinity or NaN spoils itself and the column sums only."""
    g = gen(5)
    X = T.randn(9, 300, generator=g, device=DEV).half()
    clean = sa.layer_norm_fwd(X)[0]
    X[4, 17], X[6, 299] = float("inf"), float("nan")
    Y = sa.layer_norm_fwd(X)[0]
    rows = T.tensor([0, 1, 2, 3, 5, 7, 8], device=DEV)
    assert T.equal(Y[rows], clean[rows]) and T.isnan(Y[6]).all()


# -------------------------------------------------------------------- linear
SIZES = [(1, 1, 1), (1, 64, 64), (1, 1024, 2458), (2, 5, 7), (3, 33, 1229), (7, 130, 96), (8, 256, 640), (13, 100, 100),
         (16, 1000, 512), (17, 65, 130), (33, 200, 64), (64, 64, 64), (65, 127, 257), (96, 640, 72), (128, 128, 128),
         (130, 260, 1000), (256, 512, 320), (300, 77, 1229), (257, 1030, 200), (520, 776, 136), (1000, 24, 40),
         (40, 2000, 31)]
KINDS = [("bf16", "packed"), ("bf16", "padded"), ("f16", "packed"), ("f16", "odd"), ("bf16", "odd")]


def act_tol(z, y):
    """Rounding of an activation's value or slope, given |z| and bounds of their size."""
    return (8 + 4 * z.abs().clamp(max=100.0)) * E * (y.abs() + z.abs() * E + 1e-30)


@pytest.mark.parametrize("size", range(len(SIZES)))
@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_linear(size, kind):
    (M, N, K), (dtype, pitch) = SIZES[size], KINDS[kind]
    dt, g = TYPES[dtype], gen(size * 10 + kind)
    a = ref.ACTS[(size + kind) % 6]
    X, _ = matrix(g, M, K, dt, pitch)
    W, _ = matrix(g, N, K, dt, pitch, 1 / math.sqrt(K))
    bias = vec(g, N) if size % 2 else None
    out = T.float32 if (size + kind) % 4 == 3 else dt
    R = matrix(g, M, N, out, pitch)[0] if size % 3 else None
    Y, ybuf = out_matrix(M, N, out, pitch)
    Z, zbuf = out_matrix(M, N, dt, pitch)
    sa.linear_fwd(X, W, bias, R=R, act=sa.ACTS[a], Y=Y, Z=Z)
    d = lambda t: None if t is None else t.double()
    x, w = X.double(), W.double()
    y, z = ref.linear_fwd(x, w, d(bias), d(R), a)
    mag = x.abs() @ w.abs().t()
    ez = (K + 4) * E * (mag + (0.0 if bias is None else bias.double().abs()))
    check(Z, z, ez + rounded(z, dt), "Z")
    # no slope exceeds 1.13
    er = 1.13 * ez + act_tol(z, z.abs() + ref.act(a, z).abs()) + 4 * E * (0.0 if R is None else R.double().abs())
    check(Y, y, er + rounded(y, out), "Y")
    assert padding_untouched(Y, ybuf) and padding_untouched(Z, zbuf)
    assert T.equal(sa.linear_fwd(X, W, bias, R=R, act=sa.ACTS[a], out_dtype=out), Y)
    if R is not None:
        sa.linear_fwd(X, W, bias, R=R, act=sa.ACTS[a], Y=R)
        assert T.equal(R, Y)

    dY, _ = matrix(g, M, N, dt, pitch)
    dwt = dt if kind % 2 else T.float32
    dX, xbuf = out_matrix(M, K, dt, pitch)
    dW, wbuf = out_matrix(N, K, dwt, pitch)
    db = T.full((N,), 7.0, device=DEV)
    sa.linear_bwd(dY, X, W, Z=Z, act=sa.ACTS[a], dX=dX, dW=dW, dbias=db)
    dy, zz = dY.double(), Z.double()
    rx, rw, rb = ref.linear_bwd(dy, zz, x, w, a)
    dz = dy.abs() if a == "none" else (dy * ref.dact(a, zz)).abs()
    ed = T.zeros_like(dz) if a == "none" else dy.abs() * act_tol(zz, 1 + zz.abs())
    rd = ed if a == "none" else ed + U[dt] * dz + TINY[dt]
    check(dX, rx, (N + 4) * E * (dz @ w.abs()) + 1.01 * (rd @ w.abs()) + rounded(rx, dt), "dX")
    check(dW, rw, (M + 4) * E * (dz.t() @ x.abs()) + 1.01 * (rd.t() @ x.abs()) + rounded(rw, dwt), "dW")
    check(db, rb, (M + 4) * E * dz.sum(0) + 1.01 * ed.sum(0) + 1e-30, "dbias")
    assert padding_untouched(dX, xbuf) and padding_untouched(dW, wbuf)
    # each gradient alone
    for grads, i, want in (("x", 0, dX), ("w", 1, dW), ("b", 2, db)):
        alone = sa.linear_bwd(dY, X, W, Z=Z, act=sa.ACTS[a], grads=grads, dw_dtype=dwt)
        assert T.equal(alone[i], want) and sum(t is not None for t in alone) == 1


# --------------------------------------------------------------------- gated
@pytest.mark.parametrize("size", range(len(SIZES)))
@pytest.mark.parametrize("kind", range(len(KINDS)))
def test_glu(size, kind):
    (M, N, K), (dtype, pitch) = SIZES[size], KINDS[kind]
    dt, g = TYPES[dtype], gen(1000 + size * 10 + kind)
    a = ref.ACTS[(size + kind) % 6]
    X, _ = matrix(g, M, K, dt, pitch)
    if size % 2:  # a neuron's two rows side by side
        Wgu, _ = matrix(g, N, 2 * K, dt, pitch, 1 / math.sqrt(K))
        Wg, Wu = Wgu[:, :K], Wgu[:, K:]
    else:
        Wg, Wu = (matrix(g, N, K, dt, pitch, 1 / math.sqrt(K))[0] for _ in range(2))
    bg, bu = (vec(g, N) if size % 3 else None), (vec(g, N) if size % 3 == 1 else None)
    (H, hb), (G, gb), (Uo, ub) = (out_matrix(M, N, dt, pitch) for _ in range(3))
    sa.glu_fwd(X, Wg, Wu, bg, bu, act=sa.ACTS[a], H=H, G=G, U=Uo)
    d = lambda t: None if t is None else t.double()
    x, wg, wu = X.double(), Wg.double(), Wu.double()
    h, gg, uu = ref.glu_fwd(x, wg, wu, d(bg), d(bu), a)
    eg = (K + 4) * E * (x.abs() @ wg.abs().t() + (0.0 if bg is None else bg.double().abs()))
    eu = (K + 4) * E * (x.abs() @ wu.abs().t() + (0.0 if bu is None else bu.double().abs()))
    check(G, gg, eg + rounded(gg, dt), "G")
    check(Uo, uu, eu + rounded(uu, dt), "U")
    va = ref.act(a, gg).abs()
    ea = 1.13 * eg + act_tol(gg, gg.abs() + va)
    check(H, h, 1.01 * (ea * (uu.abs() + eu) + va * eu) + 4 * E * h.abs() + rounded(h, dt), "H")
    assert padding_untouched(H, hb) and padding_untouched(G, gb) and padding_untouched(Uo, ub)
    assert T.equal(sa.glu_fwd(X, Wg, Wu, bg, bu, act=sa.ACTS[a]), H)

    dH, _ = matrix(g, M, N, dt, pitch)
    dwt = dt if kind % 2 else T.float32
    dX, xbuf = out_matrix(M, K, dt, pitch)
    dWg, dWu = (out_matrix(N, K, dwt, pitch)[0] for _ in range(2))
    dbg, dbu = T.full((N,), 7.0, device=DEV), T.full((N,), 7.0, device=DEV)
    sa.glu_bwd(dH, X, Wg, Wu, G, Uo, act=sa.ACTS[a], dX=dX, dWg=dWg, dWu=dWu, dbg=dbg, dbu=dbu)
    dh, gg, uu = dH.double(), G.double(), Uo.double()
    rx, rwg, rwu, rbg, rbu = ref.glu_bwd(dh, gg, uu, x, wg, wu, a)
    dg, du = (dh * uu * ref.dact(a, gg)).abs(), (dh * ref.act(a, gg)).abs()
    sg = (dh * uu).abs() * act_tol(gg, 1 + gg.abs()) + 4 * E * dg
    su = dh.abs() * act_tol(gg, gg.abs() + ref.act(a, gg).abs()) + 4 * E * du
    rg, ru = sg + U[dt] * dg + TINY[dt], su + U[dt] * du + TINY[dt]
    check(dX, rx, (2 * N + 4) * E * (dg @ wg.abs() + du @ wu.abs()) + 1.01 * (rg @ wg.abs() + ru @ wu.abs())
          + rounded(rx, dt), "dX")
    check(dWg, rwg, (M + 4) * E * (dg.t() @ x.abs()) + 1.01 * (rg.t() @ x.abs()) + rounded(rwg, dwt), "dWg")
    check(dWu, rwu, (M + 4) * E * (du.t() @ x.abs()) + 1.01 * (ru.t() @ x.abs()) + rounded(rwu, dwt), "dWu")
    check(dbg, rbg, (M + 4) * E * dg.sum(0) + 1.01 * sg.sum(0) + 1e-30, "dbg")
    check(dbu, rbu, (M + 4) * E * du.sum(0) + 1.01 * su.sum(0) + 1e-30, "dbu")
    assert padding_untouched(dX, xbuf)
    pair = sa.glu_bwd(dH, X, Wg, Wu, G, Uo, act=sa.ACTS[a], grads="w", dw_dtype=dwt)  # one [N, 2K] matrix
    assert T.equal(pair[1], dWg) and T.equal(pair[2], dWu) and pair[0] is None and pair[3] is None
    assert T.equal(sa.glu_bwd(dH, X, Wg, Wu, G, Uo, act=sa.ACTS[a], grads="x")[0], dX)


# Products large enough for every tile shape, against a binary64 product on the GPU.
LARGE = [(1, 4096, 9830), (4, 9830, 1024), (16, 2458, 4096), (48, 4096, 2458), (100, 4915, 1024), (512, 2458, 1024),
         (777, 1229, 2000), (1024, 4096, 1024), (2048, 1024, 4915), (4100, 2458, 640), (3000, 2458, 2458)]


@pytest.mark.parametrize("M,N,K", LARGE)
@pytest.mark.parametrize("dtype,pitch", [("bf16", "padded"), ("f16", "packed")])
def test_large_products(M, N, K, dtype, pitch):
    dt, g = TYPES[dtype], gen(M + N + K)
    X, W = matrix(g, M, K, dt, pitch)[0], matrix(g, N, K, dt, pitch, 1 / math.sqrt(K))[0]
    V = matrix(g, N, K, dt, pitch, 1 / math.sqrt(K))[0]
    R, dY = matrix(g, M, N, dt, pitch)[0], matrix(g, M, N, dt, pitch)[0]
    bias = vec(g, N)
    x, w, v, dy = X.double(), W.double(), V.double(), dY.double()
    z = x @ w.t() + bias.double()
    ez = (K + 4) * E * (x.abs() @ w.abs().t() + bias.double().abs())
    Y = sa.linear_fwd(X, W, bias, R=R)
    y = z + R.double()
    check(Y, y, ez + 4 * E * R.double().abs() + rounded(y, dt), "Y")
    dX, dW, db = sa.linear_bwd(dY, X, W, grads="xwb")
    rx, rw = dy @ w, dy.t() @ x
    check(dX, rx, (N + 4) * E * (dy.abs() @ w.abs()) + rounded(rx, dt), "dX")
    check(dW, rw, (M + 4) * E * (dy.abs().t() @ x.abs()) + rounded(rw, T.float32), "dW")
    check(db, dy.sum(0), (M + 4) * E * dy.abs().sum(0), "dbias")
    G, Uo = T.empty_like(dY), T.empty_like(dY)
    H = sa.glu_fwd(X, W, V, bias, None, G=G, U=Uo)
    u = x @ v.t()
    eu = (K + 4) * E * (x.abs() @ v.abs().t())
    h = ref.act("silu", z) * u
    check(G, z, ez + rounded(z, dt), "G")
    check(Uo, u, eu + rounded(u, dt), "U")
    va = ref.act("silu", z).abs()
    ea = 1.13 * ez + act_tol(z, z.abs() + va)
    check(H, h, 1.01 * (ea * (u.abs() + eu) + va * eu) + 4 * E * h.abs() + rounded(h, dt), "H")
    dX, dWg, dWu, _, _ = sa.glu_bwd(dY, X, W, V, G, Uo, dw_dtype=dt)
    gg, uu = G.double(), Uo.double()
    rx, rwg, rwu, _, _ = ref.glu_bwd(dy, gg, uu, x, w, v, "silu")
    dg, du = (dy * uu * ref.dact("silu", gg)).abs(), (dy * ref.act("silu", gg)).abs()
    rg = (dy * uu).abs() * act_tol(gg, 1 + gg.abs()) + 4 * E * dg + U[dt] * dg + TINY[dt]
    ru = dy.abs() * act_tol(gg, 2 * gg.abs()) + 4 * E * du + U[dt] * du + TINY[dt]
    check(dX, rx, (2 * N + 4) * E * (dg @ w.abs() + du @ v.abs()) + 1.01 * (rg @ w.abs() + ru @ v.abs())
          + rounded(rx, dt), "dX")
    check(dWg, rwg, (M + 4) * E * (dg.t() @ x.abs()) + 1.01 * (rg.t() @ x.abs()) + rounded(rwg, dt), "dWg")
    check(dWu, rwu, (M + 4) * E * (du.t() @ x.abs()) + 1.01 * (ru.t() @ x.abs()) + rounded(rwu, dt), "dWu")


# More than one round of the largest tiles and part of another: run in two pieces.
@pytest.mark.parametrize("M,N,K,dtype,pitch", [(4400, 3900, 2000, "bf16", "padded"), (2500, 4096, 2048, "f16", "packed"),
                                               (7680, 2430, 1664, "f16", "packed"), (6001, 5001, 4001, "bf16", "packed")])
def test_products_in_pieces(M, N, K, dtype, pitch):
    test_large_products(M, N, K, dtype, pitch)


# ------------------------------------------------------- empty sizes, specials
def test_empty_sizes():
    bf = dict(dtype=T.bfloat16, device=DEV)
    bias = vec(gen(3), 5)
    R = T.randn(4, 5, device=DEV).bfloat16()
    X, W = T.empty(4, 0, **bf), T.empty(5, 0, **bf)
    want = (ref.act("gelu", bias.double()) + R.double()).bfloat16()
    got = sa.linear_fwd(X, W, bias, R=R, act=sa.ACT_GELU)  # every neuron pruned: the sum is empty
    assert T.allclose(got.double(), want.double(), rtol=2 ** -7, atol=1e-6)
    assert (sa.glu_fwd(X, W, W.clone()) == 0).all()
    assert sa.linear_fwd(T.empty(0, 8, **bf), T.empty(5, 8, **bf)).shape == (0, 5)
    dX, dW, db = sa.linear_bwd(T.empty(0, 5, **bf), T.empty(0, 8, **bf), T.empty(5, 8, **bf), grads="xwb")
    assert dX.shape == (0, 8) and (dW == 0).all() and (db == 0).all()
    dX, dW, _ = sa.linear_bwd(T.empty(4, 0, **bf), T.empty(4, 8, **bf), T.empty(0, 8, **bf))
    assert (dX == 0).all() and dW.shape == (0, 8)
    e = T.empty(0, 5, **bf)
    dX, dWg, dWu, dbg, dbu = sa.glu_bwd(e, T.empty(0, 8, **bf), T.empty(5, 8, **bf), T.empty(5, 8, **bf), e.clone(),
                                        e.clone(), grads="xwb")
    assert (dWg == 0).all() and (dWu == 0).all() and (dbg == 0).all() and (dbu == 0).all()


@pytest.mark.parametrize("M,N,K", [(5, 70, 100), (70, 140, 1000), (300, 300, 200)])
def test_special_values_stay_in_their_row_and_column(M, N, K):
    g = gen(77)
    X, W = T.randn(M, K, generator=g, device=DEV).half(), T.randn(N, K, generator=g, device=DEV).half()
    V = T.randn(N, K, generator=g, device=DEV).half()
    clean, gated = sa.linear_fwd(X, W), sa.glu_fwd(X, W, V)
    X[2, K - 1], W[N - 1, 0], W[3, 5] = float("nan"), float("nan"), float("inf")
    Y, H = sa.linear_fwd(X, W), sa.glu_fwd(X, W, V)
    keep = T.ones(M, N, dtype=T.bool, device=DEV)
    keep[2], keep[:, N - 1], keep[:, 3] = False, False, False
    assert T.equal(Y[keep], clean[keep]) and T.equal(H[keep], gated[keep])
    assert T.isnan(Y[2]).all() and T.isnan(Y[:, N - 1]).all()
    assert not T.isfinite(Y[:, 3]).any()


def test_far_activations():
    """Pre-activations of the type's largest size: values and slopes at their limits."""
    for dt in (T.bfloat16, T.float16):
        big = T.finfo(dt).max
        X = T.tensor([[1.0], [-1.0], [0.0]], dtype=dt, device=DEV)
        W = T.tensor([[big], [big / 4], [100.0], [20.0]], dtype=dt, device=DEV)
        for a in ref.ACTS:
            Z = T.empty(3, 4, dtype=dt, device=DEV)
            Y = sa.linear_fwd(X, W, act=sa.ACTS[a], Z=Z, out_dtype=T.float32)
            want = {"none": X.float() @ W.float().t(), "sigmoid": T.sigmoid(X.float() @ W.float().t())}.get(
                a, T.clamp(X.float() @ W.float().t(), min=0))
            assert T.allclose(Y, want, rtol=1e-5, atol=1e-6), (a, Y)
            db = sa.linear_bwd(T.ones_like(Z), X, W, Z=Z, act=sa.ACTS[a], grads="b")[2]
            slope = {"none": 3.0, "sigmoid": 0.25, "relu": 1.0}.get(a, 1.5)
            assert T.allclose(db, T.full((4,), slope, device=DEV), rtol=1e-5, atol=1e-6), (a, db)


# ----------------------------------------------- streams, repeats, differences
def test_repeats_are_bitwise_equal_and_streams_are_kept():
    g = gen(9)
    X, W, V = (T.randn(s, generator=g, device=DEV).bfloat16() for s in ((333, 1229), (515, 1229), (515, 1229)))
    dY = T.randn(333, 515, generator=g, device=DEV).bfloat16()

    def all_of(stream=None):
        G, Uo = T.empty_like(dY), T.empty_like(dY)
        H = sa.glu_fwd(X, W, V, G=G, U=Uo, stream=stream)
        if stream is not None:
            T.cuda.current_stream().wait_stream(stream)
            stream.wait_stream(T.cuda.current_stream())
        out = [H, G, Uo, *sa.linear_bwd(dY, X, W, grads="xwb", stream=stream),
               *sa.glu_bwd(dY, X, W, V, G, Uo, grads="xwb", stream=stream),
               *sa.layer_norm_fwd(X, stream=stream)]
        return out

    first = all_of()
    T.cuda.synchronize()
    s = T.cuda.Stream()
    s.wait_stream(T.cuda.current_stream())
    second = all_of(s)
    T.cuda.synchronize()
    for a, b in zip(first, second):
        assert T.equal(a, b)


def test_graph_replays():
    """Every operator inside a captured graph, replayed with new inputs."""
    g = gen(11)
    X = T.randn(40, 520, generator=g, device=DEV).bfloat16()
    Wg, Wu = (T.randn(300, 520, generator=g, device=DEV).bfloat16() * 0.05 for _ in range(2))
    Wd = T.randn(520, 300, generator=g, device=DEV).bfloat16() * 0.05

    def step():
        n, mean, rstd = sa.layer_norm_fwd(X)
        G, Uo = T.empty(40, 300, dtype=T.bfloat16, device=DEV), T.empty(40, 300, dtype=T.bfloat16, device=DEV)
        H = sa.glu_fwd(n, Wg, Wu, G=G, U=Uo)
        Y = sa.linear_fwd(H, Wd, R=X)
        dH, dWd, _ = sa.linear_bwd(Y, H, Wd)
        dn, dWg, dWu, _, _ = sa.glu_bwd(dH, n, Wg, Wu, G, Uo)
        return [Y, dWd, dWg, dWu, *sa.layer_norm_bwd(dn, X, mean, rstd, dR=Y)]

    step()
    T.cuda.synchronize()
    graph = T.cuda.CUDAGraph()
    with T.cuda.graph(graph):
        outs = step()
    for i in range(4):
        X.copy_(T.randn(40, 520, generator=g, device=DEV))
        graph.replay()
        T.cuda.synchronize()
        for a, b in zip(outs, step()):
            assert T.equal(a, b), i
        T.cuda.synchronize()


@pytest.mark.parametrize("a", ["silu", "gelu", "gelu_tanh", "sigmoid"])
def test_gradients_against_differences(a):
    """(L(X + hV) - L(X - hV)) / 2h of the kernels' own forward pass in binary32
    against <dX, V>.  X is a multiple of 2^-6 below 2 and hV of 2^-5, so both
    points are exact in binary16.  The forward sums are off by K e of their
    magnitudes; the difference formula by h^2/6 times the third derivative along
    V, below 2 |V W^T|^3 for these activations; dX by u of its own rounding and
    that of dz; Z of Y(X) by u |Z|, times a second derivative below 1."""
    g = gen(21)
    M, N, K, h = 24, 40, 48, 2.0 ** -5
    X = (T.randint(-64, 65, (M, K), generator=g, device=DEV) * 2.0 ** -6).half()
    V = T.randint(-1, 2, (M, K), generator=g, device=DEV).half()
    W = (T.randn(N, K, generator=g, device=DEV) / math.sqrt(K)).half()
    dY = T.randn(M, N, generator=g, device=DEV).half()
    Z = T.empty(M, N, dtype=T.float16, device=DEV)
    up = sa.linear_fwd(X + V * h, W, act=sa.ACTS[a], out_dtype=T.float32).double()
    down = sa.linear_fwd(X - V * h, W, act=sa.ACTS[a], out_dtype=T.float32).double()
    sa.linear_fwd(X, W, act=sa.ACTS[a], Z=Z)
    dX, _, _ = sa.linear_bwd(dY, X, W, Z=Z, act=sa.ACTS[a], grads="x")
    got = (dX.double() * V.double()).sum()
    want = (dY.double() * (up - down)).sum() / (2 * h)
    dy, w, x, v = dY.double().abs(), W.double(), X.double(), V.double()
    dir_ = (v @ w.t()).abs()
    u = 2.0 ** -11
    tol = (dy * (1.13 * (K + 16) * E * ((x.abs() + h) @ w.abs().t() + 1) / h + h * h / 3 * dir_ ** 3)).sum() \
        + (2.2 * u * (dy @ w.abs()) * v.abs()).sum() + (u * dX.double().abs() * v.abs()).sum() \
        + (u * dy * Z.double().abs() * dir_).sum()
    assert (got - want).abs() <= tol, (got.item(), want.item(), tol.item())
    assert tol < 0.25 * (dy * dir_).sum()  # the bound says something


def test_offsets_past_32_bits():
    """Matrices of more than 2^32 bytes and 2^31 elements: the last rows are right, each operator over all rows."""
    rows, cols, n = 2 ** 20 + 70, 2112, 72
    g = gen(77)
    X = T.randn(rows, cols, generator=g, device=DEV, dtype=T.bfloat16)
    last = slice(rows - 150, rows)
    gamma = vec(g, cols, 0.2, 1.0)
    Y, mean, rstd = sa.layer_norm_fwd(X, gamma)
    alone = sa.layer_norm_fwd(X[last].clone(), gamma)
    assert T.equal(Y[last], alone[0]) and T.equal(mean[last], alone[1]) and T.equal(rstd[last], alone[2])
    dX = sa.layer_norm_bwd(Y, X, mean, rstd, gamma, dX=Y, params=False)[0]
    assert T.equal(dX[last], sa.layer_norm_bwd(alone[0], X[last].clone(), alone[1], alone[2], gamma, params=False)[0])
    del Y, dX
    W = T.randn(n, cols, generator=g, device=DEV).bfloat16()
    out = sa.linear_fwd(X, W)
    x = X[last].double()
    y = x @ W.double().t()
    check(out[last], y, (cols + 4) * E * (x.abs() @ W.double().abs().t()) + rounded(y, T.bfloat16), "Y")
    dY = T.zeros_like(out)  # only the last rows count
    dY[last] = T.randn(150, n, generator=g, device=DEV).bfloat16()
    dX, dW, db = sa.linear_bwd(dY, X, W, grads="xwb")
    dy = dY[last].double()
    rx, rw = dy @ W.double(), dy.t() @ x
    check(dX[last], rx, (n + 4) * E * (dy.abs() @ W.double().abs()) + rounded(rx, T.bfloat16), "dX")
    # the zeros add exactly
    check(dW, rw, (150 + 4) * E * (dy.abs().t() @ x.abs()) + rounded(rw, T.float32), "dW")
    check(db, dy.sum(0), (150 + 4) * E * dy.abs().sum(0), "dbias")
