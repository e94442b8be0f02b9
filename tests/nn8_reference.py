"""Plain binary64 forms of the 8-bit feed-forward operators, and the bounds that their
results keep, on any torch device.  Not a test module.

Roundings: E = 2^-24 for each binary32 operation; e4m3 has 3 bits of mantissa, so a code
is off by at most 2^-4 of its value, and by at most 2^-10 (half of the smallest step) where
it is subnormal.
"""
from __future__ import annotations

import torch

import nn_reference as ref

E = 2.0 ** -24
B = 128
E4M3 = torch.float8_e4m3fn


def blocks(n):
    return (n + B - 1) // B


def wide(scales, rows, cols, block):
    """A block matrix's scales, one for each element, in binary64."""
    s = scales.double().repeat_interleave(B, 1)[:, :cols]
    return s if block == 1 else s.repeat_interleave(B, 0)[:rows]


def values(m, block):
    """What an 8-bit matrix stands for."""
    q, s = m
    return q.double() * wide(s, *q.shape, block)


def amax(v, block):
    """Largest magnitudes of the blocks of v (NaN left out)."""
    r, c = v.shape
    a = torch.nan_to_num(v.abs(), nan=0.0, posinf=float("inf"))
    a = torch.nn.functional.pad(a, (0, blocks(c) * B - c, 0, -r % block))
    return a.view(-1, block, blocks(c), B).amax((1, 3))


def quantise(v, block):
    """The stated rule in binary32, step by step: scales and codes bit for bit."""
    v = v.float()
    top = amax(v, block)
    # two tensors: a division by a number is a multiplication by its reciprocal in torch
    s = torch.clamp(top / torch.full_like(top, 448.0), min=2.0 ** -126)
    inv = torch.ones_like(s) / s
    w = inv.repeat_interleave(B, 1)[:, :v.shape[1]]
    w = w if block == 1 else w.repeat_interleave(B, 0)[:v.shape[0]]
    return (v * w).to(E4M3), s


def check_codes(m, y, tol, what):
    """An 8-bit result with row blocks against its values y, which the kernel knows to
    within tol."""
    q, s = m
    top, off = amax(y, 1), amax(tol, 1)
    want = torch.clamp(top / 448.0, min=2.0 ** -126)
    bad = (s.double() - want).abs() > off / 448.0 + 2 * E * want
    assert not bad.any(), (what, "scales", float(((s.double() - want).abs() / want).max()))
    w = wide(s, *q.shape, 1)
    err = (q.double() * w - y).abs()
    bad = ~(err <= (y.abs() + tol) * 2.0 ** -4 * (1 + 4 * E) + w * 2.0 ** -10 + tol)
    assert not bad.any(), (what, "codes", int(bad.sum()), float(err.max()))


def rms_fwd(s, gamma, eps):
    rstd = (s.square().mean(1) + eps).rsqrt()
    y = s * rstd[:, None]
    return (y if gamma is None else y * gamma), rstd


def rms_bwd(dy, s, rstd, gamma, dr):
    xn = s * rstd[:, None]
    t = dy if gamma is None else dy * gamma
    dx = rstd[:, None] * (t - xn * (t * xn).mean(1, keepdim=True))
    return (dx if dr is None else dx + dr), (dy * xn).sum(0)


def _highest(m, block):
    """2^e of the largest exponent e of each 8 codes of a row, scaled, [rows, groups]."""
    q, s = m
    r, c = q.shape
    v = torch.nn.functional.pad(q.double().abs(), (0, -c % 8))
    e = torch.floor(torch.log2(torch.clamp(v.view(r, -1, 8).amax(2), min=2.0 ** -6)))
    return torch.exp2(e) * wide(s, r, c, block)[:, ::8]


def product(x, w, exact=True):
    """z = x w^T of two 8-bit matrices and how far a binary32 sum may be from it: within
    a block 128 exact products in any order, each addition off by at most 2 E of the
    sums of magnitudes (the matrix cores' adders may cut instead of rounding); then the
    scales' product, a multiplication and an addition for each block, and the joining of
    at most 32 parts and 8 wavefronts.

    exact=False: the 8-bit matrix instructions, which cut each product of 8 consecutive k
    at 2^-13 of 2^(largest sum of two exponents among them)."""
    a, b = values(x, 1), values(w, B)
    mag = a.abs() @ b.abs().t()
    tol = (2 * B + 2 * blocks(a.shape[1]) + 48) * E * mag
    if not exact:
        tol = tol + 8 * 2.0 ** -13 * (_highest(x, 1) @ _highest(w, B).t())
    return a @ b.t(), tol


def linear8(x, w, bias, r, act, exact=True):
    """(y, its tolerance before rounding, z, z's)."""
    z, tol = product(x, w, exact)
    if bias is not None:
        z = z + bias.double()
        tol = tol + E * (z.abs() + bias.double().abs())
    y = ref.act(act, z)
    # slopes are at most 1.13; the exponentials cost a few E of the value and (2 + |z|) E
    ty = tol if act == "none" else 1.13 * tol + (16 + z.abs()) * E * (y.abs() + z.abs() * 2.0 ** -10)
    if r is not None:
        y = y + r.double()
        ty = ty + 2 * E * (y.abs() + r.double().abs())
    return y, ty, z, tol


def glu8(x, wg, wu, bg, bu, act, exact=True):
    """(h, its tolerance, g, g's, u, u's)."""
    a, ta, g, tg = linear8(x, wg, bg, None, act, exact)
    u, tu = linear8(x, wu, bu, None, "none", exact)[:2]
    h = a * u
    return h, ta * (u.abs() + tu) + tu * a.abs() + 2 * E * h.abs(), g, tg, u, tu
