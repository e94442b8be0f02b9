"""Plain binary64 forms of the feed-forward operators (layer norm, linear layer,
gated pair) and their gradients, on any torch device.  Not a test module."""
from __future__ import annotations

import math

import torch

ACTS = ["none", "relu", "sigmoid", "silu", "gelu", "gelu_tanh"]


def act(name, z):
    if name == "none":
        return z
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))


def dact(name, z):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "sigmoid":
        p = act("sigmoid", z)
        return p * (1 - p)
    if name == "silu":
        p = act("sigmoid", z)
        return p + z * p * (1 - p)
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def ln_fwd(x, gamma, beta, eps):
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = (d.square().mean(1) + eps).rsqrt()
    y = d * rstd[:, None]
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean, rstd


def ln_bwd(dy, x, mean, rstd, gamma, dr):
    xn = (x - mean[:, None]) * rstd[:, None]
    t = dy if gamma is None else dy * gamma
    dx = rstd[:, None] * (t - t.mean(1, keepdim=True) - xn * (t * xn).mean(1, keepdim=True))
    if dr is not None:
        dx = dx + dr
    return dx, (dy * xn).sum(0), dy.sum(0)


def linear_fwd(x, w, bias, r, a):
    z = x @ w.t()
    if bias is not None:
        z = z + bias
    y = act(a, z)
    return (y if r is None else y + r), z


def linear_bwd(dy, z, x, w, a):
    dz = dy if a == "none" else dy * dact(a, z)
    return dz @ w, dz.t() @ x, dz.sum(0)


def glu_fwd(x, wg, wu, bg, bu, a):
    g, u = x @ wg.t(), x @ wu.t()
    if bg is not None:
        g = g + bg
    if bu is not None:
        u = u + bu
    return act(a, g) * u, g, u


def glu_bwd(dh, g, u, x, wg, wu, a):
    dg, du = dh * u * dact(a, g), dh * act(a, g)
    return dg @ wg + du @ wu, dg.t() @ x, du.t() @ x, dg.sum(0), du.sum(0)
