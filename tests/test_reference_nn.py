"""CPU checks of the binary64 reference of the feed-forward operators: every
gradient formula against central differences of the forward formula."""
import pytest
import torch

import nn_reference as ref

H = 1e-5  # central differences: error O(h^2) + rounding / h, both far below 1e-7 at this scale


def rnd(seed, *shape):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def differences(f, x):
    """d f / d x by central differences, f a scalar function."""
    out = torch.zeros_like(x)
    flat, o = x.view(-1), out.view(-1)
    for i in range(flat.numel()):
        keep = flat[i].item()
        flat[i] = keep + H
        up = f().item()
        flat[i] = keep - H
        down = f().item()
        flat[i] = keep
        o[i] = (up - down) / (2 * H)
    return out


def close(a, b):
    torch.testing.assert_close(a, b, rtol=1e-6, atol=1e-7)


@pytest.mark.parametrize("a", ref.ACTS)
def test_activation_slopes(a):
    z = rnd(1, 40) * 2
    y = lambda: ref.act(a, z).sum()
    close(differences(y, z), ref.dact(a, z))


@pytest.mark.parametrize("gamma", [True, False])
def test_layer_norm_gradient(gamma):
    x, dy, dr = rnd(2, 3, 7), rnd(3, 3, 7), rnd(4, 3, 7)
    g, b = (rnd(5, 7), rnd(6, 7)) if gamma else (None, None)
    loss = lambda: (ref.ln_fwd(x, g, b, 1e-5)[0] * dy).sum() + (x * dr).sum()
    _, mean, rstd = ref.ln_fwd(x, g, b, 1e-5)
    dx, dg, db = ref.ln_bwd(dy, x, mean, rstd, g, dr)
    close(differences(loss, x), dx)
    if gamma:
        close(differences(loss, g), dg)
        close(differences(loss, b), db)


@pytest.mark.parametrize("a", ref.ACTS)
def test_linear_gradient(a):
    x, w, b, r, dy = rnd(7, 4, 5), rnd(8, 3, 5), rnd(9, 3), rnd(10, 4, 3), rnd(11, 4, 3)
    loss = lambda: (ref.linear_fwd(x, w, b, r, a)[0] * dy).sum()
    z = ref.linear_fwd(x, w, b, r, a)[1]
    for t, grad in zip((x, w, b), ref.linear_bwd(dy, z, x, w, a)):
        close(differences(loss, t), grad)
    close(differences(loss, r), dy)


@pytest.mark.parametrize("a", ref.ACTS)
def test_glu_gradient(a):
    x, wg, wu, bg, bu, dh = rnd(12, 4, 5), rnd(13, 3, 5), rnd(14, 3, 5), rnd(15, 3), rnd(16, 3), rnd(17, 4, 3)
    loss = lambda: (ref.glu_fwd(x, wg, wu, bg, bu, a)[0] * dh).sum()
    _, g, u = ref.glu_fwd(x, wg, wu, bg, bu, a)
    for t, grad in zip((x, wg, wu, bg, bu), ref.glu_bwd(dh, g, u, x, wg, wu, a)):
        close(differences(loss, t), grad)
