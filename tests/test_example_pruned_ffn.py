"""The pruned feed-forward block of examples/pruned_ffn.py against binary64 autograd."""
import math
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

ROUND = 2.0 ** -9  # relative rounding of bfloat16


def plain(x, gu, down, gamma, beta):
    import torch
    K = x.shape[1]
    d = x - x.mean(1, keepdim=True)
    n = d * (d.square().mean(1, keepdim=True) + 1e-5).rsqrt() * gamma + beta
    g, u = n @ gu[:, :K].T, n @ gu[:, K:].T
    return x + (g * torch.sigmoid(g) * u) @ down.T


@pytest.mark.gpu
@pytest.mark.parametrize("width,neurons,keep,rows", [(64, 256, 128, 64), (96, 250, 151, 70), (77, 300, 33, 1), (256, 1024, 614, 300)])
def test_block_matches_autograd(width, neurons, keep, rows):
    import torch
    import pruned_ffn
    g = torch.Generator(device="cuda").manual_seed(width + rows)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    Wgu, Wd = randn(neurons, 2 * width) / width ** 0.5, randn(width, neurons) / neurons ** 0.5
    gu, down, kept = pruned_ffn.prune(Wgu, Wd, keep)
    want = torch.topk(Wgu.double().norm(dim=1), keep).indices.sort().values
    assert torch.equal(kept.long().sort().values, want)
    assert torch.equal(gu, Wgu[want].bfloat16()) and torch.equal(down, Wd[:, want].bfloat16())

    block = pruned_ffn.Block(gu, down, width, rows)
    block.gamma.add_(randn(width), alpha=0.2)
    block.beta.add_(randn(width), alpha=0.2)
    x, dy = randn(rows, width).bfloat16(), randn(rows, width).bfloat16()
    y = block.forward(x)
    dx, dgamma, dbeta = block.backward(dy)
    leaves = [t.double().detach().requires_grad_() for t in (x, gu, down, block.gamma, block.beta)]
    ref = plain(*leaves)
    grads = torch.autograd.grad(ref, leaves, dy.double())
    # at most six values in a row are rounded to bfloat16 (n, g and u, h; dh, dg and du, dn), each
    # by ROUND relatively, and each is scaled by slopes of at most 2 on its way to a result
    for got, exact in zip((y, dx, block.dgu, block.ddown, dgamma, dbeta), (ref, grads[0], *grads[1:])):
        assert (got.double() - exact).norm() <= 12 * ROUND * exact.norm()
    # the other kernels of a single row round the same values
    one = block.decode(x[:1])
    assert (one.double() - y[:1].double()).abs().max() <= 4 * ROUND * y[:1].double().abs().max() * math.sqrt(2)

    before = block.gu32.clone(), block.down32.clone()
    block.step(0.25)
    assert torch.equal(block.gu32, before[0] - 0.25 * block.dgu) and torch.equal(block.gu, block.gu32.bfloat16())
    assert torch.equal(block.down32, before[1] - 0.25 * block.ddown) and torch.equal(block.down, block.down32.bfloat16())


@pytest.mark.gpu
def test_run_lowers_the_loss():
    import pruned_ffn
    losses, off = pruned_ffn.run(128, 512, 0.6, 256, steps=4, log=lambda s: None)
    assert losses[-1] < 0.9 * losses[0] and off < 0.1
