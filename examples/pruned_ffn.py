"""A gated feed-forward block, pruned by neurons, fine-tuned and decoded.

    y = x + Wd (silu(Wg n) * (Wu n)),   n = layer_norm(x)

The neurons of the block are the filters of one [N, 2K, 1, 1] matrix, row n the pair
[Wg_n | Wu_n]: structadmm_project keeps the strongest, structadmm_compact takes the rows
of the others out, and the columns of Wd that read them.  The compacted matrices are the
operands of the layer norm, gated and linear operators as they are; their gradients in
binary32 go to structadmm_sgd_step.

    python examples/pruned_ffn.py [--width 1024] [--neurons 4096] [--keep 0.6] [--rows 4096]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1807_11091_amd as sa  # noqa: E402


def prune(Wgu, Wd, keep):
    """Keeps `keep` neurons of Wgu [N, 2K] and Wd [K, N] (float32); returns the compacted
    matrices as float32 copies for the optimiser, and the kept neurons' indices."""
    import torch
    N, K2 = Wgu.shape
    dev, W4 = Wgu.device, Wgu.view(N, K2, 1, 1)
    U, Z = torch.zeros_like(W4), torch.empty_like(W4)
    mask = torch.empty(N, dtype=torch.uint8, device=dev)
    kept = torch.empty(keep, dtype=torch.int32, device=dev)
    layer = sa.ProjectLayer(W4, U, Z, mask, kept, sa.FILTER, keep)
    ws = torch.empty(max(sa.project_workspace([layer]), 256), dtype=torch.uint8, device=dev)
    sa.project([layer], ws)
    gu, down = sa.compact_many([dict(Z=Z, row_mask=mask),
                                dict(Z=Wd.view(*Wd.shape, 1, 1), chan_mask=mask)])
    return sa.compacted_matrix(gu[0], gu[-1]), sa.compacted_matrix(down[0], down[-1]), kept


class Block:
    """The pruned block: bfloat16 matrices that the products read, binary32 ones that
    the optimiser keeps, and the buffers of a training step of `rows` rows."""

    def __init__(self, gu, down, width, rows):
        import torch
        self.K, self.N, dev = width, gu.shape[0], gu.device
        new = lambda r, c, t=torch.bfloat16: torch.empty(r, c, dtype=t, device=dev)
        self.gu, self.down = gu, down
        self.gu32, self.down32 = gu.float().contiguous(), down.float().contiguous()
        self.gamma, self.beta = torch.ones(width, device=dev), torch.zeros(width, device=dev)
        pitch = (self.N + 63) // 64 * 64  # rows of whole vectors, as the compacted matrices have them
        self.G, self.U, self.H, self.dH = (new(rows, pitch)[:, :self.N] for _ in range(4))
        self.dgu, self.ddown = new(self.N, 2 * width, torch.float32), new(width, self.N, torch.float32)

    def halves(self, m):
        return m[:, :self.K], m[:, self.K:]

    def decode(self, x):
        """y of a few rows; nothing is kept."""
        n = sa.layer_norm_fwd(x, self.gamma, self.beta, stats=False)[0]
        h = sa.glu_fwd(n, *self.halves(self.gu))
        return sa.linear_fwd(h, self.down, R=x)

    def forward(self, x):
        self.x = x
        self.n, self.mean, self.rstd = sa.layer_norm_fwd(x, self.gamma, self.beta)
        sa.glu_fwd(self.n, *self.halves(self.gu), H=self.H, G=self.G, U=self.U)
        return sa.linear_fwd(self.H, self.down, R=x)

    def backward(self, dy):
        """Gradients of both matrices; returns (dx, dgamma, dbeta)."""
        sa.linear_bwd(dy, self.H, self.down, dX=self.dH, dW=self.ddown)
        dWg, dWu = self.halves(self.dgu)
        dn = sa.glu_bwd(self.dH, self.n, *self.halves(self.gu), self.G, self.U, dWg=dWg, dWu=dWu)[0]
        return sa.layer_norm_bwd(dn, self.x, self.mean, self.rstd, self.gamma, dR=dy)

    def step(self, lr):
        items = [(m.view(*m.shape, 1, 1), g, None, None, None, sa.FILTER, 0.0, lr)
                 for m, g in ((self.gu32, self.dgu), (self.down32, self.ddown))]
        sa.sgd_step(items)
        self.gu.copy_(self.gu32)
        self.down.copy_(self.down32)


def run(width=1024, neurons=4096, keep=0.6, rows=4096, steps=5, lr=0.5, seed=0, log=print):
    """Prunes a random block, tunes it towards the unpruned block's outputs, decodes one
    row; returns the losses and the decoded row's largest difference from the batch's."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    Wgu, Wd = randn(neurons, 2 * width) / width ** 0.5, randn(width, neurons) / neurons ** 0.5
    x = randn(rows, width).bfloat16()
    whole = Block(Wgu.bfloat16(), Wd.bfloat16(), width, rows)
    target = whole.forward(x)
    gu, down, kept = prune(Wgu, Wd, int(neurons * keep))
    block = Block(gu, down, width, rows)
    losses = []
    for _ in range(steps):
        y = block.forward(x)
        error = y.float() - target.float()
        losses.append(0.5 * error.square().sum(1).mean().item())
        dx, dgamma, dbeta = block.backward((error / rows).bfloat16())
        block.step(lr)
        block.gamma.sub_(dgamma, alpha=lr)
        block.beta.sub_(dbeta, alpha=lr)
        log(f"step {len(losses)}: loss {losses[-1]:.4f}, |dx| {dx.float().norm().item():.4f}")
    one, y = block.decode(x[:1]), block.forward(x)
    off = (one.float() - y[:1].float()).abs().max().item()
    log(f"kept {len(kept)} of {neurons} neurons; one decoded row differs by at most {off:.2e}")
    return losses, off


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--width", type=int, default=1024)
    p.add_argument("--neurons", type=int, default=4096)
    p.add_argument("--keep", type=float, default=0.6)
    p.add_argument("--rows", type=int, default=4096)
    p.add_argument("--steps", type=int, default=5)
    a = p.parse_args()
    run(a.width, a.neurons, a.keep, a.rows, a.steps)
