"""Local training of a pre-norm residual block with adaptive batch sizes, M workers on one GPU.

    y = x + relu(layer_norm(x) W1') W2'

Each worker draws its own batches of short token sequences and fits a teacher block.  A local step is: layer norm forward
(abs_layer_norm), the two products, layer norm backward with one gradient row per sample (abs_layer_norm_backward),
the statistics of those rows (abs_test_stats), a Muon step on the two matrices (local_muon_step) and an AdamW step on the
norm's parameters (local_adamw_step).  After H local steps the replicas are averaged inside the last optimiser
calls and the statistics of the last step give the next round's batch size (abs_next_batch).

    python examples/local_muon_block.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2406_13936_b200 as pkg  # noqa: E402

EPS = 1e-5


class Block:
    """M replicas of the block's parameters in one [M, P] tensor: W1 [f, d], W2 [d, f], weight [d], bias [d]."""

    def __init__(self, ctx, M, d, f, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.M, self.d, self.f = ctx, M, d, f
        self.P = 2 * d * f + 2 * d
        x0 = torch.zeros(self.P, device="cuda")
        x0[:d * f] = torch.randn(d * f, device="cuda", generator=gen) * d ** -0.5
        x0[2 * d * f:2 * d * f + d] = 1.0
        self.X = x0.repeat(M, 1)
        self.grad, self.mom1, self.mom2 = (torch.zeros_like(self.X) for _ in range(3))
        self.steps = 0
        ns = pkg.make_ns_cfg()
        self.muon = {rows: pkg.make_muon_cfg(0.02, momentum=0.9, weight_decay=0.0, scale=max(1.0, rows / cols) ** 0.5, ns=ns)
                     for rows, cols in ((f, d), (d, f))}
        self.scratch = ctx.ns_scratch(M, f, d, ns)             # (the same size for either orientation)
        self.stats = ctx.new_stats(M)

    def split(self, flat):
        """(W1, W2, weight, bias) as views of a [M, P] tensor."""
        d, f = self.d, self.f
        return (flat[:, :d * f].view(self.M, f, d), flat[:, d * f:2 * d * f].view(self.M, d, f),
                flat[:, 2 * d * f:2 * d * f + d], flat[:, 2 * d * f + d:])

    def forward(self, x):
        """x [M, tokens, d] -> y and what the backward pass needs."""
        W1, W2, weight, bias = self.split(self.X)
        h = torch.empty_like(x)
        mean, rstd = (torch.empty(x.shape[:2], device="cuda") for _ in range(2))
        self.ctx.abs_layer_norm(x, weight, bias, EPS, h, mean, rstd)
        z = torch.relu(torch.bmm(h, W1.mT))
        return x + torch.bmm(z, W2.mT), (x, h, z, mean, rstd)

    def backward(self, dy, saved, samples):
        """dy: gradient of each sample's own loss.  Fills self.grad with the batch gradient, returns the per-sample
        gradients of the norm's parameters [M, samples, 2 d]."""
        x, h, z, mean, rstd = saved
        W1, W2, weight, _ = self.split(self.X)
        g1, g2, _, _ = self.split(self.grad)
        dz = torch.bmm(dy, W2) * (z > 0)
        g2.copy_(torch.bmm(dy.mT, z) / samples)
        g1.copy_(torch.bmm(dz.mT, h) / samples)
        dh = torch.bmm(dz, W1)
        rows = torch.empty((self.M, samples, 2 * self.d), device="cuda")
        self.ctx.abs_layer_norm_backward(dh, x, mean, rstd, weight, samples=samples, Gw=rows[:, :, :self.d],
                                         Gb=rows[:, :, self.d:])
        return rows

    def local_step(self, x, target, samples, average):
        """One local step of every worker on its batch of `samples` sequences; returns the workers' losses."""
        y, saved = self.forward(x)
        tokens = x.shape[1] // samples
        err = y - target
        rows = self.backward(err / (tokens * self.d), saved, samples)
        gbar = torch.empty((self.M, 2 * self.d), device="cuda")
        self.ctx.abs_test_stats(rows, self.stats, gbar)
        at = 2 * self.d * self.f
        self.grad[:, at:] = gbar
        for X, buf, grad in zip(self.split(self.X)[:2], self.split(self.mom1)[:2], self.split(self.grad)[:2]):
            self.ctx.local_muon_step(X, buf, grad, self.muon[X.shape[1]], self.scratch, average_after=average)
        self.steps += 1
        adamw = pkg.make_adamw_cfg(3e-3, 0.9, 0.95, 1e-8, 0.0, self.steps)
        self.ctx.local_adamw_step(self.X[:, at:], self.mom1[:, at:], self.mom2[:, at:], self.grad[:, at:], adamw,
                                  average_after=average)
        return 0.5 * err.square().mean(dim=(1, 2))


def train(rounds=40, H=8, M=4, d=192, f=320, tokens=16, b0=8, b_max=256, eta=0.8, seed=0, tell=lambda line: None):
    """Returns [(batch size, mean loss of the round's last step)] by round, and the block."""
    ctx = pkg.Context(0)
    teacher, block = Block(ctx, 1, d, f, seed + 1), Block(ctx, M, d, f, seed)
    W1, W2, weight, bias = teacher.split(teacher.X)
    gen = torch.Generator(device="cuda").manual_seed(seed + 2)
    W2.copy_(torch.randn(W2.shape, device="cuda", generator=gen) * f ** -0.5)
    weight.mul_(1.0 + 0.5 * torch.randn(weight.shape, device="cuda", generator=gen))
    test = pkg.make_test_cfg("norm", b_max, eta=eta)
    b_dev = torch.tensor([b0], dtype=torch.int64, device="cuda")
    b, history = b0, []
    for k in range(rounds):
        for h in range(H):
            x = torch.randn((M, b * tokens, d), device="cuda", generator=gen)
            target = teacher.forward(x.view(1, M * b * tokens, d))[0].view(x.shape)
            loss = block.local_step(x, target + 0.05 * torch.randn(x.shape, device="cuda", generator=gen), b, h == H - 1)
        ctx.abs_next_batch(block.stats, test, b_dev, b_dev)
        history.append((b, loss.mean().item()))
        tell("round %2d  batch %3d a worker  loss %.5f" % (k, b, history[-1][1]))
        b = int(b_dev.item())
    return history, block


if __name__ == "__main__":
    train(tell=print)
