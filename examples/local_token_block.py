"""Local training of one causal attention block over tokens with adaptive batch sizes, M workers on one GPU.

    x = E[tokens],  h = x + attention(rms_norm(x) Wqkv') Wo',  logits = rms_norm(h) E'

Each worker draws its own sequences of a fixed random walk over the vocabulary and learns to predict the next token; the table E
serves both ends.  A local step is: the embedding (abs_embedding), two RMS norms, the second with the residual's addition
(abs_rms_norm), attention with grouped heads over all workers' sequences at once (abs_attention), their backward passes,
which give one gradient row per sample for the norms, the statistics of those rows (abs_test_stats) and an AdamW step
(local_adamw_step).  After H local steps the replicas are averaged inside the last optimiser call and the statistics of the
last step give the next round's batch size (abs_next_batch).

    python examples/local_token_block.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2406_13936_b200 as pkg  # noqa: E402

EPS = 1e-6


class TokenBlock:
    """M replicas of the parameters in one [M, P] tensor: E [vocab, d], Wqkv [(hq + 2 hk) hd, d], Wo [d, hq hd], two norms' weights [d]."""

    def __init__(self, ctx, M, vocab, d, hq, hk, hd, act=torch.bfloat16, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.M, self.vocab, self.d, self.hq, self.hk, self.hd, self.act = ctx, M, vocab, d, hq, hk, hd, act
        self.sizes = [vocab * d, (hq + 2 * hk) * hd * d, d * hq * hd, d, d]
        x0 = torch.randn(sum(self.sizes), device="cuda", generator=gen) * d ** -0.5
        x0[-2 * d:] = 1.0
        self.X = x0.repeat(M, 1)
        self.grad, self.mom1, self.mom2 = (torch.zeros_like(self.X) for _ in range(3))
        self.steps, self.stats = 0, ctx.new_stats(M)

    def split(self, flat):
        """(E, Wqkv, Wo, w1, w2) as views of a [M, P] tensor."""
        E, Wqkv, Wo, w1, w2 = flat.split(self.sizes, dim=1)
        return E.unflatten(1, (self.vocab, self.d)), Wqkv.unflatten(1, (-1, self.d)), Wo.unflatten(1, (self.d, -1)), w1, w2

    def plan(self, samples, length):
        """The plan of M * samples sequences of `length` tokens and the scratch of their backward pass."""
        n = self.M * samples
        offsets = torch.arange(0, (n + 1) * length, length, dtype=torch.int32, device="cuda")
        return (self.ctx.attention_plan(offsets, n * length),
                self.ctx.attention_scratch(n * length, self.hq, self.hk, self.hd, n),
                self.ctx.embedding_scratch(self.M, samples * length, self.vocab, self.d))

    def forward(self, tokens, plan):
        """tokens [M, samples, length] int32 -> logits [M, samples * length, vocab] and what the backward pass needs."""
        ctx, M = self.ctx, self.M
        tokens = tokens.flatten(1)
        rows = tokens.shape[1]
        E, Wqkv, Wo, w1, w2 = self.split(self.X)
        new = lambda *shape: torch.empty(shape, device="cuda", dtype=self.act)  # noqa: E731
        rstd1, rstd2 = (torch.empty((M, rows), device="cuda") for _ in range(2))
        x = ctx.abs_embedding(E, tokens, new(M, rows, self.d))
        n1 = ctx.abs_rms_norm(x, w1, EPS, new(M, rows, self.d), rstd=rstd1)
        qkv = torch.bmm(n1, Wqkv.to(self.act).mT).view(M * rows, -1, self.hd)
        q, k, v = qkv.split((self.hq, self.hk, self.hk), dim=1)
        o, lse = new(M * rows, self.hq, self.hd), torch.empty((self.hq, M * rows), device="cuda")
        ctx.abs_attention(q, k, v, plan[0], o, lse)
        a = torch.bmm(o.view(M, rows, -1), Wo.to(self.act).mT)
        h, n2 = new(M, rows, self.d), new(M, rows, self.d)
        ctx.abs_rms_norm(a, w2, EPS, n2, residual=x, summed=h, rstd=rstd2)
        return torch.bmm(n2, E.to(self.act).mT), (tokens, x, n1, rstd1, qkv, o, lse, h, n2, rstd2)

    def backward(self, dlogits, saved, plan, samples):
        """dlogits: gradient of each sample's own loss.  Fills self.grad with the batch gradient, returns the per-sample gradients of
        the norms' weights [M, samples, 2 d]."""
        ctx, M, d = self.ctx, self.M, self.d
        tokens, x, n1, rstd1, qkv, o, lse, h, n2, rstd2 = saved
        rows = tokens.shape[1]
        E, Wqkv, Wo, w1, w2 = self.split(self.X)
        gE, gqkv, go, g1, g2 = self.split(self.grad)
        G = torch.empty((M, samples, 2 * d), device="cuda")
        gE.copy_(torch.bmm(dlogits.mT, n2).float() / samples)
        dn2, dh = torch.bmm(dlogits, E.to(self.act)), torch.empty_like(h)
        ctx.abs_rms_norm_backward(dn2, h, rstd2, w2, dX=dh, samples=samples, Gw=G[:, :, d:])
        go.copy_(torch.bmm(dh.mT, o.view(M, rows, -1)).float() / samples)
        do, dqkv = torch.bmm(dh, Wo.to(self.act)).view(o.shape), torch.empty_like(qkv)
        heads = (self.hq, self.hk, self.hk)
        ctx.abs_attention_backward(do, *qkv.split(heads, dim=1), o, lse, plan[0], *dqkv.split(heads, dim=1), plan[1])
        dqkv = dqkv.view(M, rows, -1)
        gqkv.copy_(torch.bmm(dqkv.mT, n1).float() / samples)
        dn1, dx = torch.bmm(dqkv, Wqkv.to(self.act)), torch.empty_like(x)
        ctx.abs_rms_norm_backward(dn1, x, rstd1, w1, dX=dx, dH=dh, samples=samples, Gw=G[:, :, :d])
        ctx.abs_embedding_backward(dx, tokens, gE, plan[2], scale=1.0 / samples, accumulate=True)
        g1.copy_(G[:, :, :d].mean(1))
        g2.copy_(G[:, :, d:].mean(1))
        return G

    def losses(self, logits, tokens):
        """Mean cross entropy of the next token, per sample [M, samples], and the gradient of each sample's own."""
        M, samples, length = tokens.shape
        z = logits.float().unflatten(1, (samples, length))
        logp = torch.log_softmax(z, dim=3)
        at = tokens[:, :, 1:, None].long()
        loss = -logp[:, :, :-1].gather(3, at).squeeze(3).mean(2)
        dz = logp.exp()
        dz[:, :, :-1].scatter_add_(3, at, torch.full(at.shape, -1.0, device="cuda"))
        dz[:, :, -1] = 0.0
        return loss, (dz / (length - 1)).flatten(1, 2).to(self.act)

    def local_step(self, tokens, plan, average, lr=3e-3):
        """One local step of every worker on its batch [M, samples, length]; returns the workers' losses."""
        logits, saved = self.forward(tokens, plan)
        loss, dlogits = self.losses(logits, tokens)
        rows = self.backward(dlogits, saved, plan, tokens.shape[1])
        self.ctx.abs_test_stats(rows, self.stats, torch.empty((self.M, 2 * self.d), device="cuda"))
        self.steps += 1
        adamw = pkg.make_adamw_cfg(lr, 0.9, 0.95, 1e-8, 0.0, self.steps)
        self.ctx.local_adamw_step(self.X, self.mom1, self.mom2, self.grad, adamw, average_after=average)
        return loss.mean(1)


def train(rounds=20, H=4, M=4, vocab=256, d=128, hq=4, hk=2, hd=64, length=64, b0=4, b_max=64, eta=0.8, seed=0, tell=lambda line: None):
    """Returns [(batch size, mean loss of the round's last step)] by round, and the block."""
    ctx = pkg.Context(0)
    block = TokenBlock(ctx, M, vocab, d, hq, hk, hd, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    follows = torch.randint(0, vocab, (vocab, 4), device="cuda", generator=gen, dtype=torch.int32)      # each token's successors
    test = pkg.make_test_cfg("norm", b_max, eta=eta)
    b_dev = torch.tensor([b0], dtype=torch.int64, device="cuda")
    b, history = b0, []
    for r in range(rounds):
        plan = block.plan(b, length)
        for s in range(H):
            tokens = torch.randint(0, vocab, (M, b, length), device="cuda", generator=gen, dtype=torch.int32)
            turns = torch.randint(0, 4, (M, b, length), device="cuda", generator=gen)
            for t in range(1, length):
                tokens[:, :, t] = follows[tokens[:, :, t - 1].long(), turns[:, :, t]]
            loss = block.local_step(tokens, plan, s == H - 1)
        ctx.abs_next_batch(block.stats, test, b_dev, b_dev)
        history.append((b, loss.mean().item()))
        tell("round %2d  batch %3d a worker  loss %.4f" % (r, b, history[-1][1]))
        b = int(b_dev.item())
    return history, block


if __name__ == "__main__":
    train(tell=print)
