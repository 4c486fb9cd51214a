"""The example that runs embedding, RMS norm with the residual, attention and the statistics together, as a user's program would."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2406_13936_b200 as pkg

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("local_token_block", os.path.join(ROOT, "examples", "local_token_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference(ex, block, tokens):
    """Per-sample losses [M, samples] of the block's parameters in 64 bits, and these."""
    p = block.X.double().requires_grad_(True)
    E, Wqkv, Wo, w1, w2 = block.split(p)
    M, S, L = tokens.shape

    def norm(x, w):
        return x * torch.rsqrt(x.square().mean(3, keepdim=True) + ex.EPS) * w[:, None, None]

    x = torch.stack([E[m][tokens[m].long()] for m in range(M)])
    qkv = torch.einsum("mslk,mjk->mslj", norm(x, w1), Wqkv).unflatten(3, (-1, block.hd))
    q, k, v = qkv.split((block.hq, block.hk, block.hk), dim=3)
    k, v = (t.repeat_interleave(block.hq // block.hk, dim=3) for t in (k, v))
    s = torch.einsum("msihd,msjhd->mshij", q, k) * block.hd ** -0.5
    s = s.masked_fill(~torch.ones((L, L), dtype=torch.bool, device="cuda").tril(), -math.inf)
    o = torch.einsum("mshij,msjhd->msihd", torch.softmax(s, 4), v).flatten(3)
    h = x + torch.einsum("mslk,mjk->mslj", o, Wo)
    logits = torch.einsum("mslk,mjk->mslj", norm(h, w2), E)
    logp = torch.log_softmax(logits, 3)[:, :, :-1]
    return -logp.gather(3, tokens[:, :, 1:, None].long()).squeeze(3).mean(2), p


# fp32: products and sums of up to 400 terms through a chain of ten operations, 400 * 2^-24 each.  bf16: a dozen roundings of 2^-8 lie between
# an input and a gradient, each of them relative to a whole row's size: their sum in the worst case.
@pytest.mark.parametrize("act,hd,bound", [(torch.float32, 24, 10 * 400 * 2.0 ** -24), (torch.bfloat16, 64, 12 * 2.0 ** -8), (torch.bfloat16, 128, 12 * 2.0 ** -8)])
def test_gradients_against_autograd_in_64_bits(ex, act, hd, bound):
    torch.backends.cuda.matmul.allow_tf32 = False
    ctx = pkg.Context(0)
    M, S, L, vocab, d = 2, 3, 131, 50, 48
    block = ex.TokenBlock(ctx, M, vocab, d, 4, 2, hd, act, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    block.X += 0.05 * torch.randn(block.X.shape, device="cuda", generator=gen)
    tokens = torch.randint(0, vocab, (M, S, L), device="cuda", generator=gen, dtype=torch.int32)
    plan = block.plan(S, L)
    logits, saved = block.forward(tokens, plan)
    got, dlogits = block.losses(logits, tokens)
    rows = block.backward(dlogits, saved, plan, S)
    losses, p = reference(ex, block, tokens)
    assert (got.double() - losses).abs().max().item() <= bound * losses.max().item()
    want = torch.autograd.grad(losses.mean(1).sum(), p, retain_graph=True)[0]
    for name, g, ref in zip(("E", "Wqkv", "Wo", "w1", "w2"), block.split(block.grad), block.split(want)):
        assert (g.double() - ref).norm().item() <= bound * ref.norm().item(), name
    for i in range(S):
        ref = torch.autograd.grad(losses[:, i].sum(), p, retain_graph=True)[0][:, -2 * d:]
        assert (rows[:, i].double() - ref).norm().item() <= bound * ref.norm().item(), i
    ctx.close()


def test_training_runs_and_replicas_agree_after_a_round(ex):
    history, block = ex.train(rounds=3, H=2, vocab=64, d=64, length=33, b_max=8)
    sizes = [b for b, _ in history]
    assert all(p <= q <= 8 for p, q in zip(sizes, sizes[1:])) and all(math.isfinite(v) for _, v in history)
    assert all(torch.equal(block.X[0], block.X[m]) for m in range(1, block.M))
