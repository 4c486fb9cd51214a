"""The example that runs the layer norm, the statistics and the Muon step together, as a user's program would."""
import importlib.util
import os

import pytest
import torch

import paper_2406_13936_b200 as pkg

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("local_muon_block", os.path.join(ROOT, "examples", "local_muon_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradients_of_the_block_against_autograd_in_64_bits():
    """Products of up to 320 terms in fp32 (TF32 off): 1e-5 of each gradient's norm."""
    ex = load_example()
    torch.backends.cuda.matmul.allow_tf32 = False
    ctx = pkg.Context(0)
    M, S, T, d, f = 2, 5, 7, 48, 80
    block = ex.Block(ctx, M, d, f, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    block.X += 0.1 * torch.randn(block.X.shape, device="cuda", generator=gen)
    x, target = (torch.randn((M, S * T, d), device="cuda", generator=gen) for _ in range(2))
    y, saved = block.forward(x)
    rows = block.backward((y - target) / (T * d), saved, S)
    p = block.X.double().requires_grad_(True)
    W1, W2, weight, bias = block.split(p)
    h = torch.nn.functional.layer_norm(x.double(), (d,), eps=ex.EPS) * weight[:, None] + bias[:, None]
    out = x.double() + torch.relu(h @ W1.mT) @ W2.mT
    losses = 0.5 * (out - target.double()).square().view(M, S, T * d).mean(2)
    want = torch.autograd.grad(losses.mean(1).sum(), p, retain_graph=True)[0]
    at = 2 * d * f
    for got, ref in ((block.grad[:, :at], want[:, :at]), (rows.mean(1), want[:, at:])):
        assert (got.double() - ref).norm().item() <= 1e-5 * ref.norm().item()
    for i in range(S):
        ref = torch.autograd.grad(losses[:, i].sum(), p, retain_graph=True)[0][:, at:]
        assert (rows[:, i].double() - ref).norm().item() <= 1e-5 * ref.norm().item()
    ctx.close()


def test_training_lowers_the_loss_and_never_shrinks_the_batch():
    history, block = load_example().train(rounds=12, d=64, f=96, b_max=64)
    sizes, losses = [b for b, _ in history], [v for _, v in history]
    assert all(p <= q <= 64 for p, q in zip(sizes, sizes[1:]))
    assert losses[-1] < 0.5 * losses[0]
    assert all(torch.equal(block.X[0], block.X[m]) for m in range(1, block.M))        # averaged at the round's end
