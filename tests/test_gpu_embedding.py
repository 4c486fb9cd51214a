"""Token embedding and its gradient against their definitions in 64 bits.

u = 2^-24, w = 2^-8 (bf16): the largest relative error of a rounding.  y is one product, rounded (to bf16: once more).  A row of the gradient is
a sum of n terms: n u times the sum of magnitudes in any order, one rounding for the scale and one where it is added to what was there.
"""
import pytest
import torch

import paper_2406_13936_b200 as pkg

pytestmark = pytest.mark.gpu
U, W = 2.0 ** -24, 2.0 ** -8
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    c = pkg.Context(0)
    yield c
    c.close()


def tokens_of(gen, M, rows, vocab, kind):
    if kind == "one":
        return torch.full((M, rows), vocab - 1, device="cuda", dtype=torch.int32)
    if kind == "runs":                        # the same token for long stretches
        return (torch.arange(rows, device="cuda") // 100 % vocab).to(torch.int32).expand(M, rows).contiguous()
    t = torch.randint(0, vocab, (M, rows), device="cuda", generator=gen, dtype=torch.int32)
    if kind == "falling":
        u = torch.rand((M, rows), device="cuda", generator=gen)
        t = (vocab ** u - 1).floor().clamp_(0, vocab - 1).to(torch.int32)
    if kind == "outside" and rows:            # padding of several kinds
        t[:, ::3] = -1
        t[:, 1::5] = vocab
        t[:, 2::7] = 2 ** 31 - 1
        t[:, 3::11] = -2 ** 31
    return t


SHAPES = [(1, 1, 1, 1), (1, 7, 1001, 129), (2, 33, 10, 8), (3, 100, 50, 64), (1, 300, 777, 100), (2, 4096, 3, 16), (2, 4097, 70000, 24),
          (1, 31, 5, 2050), (1, 64, 511, 4096), (1, 65, 512, 1000), (2, 10000, 513, 40), (1, 5000, 300000, 12), (1, 70000, 1000, 8)]


@pytest.mark.parametrize("M,rows,vocab,d", SHAPES)
@pytest.mark.parametrize("dtype,kind,pad", [("bf16", "uniform", 0), ("f32", "outside", 0), ("bf16", "falling", 3), ("f32", "one", 4), ("bf16", "runs", 8)])
def test_forward_and_backward(ctx, M, rows, vocab, d, dtype, kind, pad):
    gen = torch.Generator(device="cuda").manual_seed(rows + vocab)
    E = torch.randn((M, vocab, d + pad), device="cuda", generator=gen)[:, :, :d]
    tokens = tokens_of(gen, M, rows, vocab, kind)
    Y = torch.full((M, rows, d + pad), 7.0, device="cuda", dtype=TYPES[dtype])
    out = Y[:, :, :d]
    assert ctx.abs_embedding(E, tokens, out, scale=1.7) is out
    inside = (tokens >= 0) & (tokens < vocab)
    at = tokens.long().clamp(0, vocab - 1)
    scale = torch.tensor(1.7, dtype=torch.float32).double().item()
    want = scale * torch.stack([E[m].double()[at[m]] for m in range(M)]) * inside[:, :, None]
    assert ((out.double() - want).abs() <= (2 * U + (W if dtype == "bf16" else 0)) * want.abs()).all()
    assert (Y[:, :, d:] == 7.0).all()
    dY = torch.randn((M, rows, d + pad), device="cuda", generator=gen).to(TYPES[dtype])[:, :, :d]
    count = torch.zeros((M, vocab + 1), device="cuda", dtype=torch.float64)
    sums, sizes = (torch.zeros((M, vocab, d), device="cuda", dtype=torch.float64) for _ in range(2))
    for m in range(M):
        keep = inside[m]
        sums[m].index_add_(0, at[m][keep], scale * dY[m][keep].double())
        sizes[m].index_add_(0, at[m][keep], scale * dY[m][keep].double().abs())
        count[m].index_add_(0, at[m][keep], torch.ones(int(keep.sum()), device="cuda", dtype=torch.float64))
    tol = (count[:, :vocab, None] + 2) * U * sizes
    scratch = ctx.embedding_scratch(M, rows, vocab, d)
    scratch.fill_(0xff)
    full = torch.full((M, vocab, d + pad), 7.0, device="cuda")
    dE = full[:, :, :d]
    assert ctx.abs_embedding_backward(dY, tokens, dE, scratch, scale=1.7) is dE
    assert ((dE.double() - sums).abs() <= tol).all()
    assert (full[:, :, d:] == 7.0).all()
    first = dE.clone()
    dE.fill_(3.0)
    ctx.abs_embedding_backward(dY, tokens, dE, scratch, scale=1.7)
    assert torch.equal(dE, first)                                        # bit for bit
    start = torch.randn(dE.shape, device="cuda", generator=gen)
    dE.copy_(start)
    ctx.abs_embedding_backward(dY, tokens, dE, scratch, scale=1.7, accumulate=True)
    assert ((dE.double() - start.double() - sums).abs() <= tol + U * (start.double() + sums).abs()).all()
    assert torch.equal(dE[count[:, :vocab] == 0], start[count[:, :vocab] == 0])


def test_a_frequent_token_over_many_runs(ctx):
    """200 000 places, one token at a third of them: sums that pass through thousands of partial sums, in order."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows, vocab, d = 200_000, 5000, 16
    tokens = torch.randint(0, vocab, (1, rows), device="cuda", generator=gen, dtype=torch.int32)
    tokens[:, ::3] = 1234
    dY = torch.randn((1, rows, d), device="cuda", generator=gen)
    dE, scratch = torch.empty((1, vocab, d), device="cuda"), ctx.embedding_scratch(1, rows, vocab, d)
    ctx.abs_embedding_backward(dY, tokens, dE, scratch)
    want, size = (torch.zeros((vocab, d), device="cuda", dtype=torch.float64) for _ in range(2))
    want.index_add_(0, tokens[0].long(), dY[0].double())
    size.index_add_(0, tokens[0].long(), dY[0].double().abs())
    n = torch.bincount(tokens[0].long(), minlength=vocab).double()[:, None]
    assert ((dE[0].double() - want).abs() <= (n + 2) * U * size).all()


def test_shared_table_and_shared_tokens(ctx):
    gen = torch.Generator(device="cuda").manual_seed(2)
    E = torch.randn((1, 40, 64), device="cuda", generator=gen)
    tokens = torch.randint(0, 40, (1, 30), device="cuda", generator=gen, dtype=torch.int32)
    Y = torch.empty((3, 30, 64), device="cuda")
    ctx.abs_embedding(E.expand(3, 40, 64), tokens.expand(3, 30), Y)
    assert all(torch.equal(Y[m], E[0][tokens[0].long()]) for m in range(3))
    two = torch.empty((30, 64), device="cuda")
    ctx.abs_embedding(E[0], tokens[0], two)
    assert torch.equal(two, Y[0])
    dE = torch.empty((3, 40, 64), device="cuda")
    ctx.abs_embedding_backward(Y, tokens.expand(3, 30), dE, ctx.embedding_scratch(3, 30, 40, 64))
    assert torch.equal(dE[0], dE[1]) and torch.equal(dE[0], dE[2])


def test_no_rows(ctx):
    none, tokens = torch.empty((2, 0, 8), device="cuda"), torch.empty((2, 0), device="cuda", dtype=torch.int32)
    dE = torch.full((2, 300, 8), 5.0, device="cuda")
    ctx.abs_embedding(dE, tokens, none)
    scratch = ctx.embedding_scratch(2, 0, 300, 8)
    ctx.abs_embedding_backward(none, tokens, dE, scratch, accumulate=True)
    assert (dE == 5.0).all()
    ctx.abs_embedding_backward(none, tokens, dE, scratch)
    assert (dE == 0.0).all()


@pytest.mark.parametrize("rows", [500, 9000])
def test_capture(ctx, rows):
    gen = torch.Generator(device="cuda").manual_seed(3)
    tokens = torch.randint(0, 600, (2, rows), device="cuda", generator=gen, dtype=torch.int32)
    dY, dE = torch.ones((2, rows, 32), device="cuda", dtype=torch.bfloat16), torch.empty((2, 600, 32), device="cuda")
    scratch = ctx.embedding_scratch(2, rows, 600, 32)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        ctx.abs_embedding_backward(dY, tokens, dE, scratch)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ctx.abs_embedding_backward(dY, tokens, dE, scratch)
    for _ in range(2):
        tokens.copy_(torch.randint(0, 600, (2, rows), device="cuda", generator=gen, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for m in range(2):                     # sums of ones are counts, exact
            assert torch.equal(dE[m, :, 0], torch.bincount(tokens[m].long(), minlength=600).float())


@pytest.mark.parametrize("d,rows", [(64, 300), (13, 5000)])
def test_rows_far_apart(ctx, d, rows):
    """Elements behind the 2^31-st of a table: the same bits as from rows that lie together."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    vocab, apart = 520, 1 << 22
    E = torch.randn((vocab, d), device="cuda", generator=gen)
    far = torch.empty((vocab, apart), device="cuda")[:, -((d + 3) // 4 * 4):][:, :d]
    far.copy_(E)
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=gen, dtype=torch.int32)
    tokens[0] = vocab - 1
    dy = torch.randn((rows, d), device="cuda", generator=gen)
    got = []
    for table in (E, far):
        y = ctx.abs_embedding(table, tokens, torch.empty((rows, d), device="cuda"))
        scratch = ctx.embedding_scratch(1, rows, vocab, d)
        ctx.abs_embedding_backward(dy, tokens, table, scratch, scale=0.5, accumulate=True)
        got.append((y, table))
    assert all(torch.equal(p, q) for p, q in zip(*got))


@pytest.mark.parametrize("accumulate", [False, True])
def test_widest_rows_of_odd_strides(ctx, accumulate):
    """d = 2^24 in single elements: more blocks of columns than a grid has in its second dimension.  Whole numbers, so sums are exact."""
    d, vocab = 1 << 24, 3
    tokens = torch.tensor([[1, 0, 1, 5, 1]], dtype=torch.int32, device="cuda")
    dy = torch.randint(-8, 9, (1, 5, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5), dtype=torch.int32).float()
    full = torch.full((1, vocab, d + 1), 7.0, device="cuda")
    got = full[:, :, :d]
    ctx.abs_embedding_backward(dy, tokens, got, ctx.embedding_scratch(1, 5, vocab, d), scale=2.0, accumulate=accumulate)
    base = 7.0 if accumulate else 0.0
    assert torch.equal(got[0, 0], base + 2.0 * dy[0, 1])
    assert torch.equal(got[0, 1], base + 2.0 * (dy[0, 0] + dy[0, 2] + dy[0, 4]))
    assert (got[0, 2] == base).all() and (full[:, :, d] == 7.0).all()
