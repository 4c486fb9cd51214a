"""Layer norm, forward and backward, against the formulas in 64 bits.

Tolerances, from the arithmetic (u = 2^-24, the unit roundoff of fp32's 24 bits; v = 2^-8, that of bf16's 8):
  xh carries the rounding of x - mean, whose size goes with |x|: 8 u k with k = 1 + |mean| rstd, the
  condition of the centring (the mean itself is a sum of d terms in fp32, at worst a few u more);
  y is then rounded once to its type.  Sums over n rows are held to 4 u sqrt(n) of the root of the
  sum of squares of their terms, plus the error of the terms; 32 u is taken for what a term carries.
"""
import numpy as np
import pytest
import torch

import paper_2406_13936_b200 as pkg

pytestmark = pytest.mark.gpu

U, V = 2.0 ** -24, 2.0 ** -8
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    c = pkg.Context(0)
    yield c
    c.close()


def rows_of(seed, M, rows, d, pad=0, offset=0, dtype="f32", scale=1.0, shift=0.3):
    """[M, rows, d] view with rows of d + pad elements, starting `offset` elements into its memory."""
    gen = torch.Generator().manual_seed(seed)
    n = M * rows * (d + pad)
    flat = torch.randn(n + offset, generator=gen) * scale + shift
    return flat.to(TYPES[dtype]).cuda()[offset:offset + n].view(M, rows, d + pad)[:, :, :d]


def params_of(seed, M, d, pad=0):
    gen = torch.Generator().manual_seed(seed)
    p = (torch.randn((M, 2 * d + pad), generator=gen) * 0.3 + 0.8).cuda()
    return p[:, :d], p[:, d:2 * d]


def ref_forward(x, w, b):
    x = x.double()
    mean = x.mean(2)
    rstd = (x.var(2, unbiased=False) + EPS).rsqrt()
    y = (x - mean[:, :, None]) * rstd[:, :, None]
    if w is not None:
        y = y * w.double()[:, None]
    if b is not None:
        y = y + b.double()[:, None]
    return y, mean, rstd


def ref_backward(dy, x, mean, rstd, w, samples):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, :, None], rstd.double()[:, :, None]
    xh = (x - mean) * rstd
    a = dy if w is None else dy * w.double()[:, None]
    dx = rstd * (a - a.mean(2, keepdim=True) - xh * (a * xh).mean(2, keepdim=True))
    M, rows, d = x.shape
    seg = (M, samples, rows // samples if samples else 0, d)
    return dx, (dy * xh).reshape(seg), dy.reshape(seg)


def check_sum(got, terms, dim, dtype_note=""):
    terms = terms.double()
    n = max(1, terms.numel() // max(1, got.numel()))
    want = terms.sum(dim)
    size = terms.square().sum(dim).sqrt()
    err = (got.double() - want).abs()
    assert bool((err <= (4 * U * n ** 0.5 + 32 * U) * n ** 0.5 * size + 1e-30).all()), dtype_note


# (M, rows, d, pad, offset): one row, one column, odd widths, widths around every power of two a kernel
# might tile by, rows inside wider rows, bases that are not 16-byte aligned, many rows, very wide rows
SHAPES = [(1, 1, 1, 0, 0), (1, 1, 768, 0, 0), (2, 3, 5, 0, 0), (1, 7, 31, 0, 0), (3, 33, 64, 0, 0), (1, 65, 127, 1, 0),
          (2, 40, 256, 0, 0), (2, 17, 257, 7, 0), (1, 9, 768, 8, 0), (1, 130, 768, 0, 1), (2, 1, 1000, 0, 0),
          (8, 129, 768, 0, 0), (1, 12, 1021, 3, 2), (2, 50, 1024, 0, 0), (1, 37, 2048, 0, 0), (1, 21, 2056, 0, 8),
          (1, 19, 4096, 0, 0), (1, 5, 8192, 0, 0), (1, 6, 8200, 0, 0), (1, 3, 16384, 8, 0), (1, 2, 40001, 0, 0),
          (1, 3000, 96, 0, 0), (4, 700, 512, 0, 0), (1, 600, 1536, 0, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,rows,d,pad,offset", SHAPES)
def test_forward(ctx, M, rows, d, pad, offset, dtype):
    x = rows_of(1, M, rows, d, pad, offset, dtype)
    w, b = params_of(2, M, d, 5)
    y = torch.full((M, rows, d + pad), 7.0, device="cuda", dtype=TYPES[dtype])
    mean, rstd = (torch.empty((M, rows), device="cuda") for _ in range(2))
    ctx.abs_layer_norm(x, w, b, EPS, y[:, :, :d], mean, rstd)
    ry, rm, rr = ref_forward(x, w, b)
    k = 1 + rm.abs() * rr
    assert bool(((mean - rm).abs() <= 8 * U * (x.double().abs().mean(2) + 1e-30)).all())
    assert bool(((rstd - rr).abs() <= 16 * U * k * rr).all())
    xh = (ry - b.double()[:, None]).abs() + w.double().abs()[:, None]
    tol = 24 * U * k[:, :, None] * xh + 4 * U * b.double().abs()[:, None]
    if dtype == "bf16":
        tol = tol + V * ry.abs() * (1 + 4 * V)
    assert bool(((y[:, :, :d].double() - ry).abs() <= tol).all())
    assert bool((y[:, :, d:] == 7.0).all())             # nothing outside the rows is written


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,rows,d,pad,offset", SHAPES)
def test_backward_totals(ctx, M, rows, d, pad, offset, dtype):
    x = rows_of(1, M, rows, d, pad, offset, dtype)
    dy = rows_of(3, M, rows, d, pad, offset, dtype, 1e-2, 1e-3)
    w, _ = params_of(2, M, d, 3)
    _, rm, rr = ref_forward(x, None, None)
    mean, rstd = rm.float(), rr.float()
    dx = torch.full((M, rows, d + pad), 7.0, device="cuda", dtype=TYPES[dtype])
    grads = torch.full((M, 2 * d + 9), 7.0, device="cuda")
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, w, dx[:, :, :d], grads[:, :d], grads[:, d:2 * d])
    rdx, tw, tb = ref_backward(dy, x, mean, rstd, w, 1)
    check_dx(dx[:, :, :d], rdx, x, dy, w, mean, rstd, dtype)
    check_sum(grads[:, :d], tw, (1, 2))
    check_sum(grads[:, d:2 * d], tb, (1, 2))
    assert bool((dx[:, :, d:] == 7.0).all()) and bool((grads[:, 2 * d:] == 7.0).all())


def check_dx(got, want, x, dy, w, mean, rstd, dtype):
    a = dy.double() * (1 if w is None else w.double()[:, None])
    xh = (x.double() - mean.double()[:, :, None]) * rstd.double()[:, :, None]
    k = (1 + mean.abs().double() * rstd.double())[:, :, None]
    rms_a = a.square().mean(2, keepdim=True).sqrt()
    tol = 32 * U * k * rstd.double()[:, :, None] * (a.abs() + rms_a * (1 + xh.abs()) * (1 + xh.square().mean(2, keepdim=True).sqrt()))
    if dtype == "bf16":
        tol = tol + V * want.abs() * (1 + 4 * V)
    assert bool(((got.double() - want).abs() <= tol + 1e-30).all())


SAMPLES = [(1, 1, 1, 8), (2, 5, 1, 257), (1, 300, 1, 64), (3, 7, 33, 100), (2, 16, 128, 768), (1, 2, 1000, 512),
           (1, 64, 3, 1024), (8, 4, 50, 768), (1, 3, 17, 4096), (2, 9, 5, 9000), (1, 1, 2500, 320), (1, 40, 64, 2048)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,S,T,d", SAMPLES)
def test_backward_per_sample(ctx, M, S, T, d, dtype):
    """Per-sample rows, their totals, and the statistics kernel reading them where they lie."""
    x = rows_of(5, M, S * T, d, 0, 0, dtype)
    dy = rows_of(6, M, S * T, d, 0, 0, dtype, 1e-2, 1e-3)
    w, _ = params_of(7, M, d)
    _, rm, rr = ref_forward(x, None, None)
    mean, rstd = rm.float(), rr.float()
    G = torch.full((M, S + 1, 2 * d + 4), 7.0, device="cuda")
    dx = torch.empty((M, S * T, d), device="cuda", dtype=TYPES[dtype])
    dW, dB = (torch.empty((M, d), device="cuda") for _ in range(2))
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, w, dx, dW, dB, samples=S, Gw=G[:, :S, :d], Gb=G[:, :S, d:2 * d])
    rdx, tw, tb = ref_backward(dy, x, mean, rstd, w, S)
    check_dx(dx, rdx, x, dy, w, mean, rstd, dtype)
    check_sum(G[:, :S, :d], tw, 2)
    check_sum(G[:, :S, d:2 * d], tb, 2)
    check_sum(dW, tw, (1, 2))
    check_sum(dB, tb, (1, 2))
    assert bool((G[:, S:] == 7.0).all()) and bool((G[:, :, 2 * d:] == 7.0).all())
    # gradients alone (no dx, no totals) give the same rows, bit for bit
    G2 = torch.full_like(G, 7.0)
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, w, None, samples=S, Gw=G2[:, :S, :d], Gb=G2[:, :S, d:2 * d])
    assert torch.equal(G, G2)
    if S >= 2:
        stats, gbar = ctx.new_stats(M), torch.empty((M, 2 * d), device="cuda")
        ctx.abs_test_stats(G[:, :S, :2 * d], stats, gbar)
        want = torch.cat([tw.sum(2), tb.sum(2)], 2)
        for m, rec in enumerate(pkg.stats_to_dicts(stats)):
            var = want[m].var(0).sum().item()
            assert abs(rec["var_norm"] - var) <= 1e-4 * var + 1e-12
        check_sum(gbar * S, torch.cat([tw, tb], 3), (1, 2))


def test_optional_parts(ctx):
    M, rows, d = 2, 37, 200
    x, dy = rows_of(1, M, rows, d), rows_of(2, M, rows, d)
    y, mean, rstd = torch.empty_like(x), torch.empty((M, rows), device="cuda"), torch.empty((M, rows), device="cuda")
    ctx.abs_layer_norm(x, None, None, EPS, y, mean, rstd)
    ry, rm, rr = ref_forward(x, None, None)
    assert (y - ry).abs().max().item() <= 1e-5
    y2 = torch.empty_like(y)
    ctx.abs_layer_norm(x, None, None, EPS, y2)           # without the statistics
    assert torch.equal(y, y2)
    w, b = params_of(3, M, d)
    ctx.abs_layer_norm(x, None, b, EPS, y)
    assert (y - ref_forward(x, None, b)[0]).abs().max().item() <= 1e-5
    ctx.abs_layer_norm(x, w, None, EPS, y)
    assert (y - ref_forward(x, w, None)[0]).abs().max().item() <= 1e-5
    dx, dW, dB = torch.empty_like(x), torch.empty((M, d), device="cuda"), torch.empty((M, d), device="cuda")
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, None, dx, dW, dB)
    rdx, tw, tb = ref_backward(dy, x, mean, rstd, None, 1)
    check_dx(dx, rdx, x, dy, None, mean, rstd, "f32")
    only = torch.empty((M, d), device="cuda")
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, None, dB=only)
    assert torch.equal(only, dB)
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, None, dW=only)
    assert torch.equal(only, dW)
    dx2 = torch.empty_like(x)
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, None, dx2)
    assert torch.equal(dx, dx2)


@pytest.mark.parametrize("d", [96, 768, 1001, 5000])
def test_in_place_and_shared_parameters(ctx, d):
    M, rows = 3, 21
    x, dy = rows_of(1, M, rows, d), rows_of(2, M, rows, d)
    w, b = params_of(3, 1, d)
    w, b = w.expand(M, d), b.expand(M, d)                # one parameter vector for all replicas
    y, mean, rstd = torch.empty_like(x), torch.empty((M, rows), device="cuda"), torch.empty((M, rows), device="cuda")
    ctx.abs_layer_norm(x, w, b, EPS, y, mean, rstd)
    assert (y - ref_forward(x, w, b)[0]).abs().max().item() <= 1e-5
    x2 = x.clone()
    ctx.abs_layer_norm(x2, w, b, EPS, x2)
    assert torch.equal(x2, y)
    dx, dW = torch.empty_like(x), torch.empty((M, d), device="cuda")
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, w, dx, dW)
    for target in ("dy", "x"):
        a, c, dW2 = dy.clone(), x.clone(), torch.empty_like(dW)
        ctx.abs_layer_norm_backward(a, c, mean, rstd, w, a if target == "dy" else c, dW2)
        assert torch.equal(a if target == "dy" else c, dx) and torch.equal(dW, dW2)


def test_nothing_to_do(ctx):
    x = torch.empty((2, 0, 64), device="cuda")
    m = torch.empty((2, 0), device="cuda")
    ctx.abs_layer_norm(x, None, None, EPS, torch.empty_like(x), m, m)
    dW, dB = torch.full((2, 64), 7.0, device="cuda"), torch.full((2, 64), 7.0, device="cuda")
    G = torch.full((2, 3, 128), 7.0, device="cuda")
    ctx.abs_layer_norm_backward(x, x, m, m, None, torch.empty_like(x), dW, dB, samples=3, Gw=G[:, :, :64], Gb=G[:, :, 64:])
    assert not dW.any() and not dB.any() and not G.any()
    dW.fill_(7.0)
    ctx.abs_layer_norm_backward(x, x, m, m, None, torch.empty_like(x), dW)
    assert not dW.any()


@pytest.mark.parametrize("d", [48, 768, 1021, 6000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_rows(ctx, d, dtype):
    """Constant rows (variance zero), a row far from zero, and NaN / infinity staying in their row."""
    x = rows_of(1, 1, 8, d, dtype=dtype)
    x[0, 1] = 2.5
    x[0, 2] = 0.0
    x[0, 3] += 100.0
    x[0, 5, d // 2] = float("nan")
    x[0, 6, 0] = float("inf")
    w, b = params_of(2, 1, d)
    y, mean, rstd = torch.empty_like(x), torch.empty((1, 8), device="cuda"), torch.empty((1, 8), device="cuda")
    ctx.abs_layer_norm(x, w, b, EPS, y, mean, rstd)
    good = [0, 1, 2, 3, 4, 7]
    ry, rm, rr = ref_forward(x, w, b)
    lim = {"f32": 1e-5, "bf16": 2 * V}[dtype]
    for r in good:
        k = 1 + (rm[0, r].abs() * rr[0, r]).item() * (0 if r == 1 else 1)
        assert ((y[0, r].double() - ry[0, r]).abs() <= lim * k * (1 + ry[0, r].abs())).all(), r
    assert torch.isnan(y[0, 5]).all() and torch.isnan(y[0, 6]).any()
    assert abs(rstd[0, 1].item() - EPS ** -0.5) <= 1e-4 * EPS ** -0.5
    dy = rows_of(4, 1, 8, d, dtype=dtype)
    dx, dW = torch.empty_like(x), torch.empty((1, d), device="cuda")
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, w, dx, dW)
    for r in good:
        assert torch.isfinite(dx[0, r].float()).all()
    assert torch.isnan(dx[0, 5].float()).all()


def test_against_autograd_and_differences(ctx):
    """The formula's gradient (autograd in 64 bits) and central differences of the forward kernel."""
    M, rows, d = 2, 29, 320
    x, c = rows_of(1, M, rows, d), rows_of(2, M, rows, d)
    w, b = (t.contiguous() for t in params_of(3, M, d))
    y, mean, rstd = torch.empty_like(x), torch.empty((M, rows), device="cuda"), torch.empty((M, rows), device="cuda")
    ctx.abs_layer_norm(x, w, b, EPS, y, mean, rstd)
    dx, dW, dB = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    ctx.abs_layer_norm_backward(c, x, mean, rstd, w, dx, dW, dB)
    xd, wd, bd = (t.double().requires_grad_() for t in (x, w, b))
    (ref_forward(xd, wd, bd)[0] * c.double()).sum().backward()
    for got, want in ((dx, xd.grad), (dW, wd.grad), (dB, bd.grad)):
        assert ((got.double() - want).norm() / want.norm()).item() <= 1e-5

    def loss(xx, ww, bb):
        out = torch.empty_like(xx)
        ctx.abs_layer_norm(xx, ww, bb, EPS, out)
        return (out.double() * c.double()).sum().item()

    h = 2.0 ** -6
    for k, (t, g) in enumerate(((x, dx), (w, dW), (b, dB))):
        v = rows_of(10 + k, *((1,) + tuple(t.shape)) if t.dim() == 2 else t.shape, shift=0.0).view(t.shape)
        args = [x, w, b]
        plus, minus = list(args), list(args)
        plus[k], minus[k] = t + h * v, t - h * v
        num = (loss(*plus) - loss(*minus)) / (2 * h)
        want = (g.double() * v.double()).sum().item()
        # truncation h^2 and rounding u / h of about sqrt(number of outputs) independent terms
        assert abs(num - want) <= 8 * (h * h + 4 * U / h) * (M * rows * d) ** 0.5


def test_large_offsets(ctx):
    """Replicas more than 2^31 elements apart."""
    d, far = 64, (1 << 31) + 64
    flat = torch.empty(far + 4 * d, device="cuda", dtype=torch.bfloat16)
    x = torch.as_strided(flat, (2, 4, d), (far, d, 1))
    x.copy_(rows_of(1, 2, 4, d, dtype="bf16"))
    y = torch.empty((2, 4, d), device="cuda", dtype=torch.bfloat16)
    mean, rstd = torch.empty((2, 4), device="cuda"), torch.empty((2, 4), device="cuda")
    ctx.abs_layer_norm(x, None, None, EPS, y, mean, rstd)
    z = x.contiguous()
    y2 = torch.empty_like(y)
    ctx.abs_layer_norm(z, None, None, EPS, y2)
    assert torch.equal(y, y2)
    dx, dx2 = torch.empty_like(y), torch.empty_like(y)
    ctx.abs_layer_norm_backward(y, x, mean, rstd, None, dx)
    ctx.abs_layer_norm_backward(y, z, mean, rstd, None, dx2)
    assert torch.equal(dx, dx2)


def test_repeatable_and_on_a_stream(ctx):
    M, S, T, d = 4, 6, 90, 768
    x, dy = rows_of(1, M, S * T, d, dtype="bf16"), rows_of(2, M, S * T, d, dtype="bf16")
    _, rm, rr = ref_forward(x, None, None)
    mean, rstd = rm.float(), rr.float()

    def run(stream=None):
        dx, dW = torch.empty_like(x), torch.empty((M, d), device="cuda")
        G = torch.empty((M, S, d), device="cuda")
        ctx.abs_layer_norm_backward(dy, x, mean, rstd, None, dx, dW, samples=S, Gw=G, stream=stream)
        return dx, dW, G

    first = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = run(side)
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_refusals(ctx):
    x = torch.zeros((2, 4, 32), device="cuda")
    w = torch.ones((2, 32), device="cuda")
    m = torch.zeros((2, 4), device="cuda")
    for bad in (lambda: ctx.abs_layer_norm(x, w, None, -1.0, x),
                lambda: ctx.abs_layer_norm(x, w, None, float("nan"), x),
                lambda: ctx.abs_layer_norm(x.half(), w, None, EPS, x.half()),
                lambda: ctx.abs_layer_norm(x, w[:1], None, EPS, x),
                lambda: ctx.abs_layer_norm(x, w.bfloat16(), None, EPS, x),
                lambda: ctx.abs_layer_norm(x, w, None, EPS, x[:, :, :16]),
                lambda: ctx.abs_layer_norm(x.transpose(1, 2), None, None, EPS, x.transpose(1, 2)),
                lambda: ctx.abs_layer_norm(x, w, None, EPS, x, m[:1], m),
                lambda: ctx.abs_layer_norm(x[:, :1].expand(2, 4, 32), w, None, EPS, x),       # rows that overlap
                lambda: ctx.abs_layer_norm_backward(x, x, m, m, w, x, samples=3),
                lambda: ctx.abs_layer_norm_backward(x, x, m, None, w, x),
                lambda: ctx.abs_layer_norm_backward(x, x.bfloat16(), m, m, w, x),
                lambda: ctx.abs_layer_norm_backward(x, x, m, m, w, x, samples=2, Gw=torch.zeros((2, 3, 32), device="cuda")),
                lambda: ctx.abs_layer_norm_backward(x, x, m, m, w, x, w.double())):
        with pytest.raises(pkg.AbsError):
            bad()
    small = pkg.Context(0, workspace_bytes=4096)
    try:
        G = torch.zeros((1, 64, 32), device="cuda")
        y = torch.zeros((1, 64, 32), device="cuda")
        mm = torch.zeros((1, 64), device="cuda")
        dW = torch.empty((1, 32), device="cuda")
        small.abs_layer_norm_backward(y, y, mm, mm, None, None, dW)           # one partial sum fits
        with pytest.raises(pkg.AbsError, match="workspace"):
            big = torch.zeros((1, 8, 4096), device="cuda")
            small.abs_layer_norm_backward(big, big, mm[:, :8].contiguous(), mm[:, :8].contiguous(), None, None,
                                          torch.empty((1, 4096), device="cuda"))
        del G
    finally:
        small.close()
    assert np.isfinite(dW.sum().item())


# (M, samples, tokens, d, offset, spare places of the workspace): rows staged in shared memory, in registers, of any width
TIGHT = [(1, 64, 2, 96, 0, 3), (1, 300, 23, 512, 0, 7), (3, 50, 5, 257, 0, 7), (2, 1000, 11, 96, 1, 40), (1, 40, 3, 9000, 0, 2),
         (4, 7, 1, 768, 0, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,S,T,d,offset,spare", TIGHT)
def test_a_workspace_with_barely_enough_places(ctx, M, S, T, d, offset, spare, dtype):
    """One of the two per-sample gradients of short samples, or both, or the totals alone."""
    x, dy = rows_of(31, M, S * T, d, 0, offset, dtype), rows_of(32, M, S * T, d, 0, offset, dtype, 1e-2, 1e-3)
    w, _ = params_of(33, M, d)
    _, rm, rr = ref_forward(x, None, None)
    mean, rstd = rm.float(), rr.float()
    _, tw, tb = ref_backward(dy, x, mean, rstd, w, S)
    for gw, gb, totals in ((1, 0, 0), (0, 1, 1), (1, 1, 1), (0, 0, 1)):
        places = 2 if gw and gb else M * (S if gw or gb else 1) + 1
        small = pkg.Context(0, workspace_bytes=(places + spare - 1) * 8 * d)
        try:
            G, H = (torch.full((M, S, d), 7.0, device="cuda") for _ in range(2))
            dW, dB = (torch.full((M, d), 7.0, device="cuda") for _ in range(2))
            small.abs_layer_norm_backward(dy, x, mean, rstd, w, None, dW if totals else None, dB if totals else None, samples=S,
                                          Gw=G if gw else None, Gb=H if gb else None)
            for wanted, got, terms, dim in ((gw, G, tw, 2), (gb, H, tb, 2), (totals, dW, tw, (1, 2)), (totals, dB, tb, (1, 2))):
                if wanted:
                    check_sum(got, terms, dim)
            if places > 2:
                with pytest.raises(pkg.AbsError, match="workspace"):
                    tiny = pkg.Context(0, workspace_bytes=(places - 1) * 8 * d)
                    tiny.abs_layer_norm_backward(dy, x, mean, rstd, w, None, dW if totals else None, dB if totals else None,
                                                 samples=S, Gw=G if gw else None, Gb=H if gb else None)
        finally:
            small.close()


@pytest.mark.parametrize("which", ["Gw", "Gb"])
def test_one_gradient_of_many_short_samples(ctx, which):
    """14738 samples of 23 rows of 512: their places and the CTAs' nearly fill the default workspace."""
    S, T, d = 14738, 23, 512
    x, dy = rows_of(34, 1, S * T, d), rows_of(35, 1, S * T, d, scale=1e-2, shift=1e-3)
    mean, rstd = (t.float() for t in ref_forward(x, None, None)[1:])
    G = torch.full((1, S + 1, d), 7.0, device="cuda")
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, None, samples=S, **{which: G[:, :S]})
    _, tw, tb = ref_backward(dy, x, mean, rstd, None, S)
    check_sum(G[:, :S], tw if which == "Gw" else tb, 2)
    assert bool((G[:, S:] == 7.0).all())


@pytest.mark.parametrize("dtype,d", [("bf16", 768), ("f32", 257), ("f32", 9000)])
def test_in_a_graph(ctx, dtype, d):
    """Forward and backward captured once, replayed on new inputs (rows in shared memory, in registers, of any width)."""
    M, S, T = 2, 40, 9
    x, dy = rows_of(51, M, S * T, d, dtype=dtype), rows_of(52, M, S * T, d, dtype=dtype)
    w, b = params_of(53, M, d)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty((M, S * T), device="cuda") for _ in range(2))
    dW, dB = (torch.empty((M, d), device="cuda") for _ in range(2))
    G = torch.empty((M, S, 2 * d), device="cuda")
    outputs = (y, dx, mean, rstd, dW, dB, G)

    def run():
        ctx.abs_layer_norm(x, w, b, EPS, y, mean, rstd)
        ctx.abs_layer_norm_backward(dy, x, mean, rstd, w, dx, dW, dB, samples=S, Gw=G[:, :, :d], Gb=G[:, :, d:])

    run()                                                # what a context does once is not captured
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in (54, 55):
        x.copy_(rows_of(seed, M, S * T, d, dtype=dtype))
        for t in outputs:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outputs]
        run()
        for got, want in zip(replayed, outputs):
            assert torch.equal(got, want)
    check_dx(dx, ref_backward(dy, x, mean, rstd, w, S)[0], x, dy, w, mean, rstd, dtype)


# the last widths of the kernels that hold a row in one CTA and the first ones past them, aligned and not
@pytest.mark.parametrize("dtype,d", [("f32", 6144), ("f32", 6148), ("f32", 9216), ("f32", 9220), ("bf16", 9216), ("bf16", 9224),
                                     ("bf16", 12800), ("bf16", 12808), ("bf16", 18432), ("f32", 6143), ("f32", 6145), ("bf16", 6143),
                                     ("bf16", 6146)])
def test_widths_around_the_limits(ctx, dtype, d):
    x, dy = rows_of(56, 2, 11, d, dtype=dtype), rows_of(57, 2, 11, d, dtype=dtype, scale=1e-2, shift=1e-3)
    w, b = params_of(58, 2, d)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty((2, 11), device="cuda") for _ in range(2))
    dW, dB = (torch.empty((2, d), device="cuda") for _ in range(2))
    ctx.abs_layer_norm(x, w, b, EPS, y, mean, rstd)
    ry, rm, rr = ref_forward(x, w, b)
    k = (1 + rm.abs() * rr)[:, :, None]
    xh = (ry - b.double()[:, None]).abs() + w.double().abs()[:, None]
    tol = 24 * U * k * xh + 4 * U * b.double().abs()[:, None]
    if dtype == "bf16":
        tol = tol + V * ry.abs() * (1 + 4 * V)
    assert bool(((y.double() - ry).abs() <= tol).all())
    ctx.abs_layer_norm_backward(dy, x, mean, rstd, w, dx, dW, dB)
    rdx, tw, tb = ref_backward(dy, x, mean, rstd, w, 1)
    check_dx(dx, rdx, x, dy, w, mean, rstd, dtype)
    check_sum(dW, tw, (1, 2))
    check_sum(dB, tb, (1, 2))
