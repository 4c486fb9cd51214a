"""Root-mean-square norm with the residual's addition against its definition in 64 bits.

u = 2^-24, w = 2^-8 (bf16): the largest relative error of a rounding.  A sum of d squares in any order is off by at most d u; rstd has
half of that and a few roundings: (d / 2 + 8) u.  y has rstd's and three roundings more, and the output's.  A sum of n products with terms
off by k u each is off by (n + k) u times the sum of magnitudes.
"""
import math

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


def half_step(x, dtype):
    return x.abs() * (W if dtype == torch.bfloat16 else U)


def rows_of(gen, M, rows, d, pad, dtype, scale=1.0):
    full = scale * torch.randn((M, rows, d + pad), device="cuda", generator=gen) + 0.3
    return full.to(TYPES[dtype])[:, :, :d]


SHAPES = [(1, 1, 1, 0), (1, 1, 5, 0), (2, 3, 8, 0), (1, 7, 64, 8), (3, 5, 257, 0), (2, 9, 768, 0), (1, 300, 768, 8), (8, 17, 96, 3),
          (1, 4, 1000, 0), (1, 3, 4096, 0), (2, 2, 5000, 1), (1, 2, 8192, 0), (1, 2, 12800, 0), (1, 2, 20000, 0), (1, 2000, 40, 0),
          (4, 700, 1024, 0), (1, 3, 1021, 10), (2, 50, 2050, 2)]


@pytest.mark.parametrize("M,rows,d,pad", SHAPES)
@pytest.mark.parametrize("dtype,residual,quant", [("f32", True, False), ("bf16", False, False), ("bf16", True, True), ("f32", False, True),
                                                  ("bf16", True, False)])
def test_forward(ctx, M, rows, d, pad, dtype, residual, quant):
    gen = torch.Generator(device="cuda").manual_seed(d + rows)
    x = rows_of(gen, M, rows, d, pad, dtype)
    r = rows_of(gen, M, rows, d, 2 * pad, dtype, 2.0) if residual else None
    w = (1.0 + 0.2 * torch.randn((M, d + 5), device="cuda", generator=gen))[:, :d]
    h = torch.empty((M, rows, d), device="cuda", dtype=TYPES[dtype]) if residual else None
    y = torch.empty((M, rows, d + pad), device="cuda", dtype=TYPES[dtype])[:, :, :d]
    q = torch.empty((M, rows, d), device="cuda", dtype=torch.float8_e4m3fn) if quant else None
    rstd, scales = (torch.empty((M, rows), device="cuda") for _ in range(2))
    assert ctx.abs_rms_norm(x, w, 1e-6, y, residual=r, summed=h, rstd=rstd, Q=q, scales=scales if quant else None) is y
    hh = x.double()
    if residual:
        hh = (x.float() + r.float()).to(TYPES[dtype])
        assert torch.equal(h, hh)
        hh = hh.double()
    root = (hh.square().mean(2) + 1e-6).rsqrt()
    assert ((rstd.double() - root).abs() <= (d / 2 + 8) * U * root).all()
    want = hh * root[:, :, None] * w.double()[:, None]
    slack = (d / 2 + 12) * U * want.abs()
    assert ((y.double() - want).abs() <= slack + half_step(want, y.dtype)).all()
    if quant:
        top = want.abs().amax(2)
        assert ((scales.double() - top / 448).abs() <= (d / 2 + 14) * U * top / 448).all()
        scaled = want / scales.double()[:, :, None]
        # half a step of e4m3 is 2^-4 of the value, below 2^-6 half of 2^-9
        step = torch.clamp(scaled.abs() * 2.0 ** -4, min=2.0 ** -10)
        assert ((q.double() - scaled).abs() <= step + (d / 2 + 14) * U * scaled.abs()).all()


def check_backward(dy, h, dh, rstd, w, samples, dx, dw, gw):
    M, rows, d = h.shape
    g, hh, rs = dy.double(), h.double(), rstd.double()[:, :, None]
    xh = hh * rs
    a = g * (w.double()[:, None] if w is not None else 1.0)
    c = (a * xh).mean(2, keepdim=True)
    want = rs * (a - xh * c)
    slack = rs * ((8 * U) * a.abs() + xh.abs() * (d + 12) * U * (a * xh).abs().mean(2, keepdim=True))
    if dh is not None:
        want = want + dh.double()
        slack = slack + U * (dh.double().abs() + want.abs())
    if dx is not None:
        assert ((dx.double() - want).abs() <= slack + half_step(want, dx.dtype) + 1e-38).all()
    terms = (g * xh).view(M, samples, -1, d)
    n = terms.shape[2]
    if gw is not None:
        assert ((gw.double() - terms.sum(2)).abs() <= (n + 4) * U * terms.abs().sum(2) + 1e-38).all()
    if dw is not None:
        assert ((dw.double() - terms.sum((1, 2))).abs() <= (n * samples + 4) * U * terms.abs().sum((1, 2)) + 1e-38).all()


BACKWARD = [(1, 1, 1, 1, 0), (1, 1, 1, 8, 0), (2, 8, 1, 257, 0), (2, 3, 5, 64, 8), (1, 16, 300, 768, 0), (8, 4, 100, 768, 8), (3, 500, 2, 96, 0),
            (1, 1, 3000, 1024, 0), (1, 2, 37, 4096, 0), (1, 3, 7, 5000, 1), (2, 1, 9, 8192, 0), (1, 2, 3, 20000, 0), (1, 1000, 1, 40, 0),
            (2, 13, 11, 1021, 10), (1, 5, 64, 2050, 2), (1, 2, 200, 40, 0)]


@pytest.mark.parametrize("M,S,T,d,pad", BACKWARD)
@pytest.mark.parametrize("dtype,residual,what", [("f32", False, "dx dw gw"), ("bf16", True, "dx dw gw"), ("bf16", False, "dx dw"),
                                                 ("f32", True, "gw"), ("bf16", True, "dx"), ("f32", False, "dw")])
def test_backward(ctx, M, S, T, d, pad, dtype, residual, what):
    gen = torch.Generator(device="cuda").manual_seed(d + S)
    h, dy = rows_of(gen, M, S * T, d, pad, dtype), rows_of(gen, M, S * T, d, 0, dtype)
    dh = rows_of(gen, M, S * T, d, pad, dtype) if residual else None
    rstd = (h.double().square().mean(2) + 1e-6).rsqrt().float()
    w = (1.0 + 0.2 * torch.randn((M, d + 3), device="cuda", generator=gen))[:, :d]
    dx = torch.full((M, S * T, d + pad), 9.0, device="cuda", dtype=TYPES[dtype])[:, :, :d] if "dx" in what else None
    dw = torch.full((M, d + 7), 9.0, device="cuda")[:, :d] if "dw" in what else None
    gw = torch.full((M, S, d + 4), 9.0, device="cuda")[:, :, :d] if "gw" in what else None
    ctx.abs_rms_norm_backward(dy, h, rstd, w, dx, dH=dh, dW=dw, samples=S, Gw=gw)
    check_backward(dy, h, dh, rstd, w, S, dx, dw, gw)
    again = [t.clone() for t in (dx, dw, gw) if t is not None]
    ctx.abs_rms_norm_backward(dy, h, rstd, w, dx, dH=dh, dW=dw, samples=S, Gw=gw)
    assert all(torch.equal(x, y) for x, y in zip(again, [t for t in (dx, dw, gw) if t is not None]))


@pytest.mark.parametrize("workspace", [1 << 12, 1 << 16, 1 << 20])
@pytest.mark.parametrize("S,T", [(1, 4000), (7, 500), (3000, 2)])
def test_backward_with_a_small_workspace(workspace, S, T):
    c = pkg.Context(0, workspace)
    gen = torch.Generator(device="cuda").manual_seed(1)
    h, dy = rows_of(gen, 2, S * T, 200, 0, "f32"), rows_of(gen, 2, S * T, 200, 0, "f32")
    rstd = (h.double().square().mean(2) + 1e-6).rsqrt().float()
    dw, gw = torch.empty((2, 200), device="cuda"), torch.empty((2, S, 200), device="cuda")
    c.abs_rms_norm_backward(dy, h, rstd, None, None, dW=dw, samples=S, Gw=gw)
    check_backward(dy, h, None, rstd, None, S, None, dw, gw)
    c.abs_rms_norm_backward(dy, h, rstd, None, None, dW=dw)
    check_backward(dy, h, None, rstd, None, S, None, dw, None)
    c.close()


@pytest.mark.parametrize("dtype,d", [("bf16", 768), ("f32", 768), ("bf16", 77), ("f32", 20000)])
def test_in_place(ctx, dtype, d):
    """The sum in the residual's or the branch's place, y in x's; dx in dy's, h's or dh's."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, r = rows_of(gen, 2, 33, d, 0, dtype), rows_of(gen, 2, 33, d, 0, dtype)
    w = 1.0 + 0.2 * torch.randn((2, d), device="cuda", generator=gen)
    y, h, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty((2, 33), device="cuda")
    ctx.abs_rms_norm(x, w, 1e-6, y, residual=r, summed=h, rstd=rstd)
    for place in ("residual", "x"):
        x2, r2 = x.clone(), r.clone()
        y2 = torch.empty_like(y)
        ctx.abs_rms_norm(x2, w, 1e-6, y2, residual=r2, summed=r2 if place == "residual" else x2)
        assert torch.equal(y2, y) and torch.equal(r2 if place == "residual" else x2, h)
    x2, r2 = x.clone(), r.clone()
    ctx.abs_rms_norm(x2, w, 1e-6, x2, residual=r2, summed=r2)
    assert torch.equal(x2, y) and torch.equal(r2, h)
    h2 = h.clone()
    ctx.abs_rms_norm(h2, w, 1e-6, h2)
    assert torch.equal(h2, y)
    dy, dh = rows_of(gen, 2, 33, d, 0, dtype), rows_of(gen, 2, 33, d, 0, dtype)
    dx, dw = torch.empty_like(dy), torch.empty((2, d), device="cuda")
    ctx.abs_rms_norm_backward(dy, h, rstd, w, dx, dH=dh, dW=dw)
    for place in range(3):
        t = [dy.clone(), h.clone(), dh.clone()]
        dw2 = torch.empty_like(dw)
        ctx.abs_rms_norm_backward(t[0], t[1], rstd, w, t[place], dH=t[2], dW=dw2)
        assert torch.equal(t[place], dx) and torch.equal(dw2, dw)


@pytest.mark.parametrize("d", [64, 77])
def test_zeros_infinities_and_nan(ctx, d):
    x = torch.randn((1, 5, d), device="cuda")
    x[0, 1] = 0.0
    x[0, 2, 3] = math.inf
    x[0, 3, 3] = math.nan
    q, s = torch.empty(x.shape, device="cuda", dtype=torch.uint8), torch.empty((1, 5), device="cuda")
    y = torch.empty_like(x)
    ctx.abs_rms_norm(x, None, 0.0, y, Q=q, scales=s)
    values = q.view(torch.float8_e4m3fn).float()
    assert s[0, 1].isnan() or s[0, 1] == 1.0          # eps = 0: 0 / 0
    ctx.abs_rms_norm(x, None, 1e-6, y, Q=q, scales=s)
    values = q.view(torch.float8_e4m3fn).float()
    assert s[0, 1] == 1.0 and (values[0, 1] == 0).all() and (y[0, 1] == 0).all()
    for row in (2, 3):
        assert s[0, row].isnan() and values[0, row].isnan().all()
    for row in (0, 4):
        assert values[0, row].abs().max() == 448.0 and torch.isfinite(y[0, row]).all()


def test_nothing_to_do(ctx):
    dw, gw = torch.full((2, 10), 3.0, device="cuda"), torch.full((2, 4, 10), 3.0, device="cuda")
    none = torch.empty((2, 0, 10), device="cuda")
    stats = torch.empty((2, 0), device="cuda")
    ctx.abs_rms_norm(none, None, 1e-6, none)
    ctx.abs_rms_norm_backward(none, none, stats, None, None, dW=dw, samples=4, Gw=gw)
    assert (dw == 0).all() and (gw == 0).all()


def test_per_sample_rows_feed_the_statistics(ctx):
    """Gw as rows of abs_test_stats: the mean is dW / samples."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    M, S, T, d = 2, 12, 20, 256
    h, dy = rows_of(gen, M, S * T, d, 0, "bf16"), rows_of(gen, M, S * T, d, 0, "bf16")
    rstd = (h.double().square().mean(2) + 1e-6).rsqrt().float()
    dw, gw = torch.empty((M, d), device="cuda"), torch.empty((M, S, d), device="cuda")
    ctx.abs_rms_norm_backward(dy, h, rstd, None, None, dW=dw, samples=S, Gw=gw)
    gbar = torch.empty((M, d), device="cuda")
    stats = ctx.abs_test_stats(gw, ctx.new_stats(M), gbar)
    assert ((gbar - dw / S).abs() <= 2 * S * U * gw.abs().mean(1)).all()
    for m, rec in enumerate(pkg.stats_to_dicts(stats)):
        assert abs(rec["var_norm"] - gw[m].double().var(0).sum().item()) <= 1e-5 * rec["var_norm"]


def test_capture(ctx):
    gen = torch.Generator(device="cuda").manual_seed(4)
    h, dy = rows_of(gen, 2, 640, 768, 0, "bf16"), rows_of(gen, 2, 640, 768, 0, "bf16")
    w = torch.ones((2, 768), device="cuda")
    y, rstd = torch.empty_like(h), torch.empty((2, 640), device="cuda")
    dx, dw, gw = torch.empty_like(h), torch.empty((2, 768), device="cuda"), torch.empty((2, 10, 768), device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()

    def both():
        ctx.abs_rms_norm(h, w, 1e-6, y, rstd=rstd)
        ctx.abs_rms_norm_backward(dy, h, rstd, w, dx, dW=dw, samples=10, Gw=gw)

    with torch.cuda.stream(stream):
        both()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            both()
    for _ in range(2):
        h.copy_(torch.randn_like(h))
        graph.replay()
        torch.cuda.synchronize()
        check_backward(dy, h, None, rstd, w, 10, dx, dw, gw)


@pytest.mark.parametrize("d", [768, 77])
def test_rows_far_apart(ctx, d):
    """Elements behind the 2^31-st of a tensor: the same bits as from rows that lie together."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    rows, apart = 520, 1 << 22
    x = torch.randn((rows, d), device="cuda", generator=gen).bfloat16()
    w = torch.rand(d, device="cuda", generator=gen)
    far_x, far_y, far_dx = (torch.empty((rows, apart), device="cuda", dtype=torch.bfloat16)[:, -((d + 7) // 8 * 8):][:, :d] for _ in range(3))
    far_x.copy_(x)
    got = []
    for a, y, dx in ((x, torch.empty_like(x), torch.empty_like(x)), (far_x, far_y, far_dx)):
        rstd, dw = torch.empty((1, rows), device="cuda"), torch.empty((1, d), device="cuda")
        ctx.abs_rms_norm(a, w, 1e-6, y, rstd=rstd)
        ctx.abs_rms_norm_backward(y, a, rstd, w, dX=dx, dW=dw)
        got.append((y, rstd, dx))
    assert all(torch.equal(p, q) for p, q in zip(*got))


LEAST = 2.0 ** -149                                  # the least positive fp32


@pytest.mark.parametrize("d", [64, 258, 1021, 20000])
@pytest.mark.parametrize("residual", [False, True])
def test_8_bits_of_rows_of_very_small_values(ctx, d, residual):
    """Largest values from 1 down to the least positive fp32, zeros beside them: with y as it was written, scales and Q are the
    quotients in fp32, bit for bit, and a scale that would round to zero is the least positive number instead."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    tops = [1.0, 1e-30, 5e-36, 1.2e-36, 1e-36, 1e-37, 1e-39, 1e-41, 1e-42] + [k * LEAST for k in (1, 100, 223, 224, 225, 448, 700)]
    M = len(tops)
    x = 2.0 * torch.rand((M, 3, d), device="cuda", generator=gen) - 1.0
    x[:, :, ::3] = 0.0
    x[:, 2] = 0.0
    r = torch.zeros_like(x) if residual else None
    w = torch.tensor(tops, device="cuda", dtype=torch.float64).float()[:, None].expand(M, d).contiguous()
    y, q = torch.empty_like(x), torch.empty((M, 3, d), device="cuda", dtype=torch.float8_e4m3fn)
    s, h = torch.empty((M, 3), device="cuda"), torch.empty_like(x) if residual else None
    ctx.abs_rms_norm(x, w, 1e-6, y, residual=r, summed=h, Q=q, scales=s)
    top = y.abs().amax(2)
    assert (top[:, :2] > 0).all()
    want = (top.cpu() / 448.0).clamp_(min=LEAST).cuda()
    want[top == 0] = 1.0
    assert torch.equal(s, want)
    scaled = (y.cpu() / want.cpu()[:, :, None]).clamp_(-448.0, 448.0)
    assert torch.equal(q.cpu().float(), scaled.to(torch.float8_e4m3fn).float())


@pytest.mark.parametrize("d", [64, 1021, 20000])
def test_8_bits_of_small_bf16_rows(ctx, d):
    """Subnormal bf16 rows with eps = 0 are of order one; with small weights they are finite, zeros stay zeros."""
    gen = torch.Generator(device="cuda").manual_seed(d + 1)
    x = torch.randn((1, 4, d), device="cuda", generator=gen).bfloat16()
    x[:, :, 1::2] = 0.0
    w = torch.full((1, d), 1e-37, device="cuda")
    q, s = torch.empty((1, 4, d), device="cuda", dtype=torch.float8_e4m3fn), torch.empty((1, 4), device="cuda")
    ctx.abs_rms_norm(x, w, 1e-6, None, Q=q, scales=s)
    v = x.double()
    want = v * (v.square().mean(2, keepdim=True) + 1e-6).rsqrt() * w.double()
    got = q.double() * s.double()[:, :, None]
    assert torch.isfinite(got).all() and (got[:, :, 1::2] == 0).all()
    # the scale is a subnormal number of steps of 2^-149; half a step of e4m3 is 2^-4 of the value, below 2^-6 scales half of 2^-9; y is off by
    # its own roundings and by a step of 2^-149
    top = want.abs().amax(2, keepdim=True)
    assert ((s.double() - top[:, :, 0] / 448).abs() <= LEAST + (d / 2 + 14) * U * top[:, :, 0] / 448).all()
    lost = (want.abs() - 448 * s.double()[:, :, None]).clamp(min=0)                # (what a scale that was rounded down leaves out)
    step = torch.maximum(want.abs() * 2.0 ** -4, s.double()[:, :, None] * 2.0 ** -10)
    assert ((got - want).abs() <= step + lost + (d / 2 + 16) * U * want.abs() + 2 * LEAST).all()


@pytest.mark.parametrize("d", [64, 77, 20000])
def test_a_row_of_zeros_without_eps_is_nan(ctx, d):
    """0 / 0: y, the scale and the row in 8 bits are NaN; its neighbours are as ever."""
    x = torch.ones((1, 3, d), device="cuda")
    x[0, 1] = 0.0
    q, s, y = torch.empty(x.shape, device="cuda", dtype=torch.float8_e4m3fn), torch.empty((1, 3), device="cuda"), torch.empty_like(x)
    ctx.abs_rms_norm(x, None, 0.0, y, Q=q, scales=s)
    for t in (y, q.float(), s.unsqueeze(2)):
        assert t[0, 1].isnan().all() and torch.isfinite(t[0, ::2]).all()
