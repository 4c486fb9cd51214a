"""Orthogonalisation by Newton-Schulz products and the local Muon step, against the iteration in 64 bits.

Tolerances.  Simulating the iteration in 64 bits with every operand of a product rounded to 11 bits
(X carried with 22) gave 0.1e-3 to 1.6e-3 of the result's norm on Gaussian, 1/k, exponential, rank-8
and spiked spectra: 4e-3 is asked of precision f16, plus half a bf16 unit where the result is bf16.
The amplification seen there (1.6e-3 from roundings of 2.4e-4) on operands of 22 bits and fp32 sums of
up to a thousand terms gives below 1e-5 for full-rank matrices: 2e-5 is asked of precision f32.
Directions that a matrix does not have receive the rounding of X (22 bits: 1.2e-7 of its norm) times
the growth of small singular values (3.4445^5 = 485): 2e-4 there.
"""
import numpy as np
import pytest
import torch

import paper_2406_13936_b200 as pkg

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    c = pkg.Context(0)
    yield c
    c.close()


def ref_ns(G, steps=5, a=3.4445, b=-4.7750, c=2.0315, eps=1e-7):
    X = G.double()
    tall = X.shape[-2] > X.shape[-1]
    if tall:
        X = X.mT
    a, b, c, eps = (float(np.float32(v)) for v in (a, b, c, eps))
    X = X / (X.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.mT if tall else X


def matrices(seed, count, m, n, kind="gauss", scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    if kind == "gauss":
        return (torch.randn((count, m, n), generator=gen) * scale).cuda()
    k = min(m, n)
    U = torch.linalg.qr(torch.randn((count, m, k), generator=gen, dtype=torch.float64))[0]
    V = torch.linalg.qr(torch.randn((count, n, k), generator=gen, dtype=torch.float64))[0]
    i = torch.arange(1, k + 1, dtype=torch.float64)
    s = {"1/k": 1 / i, "exp": torch.exp(-i / max(1.0, k / 20)), "rank8": (i <= 8).double(),
         "spike": 0.01 + 10.0 * (i <= 4)}[kind]
    return ((U * s) @ V.mT * scale).float().cuda()


def orthogonalise(ctx, G, dst="f32", **kw):
    cfg = pkg.make_ns_cfg(**kw)
    count, m, n = G.shape
    O = torch.full(G.shape, 7.0, device="cuda", dtype=TYPES[dst])
    ctx.abs_orthogonalise(G, O, cfg, ctx.ns_scratch(count, m, n, cfg))
    return O


def check(got, want, tol, dst="f32"):
    for q in range(want.shape[0]):
        norm = want[q].norm().item()
        extra = 2.0 ** -9 if dst == "bf16" else 0.0
        err = (got[q].double() - want[q]).norm().item()
        assert err <= (tol + extra) * norm, (q, err / max(norm, 1e-300))


# one row, one column, one element, sides around the 8-, 64-, 128- and 256-wide pieces, both orientations,
# several matrices, more tiles than SMs
SHAPES = [(1, 1, 1), (2, 1, 7), (1, 9, 1), (3, 5, 5), (8, 10, 1024), (2, 33, 20), (1, 64, 64), (2, 64, 192), (1, 127, 128),
          (2, 128, 129), (1, 129, 127), (1, 200, 300), (1, 300, 200), (3, 257, 255), (1, 256, 512), (2, 384, 640),
          (1, 513, 1000), (1, 1000, 513), (2, 784, 1024), (1, 1024, 784), (5, 768, 768), (1, 1500, 1100), (40, 96, 260)]


@pytest.mark.parametrize("precision,tol", [("f16", 4e-3), ("f32", 2e-5)])
@pytest.mark.parametrize("count,m,n", SHAPES)
def test_shapes(ctx, count, m, n, precision, tol):
    G = matrices(1, count, m, n, scale=1e-3)
    check(orthogonalise(ctx, G, precision=precision), ref_ns(G), tol)


@pytest.fixture
def tiles(ctx):
    """Forces 128 x 128 tiles of single CTAs (1) or 256 x 256 tiles of pairs (2)."""
    yield lambda kind: ctx.set_tuning("ns_pair_tiles", kind)
    ctx.set_tuning("ns_pair_tiles", 0)


# sides just over and under the tiles' (a last block of 1, 2, 127 or 255 rows), far more tiles than CTAs
TILED = [(1, 129, 129), (2, 255, 257), (1, 257, 130), (3, 256, 256), (2, 383, 640), (1, 513, 2000), (1, 1500, 1100), (12, 770, 768),
         (30, 512, 300), (1, 2304, 2300)]


@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("count,m,n", TILED)
def test_both_tile_shapes(ctx, tiles, count, m, n, kind):
    tiles(kind)
    G = matrices(21, count, m, n, scale=1e-2)
    check(orthogonalise(ctx, G), ref_ns(G), 4e-3)


@pytest.mark.parametrize("kind", [1, 2])
def test_both_tile_shapes_repeat_their_bits_and_end_when_a_wait_runs_out(ctx, tiles, kind):
    tiles(kind)
    G = matrices(22, 3, 400, 700)
    want = orthogonalise(ctx, G)
    for _ in range(5):
        assert torch.equal(orthogonalise(ctx, G), want)
    ctx.set_tuning("stats_timeout_cycles", 200000)
    ctx.set_tuning("stats_fault_drop_loads", 1)
    try:
        lost = orthogonalise(ctx, G)
        torch.cuda.synchronize()
    finally:
        ctx.set_tuning("stats_fault_drop_loads", 0)
        ctx.set_tuning("stats_timeout_cycles", 0)
    assert torch.isnan(lost).all()
    assert torch.equal(orthogonalise(ctx, G), want)


# Short sides around what changes the layout of a small matrix: 16 (columns of a product), 32 and 64 (copies of B), 128;
# long sides with one CTA and clusters of 2 to 8, with a last CTA of few columns
# (and, the wide ones of the last row, clusters of 10, 11 and 16)
SMALL = [(7, 2048), (16, 250), (17, 259), (31, 513), (32, 1030), (33, 300), (64, 257), (64, 1799), (65, 140), (65, 260), (100, 90),
         (113, 400), (128, 1000), (128, 200), (18, 2474), (64, 4096), (86, 2085), (128, 2048), (97, 1300)]


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("m,n", SMALL)
def test_small_matrices_in_wider_rows(ctx, m, n, tall, pad, src):
    """Their products have split operands at either precision."""
    if tall:
        m, n = n, m
    G = matrices(23, 3, m, n).to(TYPES[src])
    wide = torch.full((3, m, n + pad), 5.0, device="cuda", dtype=TYPES[src])
    wide[:, :, :n] = G
    out = torch.full((3, m, n + pad), 5.0, device="cuda")
    cfg = pkg.make_ns_cfg()
    ctx.abs_orthogonalise(wide[:, :, :n], out[:, :, :n], cfg, ctx.ns_scratch(3, m, n, cfg))
    check(out[:, :, :n], ref_ns(G), 2e-5)
    assert bool((out[:, :, n:] == 5.0).all()) and torch.equal(wide[:, :, :n], G)
    again = torch.empty_like(G, dtype=torch.float32)
    ctx.abs_orthogonalise(G, again, cfg, ctx.ns_scratch(3, m, n, cfg))
    assert torch.equal(again, out[:, :, :n])                   # alignment changes the loads, not the result


@pytest.mark.parametrize("src", ["f32", "bf16"])
@pytest.mark.parametrize("dst", ["f32", "bf16"])
@pytest.mark.parametrize("precision,tol", [("f16", 4e-3), ("f32", 2e-5)])
def test_types(ctx, src, dst, precision, tol):
    G = matrices(2, 2, 190, 330).to(TYPES[src])
    check(orthogonalise(ctx, G, dst, precision=precision), ref_ns(G), tol, dst)


@pytest.mark.parametrize("kind", ["1/k", "exp", "rank8", "spike"])
@pytest.mark.parametrize("m,n", [(256, 256), (320, 512), (512, 320)])
def test_spectra(ctx, kind, m, n):
    G = matrices(3, 2, m, n, kind)
    want = ref_ns(G)
    check(orthogonalise(ctx, G), want, 4e-3)
    check(orthogonalise(ctx, G, precision="f32"), want, 2e-5 if kind == "1/k" else 2e-4)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e6, 1e30])
def test_scales(ctx, scale):
    """The range of fp32 gradients does not reach the fp16 operands (eps small enough to matter nowhere)."""
    G = matrices(4, 2, 100, 150, scale=scale)
    check(orthogonalise(ctx, G, eps=1e-38), ref_ns(G, eps=1e-38), 4e-3)
    check(orthogonalise(ctx, G, eps=1e-38, precision="f32"), ref_ns(G, eps=1e-38), 2e-5)


@pytest.mark.parametrize("kw", [dict(steps=1), dict(steps=3), dict(steps=10), dict(steps=8, a=1.5, b=-0.5, c=0.0),
                                dict(steps=5, a=2.0, b=-1.5, c=0.5), dict(steps=2, a=1.0, b=0.0, c=0.0)])
def test_coefficients(ctx, kw):
    G = matrices(5, 1, 140, 260)
    check(orthogonalise(ctx, G, **kw), ref_ns(G, **kw), 4e-3)
    check(orthogonalise(ctx, G, precision="f32", **kw), ref_ns(G, **kw), 2e-5)


def test_the_result_is_nearly_orthogonal(ctx):
    O = orthogonalise(ctx, matrices(6, 1, 300, 700)).double()
    s = torch.linalg.svdvals(O[0])
    assert s.min().item() > 0.5 and s.max().item() < 1.3


@pytest.mark.parametrize("m,n", [(150, 260), (260, 150)])
def test_strides_in_place_and_zero_rows(ctx, m, n):
    G = matrices(7, 3, m, n)
    G[:, 3] = 0.0
    G[:, :, n - 2] = 0.0
    want = ref_ns(G)
    cfg = pkg.make_ns_cfg()
    scratch = ctx.ns_scratch(3, m, n, cfg)
    wide = torch.full((3, m + 2, n + 3), 7.0, device="cuda")
    view = wide[:, 1:1 + m, 2:2 + n]
    view.copy_(G)
    ctx.abs_orthogonalise(view, view, cfg, scratch)          # in place, rows inside wider rows
    check(view, want, 4e-3)
    assert not view[:, 3].any() and not view[:, :, n - 2].any()
    assert bool((wide[:, 0] == 7.0).all()) and bool((wide[:, :, :2] == 7.0).all()) and bool((wide[:, :, 2 + n:] == 7.0).all())
    O = torch.empty((m, n), device="cuda")
    ctx.abs_orthogonalise(G[0], O, cfg, scratch)             # one matrix
    check(O[None], want[:1], 4e-3)


def test_zero_and_non_finite_matrices(ctx):
    G = matrices(8, 5, 70, 140)
    G[1] = 0.0
    G[2, 5, 7] = float("nan")
    G[3, 0, 0] = float("inf")
    O = orthogonalise(ctx, G)
    want = ref_ns(G)
    assert not O[1].any()
    assert torch.isnan(O[2]).all() and torch.isnan(O[3]).all()
    check(O[[0, 4]], want[[0, 4]], 4e-3)
    assert torch.isnan(orthogonalise(ctx, G[1:2], eps=0.0)).all()


def test_groups_give_the_same_bits(ctx):
    """More matrices than are worked on together: each as if alone, and repeatable."""
    G = matrices(9, 130, 300, 520)
    cfg = pkg.make_ns_cfg(precision="f32")
    one, all_ = (ctx.ns_scratch(k, 300, 520, cfg).numel() for k in (1, 130))
    assert all_ < 0.6 * 130 * one                            # two groups
    O = orthogonalise(ctx, G, precision="f32")
    assert torch.equal(O, orthogonalise(ctx, G, precision="f32"))
    for q in (0, 64, 65, 129):
        assert torch.equal(O[q:q + 1], orthogonalise(ctx, G[q:q + 1], precision="f32"))


def replicas(seed, M, L, m, n, pad, scale=1.0, kind="gauss"):
    size = m * n
    flat = torch.full((M, L * (size + pad) + 11), 7.0, device="cuda")
    view = torch.as_strided(flat, (M, L, m, n), (flat.stride(0), size + pad, n, 1))
    view.copy_(matrices(seed, M * L, m, n, kind, scale).view(M, L, m, n))
    return view, flat


MUON = [(1, 1, 1, 1, 0), (4, 1, 64, 192, 0), (2, 3, 50, 30, 5), (8, 1, 10, 1024, 0), (3, 2, 129, 257, 0), (2, 2, 300, 128, 3),
        (8, 2, 256, 256, 0), (1, 5, 384, 200, 0)]


@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("M,L,m,n,pad", MUON)
def test_muon_step(ctx, M, L, m, n, pad, nesterov, average):
    lr, mu, wd, scale = 0.02, 0.95, 0.1, 0.2 * max(m, n) ** 0.5
    X, xf = replicas(1, M, L, m, n, pad, 0.02)
    B, bf = replicas(2, M, L, m, n, pad, 5e-3)
    G, gf = replicas(3, M, L, m, n, pad, 1e-3)
    x0, b0, g0 = X.double(), B.double(), gf.clone()
    b1 = mu * b0 + G.double()
    u = G.double() + mu * b1 if nesterov else b1
    O = ref_ns(u.reshape(M * L, m, n)).reshape(X.shape)
    x1 = (1 - lr * wd) * x0 - lr * scale * O
    if average:
        x1 = x1.mean(0, keepdim=True).expand_as(x1)
    cfg = pkg.make_muon_cfg(lr, mu, wd, scale, nesterov)
    ctx.local_muon_step(X, B, G, cfg, ctx.ns_scratch(M * L, m, n, cfg.ns), average_after=average)
    assert (B.double() - b1).norm().item() <= 2.0 ** -23 * 2 * b1.norm().item()
    assert (X.double() - x1).norm().item() <= lr * scale * 4e-3 * O.norm().item() + 2.0 ** -22 * x1.norm().item()
    if average:
        for k in range(1, M):
            assert torch.equal(X[0], X[k])
    assert torch.equal(gf, g0)
    for view, flat in ((X, xf), (B, bf)):                     # what lies between the matrices is untouched
        view.fill_(7.0)
        assert bool((flat == 7.0).all())


def test_muon_f32_precision_and_many_groups(ctx):
    M, L, m, n = 4, 32, 300, 520
    X, _ = replicas(1, M, L, m, n, 0, 0.02)
    B, _ = replicas(2, M, L, m, n, 0, 5e-3)
    G, _ = replicas(3, M, L, m, n, 0, 1e-3)
    x0, b0 = X.double(), B.double()
    b1 = 0.9 * b0 + G.double()
    O = ref_ns((0.9 * b1 + G.double()).reshape(M * L, m, n)).reshape(X.shape)
    x1 = (x0 - 0.1 * O).mean(0, keepdim=True).expand_as(x0)
    cfg = pkg.make_muon_cfg(0.1, 0.9, 0.0, 1.0, True, pkg.make_ns_cfg(precision="f32"))
    ctx.local_muon_step(X, B, G, cfg, ctx.ns_scratch(M * L, m, n, cfg.ns), average_after=True)
    assert (X.double() - x1).norm().item() <= 0.1 * 2e-5 * O.norm().item() + 2.0 ** -22 * x1.norm().item()


def test_on_another_stream_and_in_a_graph(ctx):
    G = matrices(11, 3, 200, 333)
    cfg = pkg.make_ns_cfg()
    scratch, O = ctx.ns_scratch(3, 200, 333, cfg), torch.empty_like(G)
    want = orthogonalise(ctx, G)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.abs_orthogonalise(G, O, cfg, scratch)
    side.synchronize()
    assert torch.equal(O, want)
    O.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.abs_orthogonalise(G, O, cfg, scratch)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(O, want)
    G.copy_(matrices(12, 3, 200, 333))
    graph.replay()
    torch.cuda.synchronize()
    check(O, ref_ns(G), 4e-3)


@pytest.mark.parametrize("precision", ["f16", "f32"])
@pytest.mark.parametrize("m,n", [(64, 96), (400, 700)])
def test_a_wait_that_runs_out_gives_nan_and_passes(ctx, precision, m, n):
    """No operand tile is ever loaded (a test hook on the host side): the waits end by their limit."""
    G = matrices(13, 2, m, n)
    ctx.set_tuning("stats_timeout_cycles", 200000)
    ctx.set_tuning("stats_fault_drop_loads", 1)
    try:
        O = orthogonalise(ctx, G, precision=precision)
        torch.cuda.synchronize()
    finally:
        ctx.set_tuning("stats_fault_drop_loads", 0)
        ctx.set_tuning("stats_timeout_cycles", 0)
    assert torch.isnan(O).all()
    check(orthogonalise(ctx, G, precision=precision), ref_ns(G), 4e-3)


def test_refusals(ctx):
    G = matrices(14, 2, 30, 40)
    cfg = pkg.make_ns_cfg()
    scratch = ctx.ns_scratch(2, 30, 40, cfg)
    O = torch.empty_like(G)
    for bad in (lambda: ctx.abs_orthogonalise(G, O, pkg.make_ns_cfg(steps=0), scratch),
                lambda: ctx.abs_orthogonalise(G, O, pkg.make_ns_cfg(steps=33), scratch),
                lambda: ctx.abs_orthogonalise(G, O, pkg.make_ns_cfg(eps=-1.0), scratch),
                lambda: ctx.abs_orthogonalise(G, O, pkg.make_ns_cfg(a=float("nan")), scratch),
                lambda: ctx.abs_orthogonalise(G, O, pkg.make_ns_cfg(a=100.0), scratch),          # singular values blow up
                lambda: ctx.abs_orthogonalise(G, O, cfg, scratch[:1000]),
                lambda: ctx.abs_orthogonalise(G, O[:, :, :20], cfg, scratch),
                lambda: ctx.abs_orthogonalise(G.half(), O, cfg, scratch),
                lambda: ctx.abs_orthogonalise(G.mT, O.mT, cfg, scratch),
                lambda: ctx.abs_orthogonalise(G[:1].expand(2, 30, 40), O, cfg, scratch),
                lambda: ctx.ns_scratch(0, 30, 40, cfg),
                lambda: ctx.ns_scratch(1, 30, 0, cfg)):
        with pytest.raises(pkg.AbsError):
            bad()
    X = G.view(2, 1, 30, 40)
    muon = pkg.make_muon_cfg(0.1)
    for bad in (lambda: ctx.local_muon_step(X, X.clone(), X.clone()[:, :, :, :20], muon, scratch),
                lambda: ctx.local_muon_step(X.bfloat16(), X, X, muon, scratch),
                lambda: ctx.local_muon_step(X, X.clone(), X.clone(), pkg.make_muon_cfg(0.1, momentum=1.0), scratch),
                lambda: ctx.local_muon_step(X, X.clone(), X.clone(), pkg.make_muon_cfg(float("inf")), scratch),
                lambda: ctx.local_muon_step(X, X.clone(), X.clone(), muon, scratch[:64])):
        with pytest.raises(pkg.AbsError):
            bad()


@pytest.mark.parametrize("m,n,precision,most,fewer", [(300, 520, "f32", 98, (97, 60, 1)), (768, 768, "f16", 36, (35, 2)),
                                                      (64, 4000, "f16", 33, (32, 5)), (200, 140, "f32", 3, (2, 1))])
def test_scratch_for_some_number_serves_every_smaller_one(ctx, m, n, precision, most, fewer):
    """Past one group the scratch of one matrix more is that of half as many: 98 of 300 x 520 ask for 106 MB, 97 for 209."""
    cfg = pkg.make_ns_cfg(steps=2, precision=precision)
    scratch = ctx.ns_scratch(most, m, n, cfg)
    G = matrices(41, 2, m, n).repeat(most // 2 + 1, 1, 1)
    for count in (most,) + fewer:
        O = torch.full((count, m, n), 7.0, device="cuda")
        ctx.abs_orthogonalise(G[:count], O, cfg, scratch)
        check(O[:2], ref_ns(G[:min(2, count)], steps=2), 4e-3 if precision == "f16" else 2e-5)
        assert torch.equal(O, O[:2].repeat(count // 2 + 1, 1, 1)[:count])


def test_less_scratch_makes_smaller_groups(ctx):
    cfg = pkg.make_ns_cfg(precision="f32")
    G = matrices(42, 7, 200, 300)
    want = orthogonalise(ctx, G, precision="f32")
    one, three = (ctx.ns_scratch(k, 200, 300, cfg) for k in (1, 3))
    for scratch in (one, three, three[:-1]):
        O = torch.empty_like(G)
        ctx.abs_orthogonalise(G, O, cfg, scratch)
        assert torch.equal(O, want)
    X, Buf, Gb = (matrices(k, 7, 200, 300).view(7, 1, 200, 300) for k in (43, 44, 45))
    muon = pkg.make_muon_cfg(0.1, ns=cfg)
    X2, Buf2 = X.clone(), Buf.clone()
    ctx.local_muon_step(X, Buf, Gb, muon, one, average_after=True)
    ctx.local_muon_step(X2, Buf2, Gb, muon, ctx.ns_scratch(7, 200, 300, cfg), average_after=True)
    assert torch.equal(X, X2) and torch.equal(Buf, Buf2)
    with pytest.raises(pkg.AbsError, match="scratch"):
        ctx.abs_orthogonalise(G, torch.empty_like(G), cfg, one[:-1])


@pytest.mark.parametrize("m,n", [(18, 2474), (64, 4096), (2048, 128), (97, 1300)])
def test_clusters_that_the_device_does_not_hold(ctx, m, n):
    """Without clusters beyond 8 CTAs such matrices take the general path, with the scratch that was asked for."""
    G = matrices(46, 3, m, n)
    want = ref_ns(G)
    cfg = pkg.make_ns_cfg(precision="f32")
    ctx.set_tuning("ns_max_cluster", 8)
    try:
        O = orthogonalise(ctx, G, precision="f32")
        X, Buf = G.clone().unsqueeze(1), torch.zeros_like(G).unsqueeze(1)
        ctx.local_muon_step(X, Buf, G.unsqueeze(1), pkg.make_muon_cfg(1.0, nesterov=False, ns=cfg), ctx.ns_scratch(3, m, n, cfg))
    finally:
        ctx.set_tuning("ns_max_cluster", 0)
    check(O, want, 2e-5)
    check(G - X[:, 0], want, 2e-5 + 2.0 ** -22 * (G.norm() / want.norm()).item())
    check(orthogonalise(ctx, G, precision="f32"), want, 2e-5)
    for bad in (7, 17):
        with pytest.raises(pkg.AbsError):
            ctx.set_tuning("ns_max_cluster", bad)


@pytest.mark.parametrize("count,m,n", [(100, 128, 500), (90, 10, 1024), (50, 64, 1000), (40, 100, 700), (300, 24, 40), (32, 18, 2474),
                                       (33, 18, 2474), (4, 128, 2048), (5, 128, 2048)])
def test_more_small_matrices_than_fit_at_a_time(ctx, count, m, n):
    """Clusters of 4 to 16 CTAs in several waves; numbers on either side of what sends wide ones to the general path."""
    G = matrices(47, count, m, n)
    O = orthogonalise(ctx, G, precision="f32")
    check(O, ref_ns(G), 2e-5)
    assert torch.equal(O, orthogonalise(ctx, G, precision="f32"))
    X, Buf, Gb = G.view(count, 1, m, n).clone(), torch.zeros((count, 1, m, n), device="cuda"), G.view(count, 1, m, n)
    cfg = pkg.make_muon_cfg(1.0, nesterov=False, ns=pkg.make_ns_cfg(precision="f32"))
    ctx.local_muon_step(X, Buf, Gb, cfg, ctx.ns_scratch(count, m, n, cfg.ns))
    assert torch.equal(Buf[:, 0], G) and torch.equal(X[:, 0], G - O)
