"""Causal attention over packed sequences against its definition in 64 bits.

Tolerances are sums of absolute values, element by element, with u = 2^-24 (fp32) and w = 2^-8 (bf16), the largest relative error
of a rounding:
  scores        a dot product of hd terms in fp32 is off by at most (hd + 2) u sum |q k|; the exponent carries that, and the
                rounding of its argument (magnitude up to 2 max |s|), so a weight p is off by e_p = that + 8 u relative to itself
  o             sum_j p |v| (2 e_p + n u), and w sum_j p |v| where the weights are rounded to bf16 for the tensor cores
  ds            p (|dp - delta| e_p + (hd + 2) u (sum |do v| + sum |do o|)), and w |ds| where it is rounded to bf16
  sums over n rows or keys: n u times the sum of magnitudes
and half a step of the output's type.  Sums of n terms are taken to be off by n u, which no order of additions exceeds.
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


class Batch:
    """Packed inputs: `front` rows before the first sequence, `tail` behind the last, views of one fused tensor."""

    def __init__(self, lens, hq, hk, hd, dtype, seed=0, front=0, tail=0, amp=1.0, pad=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.hq, self.hk, self.hd, self.dtype = lens, hq, hk, hd, TYPES[dtype]
        self.total = front + sum(lens) + tail
        start = [front]
        for n in lens:
            start.append(start[-1] + n)
        self.start = start
        self.offsets = torch.tensor(start, dtype=torch.int32, device="cuda")
        self.fused = (amp * torch.randn((self.total, (hq + 2 * hk) * hd + pad), device="cuda", generator=gen)).to(self.dtype)
        width = (hq + 2 * hk) * hd
        heads = self.fused[:, :width].view(self.total, hq + 2 * hk, hd) if pad == 0 else self.fused[:, :width].unflatten(1, (hq + 2 * hk, hd))
        self.q, self.k, self.v = heads[:, :hq], heads[:, hq:hq + hk], heads[:, hq + hk:]
        self.do = (0.1 * torch.randn((self.total, hq, hd), device="cuda", generator=gen)).to(self.dtype)
        self.scale = hd ** -0.5

    def outputs(self, fill=7.0):
        o = torch.full((self.total, self.hq, self.hd), fill, device="cuda", dtype=self.dtype)
        lse = torch.full((self.hq, self.total), fill, device="cuda")
        return o, lse

    def gradients(self, fill=7.0):
        width = (self.hq + 2 * self.hk) * self.hd
        g = torch.full((self.total, self.fused.shape[1]), fill, device="cuda", dtype=self.dtype)[:, :width].unflatten(
            1, (self.hq + 2 * self.hk, self.hd))
        return g[:, :self.hq], g[:, self.hq:self.hq + self.hk], g[:, self.hq + self.hk:]

    def outside(self):
        keep = torch.ones(self.total, dtype=torch.bool, device="cuda")
        keep[self.start[0]:self.start[-1]] = False
        return keep

    def each(self):
        """(rows, query head, key head) of every sequence that has rows."""
        for i, n in enumerate(self.lens):
            if n:
                for h in range(self.hq):
                    yield slice(self.start[i], self.start[i + 1]), h, h * self.hk // self.hq


def half_step(x, dtype):
    return x.abs() * (W if dtype == torch.bfloat16 else U)


def weights(b, at, h, g):
    """Scores, weights, their relative error bound, log of the sums."""
    q, k = b.q[at, h].double(), b.k[at, g].double()
    n = q.shape[0]
    looks = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    s = torch.where(looks, b.scale * (q @ k.T), torch.full((n, n), -math.inf, dtype=torch.float64, device="cuda"))
    lse = torch.logsumexp(s, 1, keepdim=True)
    size = abs(b.scale) * (q.abs() @ k.abs().T)
    e = (b.hd + 2) * U * size.amax(1, keepdim=True) * 2 + (8 + 2 * s.masked_fill(~looks, 0).abs().amax(1, keepdim=True)) * U
    return torch.exp(s - lse), e, lse


def check_forward(b, o, lse):
    rounded = W if b.dtype == torch.bfloat16 else 0.0
    for at, h, g in b.each():
        p, e, want_lse = weights(b, at, h, g)
        v = b.v[at, g].double()
        n = p.shape[0]
        want, size = p @ v, p @ v.abs()
        tol = size * (2 * e + rounded + n * U) + half_step(want, b.dtype) + 1e-30
        worst = ((o[at, h].double() - want).abs() / tol).max().item()
        assert worst <= 1.0, (n, h, worst)
        if lse is not None:
            tol = 2 * e + n * U + 2 * U * want_lse.abs()
            worst = ((lse[h, at].double()[:, None] - want_lse).abs() / tol).max().item()
            assert worst <= 1.0, (n, h, worst)


def check_backward(b, o, lse, dq, dk, dv):
    rounded = W if b.dtype == torch.bfloat16 else 0.0
    want = {}
    for at, h, g in b.each():
        q, k, v, do, oo = (t.double() for t in (b.q[at, h], b.k[at, g], b.v[at, g], b.do[at, h], o[at, h]))
        n = q.shape[0]
        _, e, _ = weights(b, at, h, g)
        l = lse[h, at].double()[:, None]
        looks = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
        p = torch.where(looks, torch.exp(b.scale * (q @ k.T) - l), torch.zeros((n, n), dtype=torch.float64, device="cuda"))
        e = e + 2 * U * l.abs()
        dp, delta = do @ v.T, (do * oo).sum(1, keepdim=True)
        ds = p * (dp - delta)
        d_ds = p * ((dp - delta).abs() * e + (b.hd + 2) * U * (do.abs() @ v.abs().T + (do * oo).abs().sum(1, keepdim=True)))
        d_ds = d_ds + rounded * (ds.abs() + d_ds)
        group = (b.hq // b.hk) * n
        x = want.setdefault((at.start, at.stop, g), [torch.zeros_like(k), torch.zeros_like(k), torch.zeros_like(k), torch.zeros_like(k)])
        x[0] += b.scale * (ds.T @ q)
        x[1] += b.scale * ((d_ds + group * U * ds.abs()).T @ q.abs())
        x[2] += p.T @ do
        x[3] += (p * (e + rounded + group * U)).T @ do.abs()
        ref = b.scale * (ds @ k)
        tol = abs(b.scale) * ((d_ds + n * U * ds.abs()) @ k.abs()) + half_step(ref, b.dtype) + 1e-30
        worst = ((dq[at, h].double() - ref).abs() / tol).max().item()
        assert worst <= 1.0, ("dq", n, h, worst)
    for (first, end, g), (rk, tk, rv, tv) in want.items():
        for name, got, ref, tol in (("dk", dk, rk, tk), ("dv", dv, rv, tv)):
            worst = ((got[first:end, g].double() - ref).abs() / (tol + half_step(ref, b.dtype) + 1e-30)).max().item()
            assert worst <= 1.0, (name, end - first, g, worst)


def run_forward(ctx, b, fill=7.0, plan=None):
    o, lse = b.outputs(fill)
    plan = plan or ctx.attention_plan(b.offsets, b.total)
    assert ctx.abs_attention(b.q, b.k, b.v, plan, o, lse, scale=b.scale) is o
    return plan, o, lse


def run_backward(ctx, b, plan, o, lse, fill=7.0):
    dq, dk, dv = b.gradients(fill)
    scratch = ctx.attention_scratch(b.total, b.hq, b.hk, b.hd, len(b.lens))
    scratch.fill_(0xff)
    ctx.abs_attention_backward(b.do, b.q, b.k, b.v, o, lse, plan, dq, dk, dv, scratch, scale=b.scale)
    return dq, dk, dv


EDGES = [63, 64, 65, 0, 127, 128, 129, 1, 255, 256, 257, 2]
CASES = [
    ([1], 1, 1, 64, "bf16", {}),
    ([1], 2, 1, 128, "f32", {}),
    ([5], 3, 3, 8, "bf16", {}),
    (EDGES, 4, 2, 64, "bf16", dict(tail=3)),
    (EDGES, 4, 4, 128, "bf16", dict(front=5, tail=200)),
    (EDGES, 2, 1, 64, "f32", dict(front=1)),
    ([300, 77, 0, 0, 513], 6, 1, 128, "bf16", {}),
    ([300, 77, 0, 0, 513], 6, 2, 128, "f32", {}),
    ([200, 385], 4, 2, 80, "bf16", dict(tail=1)),
    ([200, 385], 4, 2, 96, "f32", dict(tail=1)),
    ([130, 40], 2, 2, 40, "bf16", {}),
    ([130, 40], 2, 2, 33, "bf16", {}),                       # rows that are not 16-byte aligned
    ([130, 40], 3, 1, 64, "bf16", dict(pad=1)),
    ([130, 40], 3, 1, 7, "f32", dict(pad=3)),
    ([700], 2, 2, 64, "bf16", dict(amp=3.0)),                # weights that one key takes most of
    ([700], 2, 2, 128, "bf16", dict(amp=2.5)),
    ([1500, 3], 2, 1, 64, "bf16", {}),
    ([1500, 3], 8, 1, 128, "bf16", {}),
    ([2] * 50 + [129] * 3, 2, 2, 64, "bf16", {}),
]


@pytest.mark.parametrize("lens,hq,hk,hd,dtype,kw", CASES)
def test_forward_and_backward(ctx, lens, hq, hk, hd, dtype, kw):
    b = Batch(lens, hq, hk, hd, dtype, seed=hd + sum(lens), **kw)
    plan, o, lse = run_forward(ctx, b)
    check_forward(b, o, lse)
    out = b.outside()
    assert (o[out] == 7.0).all() and (lse[:, out] == 7.0).all()
    dq, dk, dv = run_backward(ctx, b, plan, o, lse)
    check_backward(b, o, lse, dq, dk, dv)
    assert all((x[out] == 7.0).all() for x in (dq, dk, dv))


@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "bf16"), (64, "f32")])
def test_nothing_outside_a_sequence_reaches_it(ctx, hd, dtype):
    """NaN in the rows around the sequences, and in all of another sequence."""
    b = Batch([70, 130, 200], 4, 2, hd, dtype, seed=3, front=9, tail=61)
    plan, o, lse = run_forward(ctx, b)
    grads = run_backward(ctx, b, plan, o, lse)
    bad = b.outside()
    bad[b.start[1]:b.start[2]] = True
    for t in (b.fused, b.do):
        t[bad] = math.nan
    o2, lse2 = b.outputs()
    o2[bad], lse2[:, bad] = math.nan, math.nan
    ctx.abs_attention(b.q, b.k, b.v, plan, o2, lse2, scale=b.scale)
    for t in (o2,):
        assert torch.equal(t[~bad], o[~bad])
    assert torch.equal(lse2[:, ~bad], lse[:, ~bad])
    o2[b.outside()] = math.nan
    again = run_backward(ctx, b, plan, o2, lse2)
    for x, y in zip(grads, again):
        assert torch.equal(x[~bad], y[~bad])


@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "bf16"), (48, "f32")])
def test_results_repeat_bit_for_bit(ctx, hd, dtype):
    b = Batch([1100, 1, 640], 6, 2, hd, dtype, seed=4)
    plan, o, lse = run_forward(ctx, b)
    grads = run_backward(ctx, b, plan, o, lse)
    for _ in range(3):
        plan, o2, lse2 = run_forward(ctx, b)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        assert all(torch.equal(x, y) for x, y in zip(grads, run_backward(ctx, b, plan, o2, lse2)))


@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "bf16"), (64, "f32")])
def test_large_scores_of_equal_keys(ctx, hd, dtype):
    """All keys equal: every weight is 1 / (t + 1) whatever the scores' size, and the outputs are running means of V."""
    b = Batch([333], 2, 1, hd, dtype, seed=5)
    b.k[:] = 8.0 * torch.sign(b.k[:1])
    b.q[:] = 8.0 * torch.sign(b.q)
    _, o, lse = run_forward(ctx, b)
    v = b.v[:, 0].double()
    n = torch.arange(1, 334, device="cuda", dtype=torch.float64)[:, None]
    mean, size = v.cumsum(0) / n, v.abs().cumsum(0) / n
    tol = size * ((W if dtype == "bf16" else 0.0) + 400 * U) + half_step(mean, b.dtype)
    for h in range(2):
        assert ((o[:, h].double() - mean).abs() <= tol).all()
        s = b.scale * (b.q[:, h].double() @ b.k[:, 0].double().T)[:, :1]        # exact: sums of +-64
        assert ((lse[h].double()[:, None] - s - n.log()).abs() <= 400 * U + 6 * U * (s.abs() + n.log())).all()


@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (64, "f32")])
def test_scores_of_minus_infinity(ctx, hd, dtype):
    """Keys whose scores are all -infinity weigh nothing; a row with no other key has no answer (NaN)."""
    b = Batch([200], 1, 1, hd, dtype, seed=6)
    b.q[:, :, 0] = 1.0
    b.k[:150, :, 0] = -math.inf
    _, o, lse = run_forward(ctx, b)
    s = b.scale * (b.q[150:, 0].double() @ b.k[150:, 0].double().T)
    n = s.shape[0]
    s = s.masked_fill(torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1), -math.inf)
    want = torch.softmax(s, 1) @ b.v[150:, 0].double()
    assert torch.isnan(o[:150].float()).all()
    size = torch.softmax(s, 1) @ b.v[150:, 0].double().abs()
    assert ((o[150:, 0].double() - want).abs() <= size * (2 * W + 300 * U) + half_step(want, b.dtype)).all()
    assert (lse[0, :150] == -math.inf).all() and torch.isfinite(lse[0, 150:]).all()


def test_gradients_against_differences(ctx):
    """<dO, O> along random directions of the inputs, fp32: central differences of step h are off by truncation, of the order
    of h^2 of the values, and by rounding, u / h of the sum's size."""
    b = Batch([90, 41], 4, 2, 32, "f32", seed=7)
    plan, o, lse = run_forward(ctx, b)
    grads = run_backward(ctx, b, plan, o, lse)
    gen = torch.Generator(device="cuda").manual_seed(8)
    h = 2.0 ** -7
    for t, g in zip((b.q, b.k, b.v), grads):
        d = torch.randn(t.shape, device="cuda", generator=gen)
        keep = t.clone()
        values = []
        for sign in (1, -1):
            t.copy_(keep + sign * h * d)
            values.append((run_forward(ctx, b, plan=plan)[1].double() * b.do.double()).sum().item())
        t.copy_(keep)
        got, want = (g.double() * d.double()).sum().item(), (values[0] - values[1]) / (2 * h)
        scale = (b.do.double().norm() * o.double().norm()).item()
        # each of the 131 x 4 rows moves by about |d| ~ sqrt(hd) / sqrt(hd) in its scores: third derivatives of order one
        assert abs(got - want) <= scale * (4 * h * h + 64 * U / h), (got, want, scale)


def test_replicas_are_packed_sequences(ctx):
    """M replicas' [M, S, T, heads, hd] tensors flattened over their tokens: a sequence's result does not depend on what it is packed with."""
    b = Batch([96] * 6, 4, 4, 64, "bf16", seed=9)
    _, o, lse = run_forward(ctx, b)
    for i in range(6):
        at = slice(96 * i, 96 * (i + 1))
        one = ctx.attention_plan(torch.tensor([0, 96], dtype=torch.int32, device="cuda"), 96)
        oo, ll = torch.empty_like(o[at]), torch.empty((4, 96), device="cuda")
        ctx.abs_attention(b.q[at], b.k[at], b.v[at], one, oo, ll)
        assert torch.equal(oo, o[at]) and torch.equal(ll, lse[:, at])


@pytest.mark.parametrize("lens,hq,hk,hd", [([512] * 40, 8, 8, 64), ([130, 700, 40] * 12, 8, 4, 128), ([100] * 300, 6, 6, 64)])
def test_many_tiles_and_calls_behind_one_another(ctx, lens, hq, hk, hd):
    """More tiles than a GPU holds at a time, and calls that nothing waits between: all the same, and right."""
    b = Batch(lens, hq, hk, hd, "bf16", seed=14)
    plan, o, lse = run_forward(ctx, b)
    first = run_backward(ctx, b, plan, o, lse)
    scratch = ctx.attention_scratch(b.total, hq, hk, hd, len(lens))
    runs = [(b.outputs(), b.gradients(3.0)) for _ in range(12)]
    for (o2, lse2), g in runs:
        ctx.abs_attention(b.q, b.k, b.v, plan, o2, lse2, scale=b.scale)
        ctx.abs_attention_backward(b.do, b.q, b.k, b.v, o2, lse2, plan, *g, scratch, scale=b.scale)
    for (o2, lse2), g in runs:
        assert torch.equal(o2, o) and torch.equal(lse2, lse) and all(torch.equal(x, y) for x, y in zip(g, first))
    check_forward(b, o, lse)
    check_backward(b, o, lse, *first)


def test_capture_replay_and_new_offsets(ctx):
    """A captured forward and backward pass follows the inputs and the plan that are there when it is replayed."""
    b = Batch([300, 212], 4, 2, 64, "bf16", seed=10)
    stream = torch.cuda.Stream()
    plan = ctx.attention_plan(b.offsets, b.total)
    scratch = ctx.attention_scratch(b.total, 4, 2, 64, 2)
    o, lse = b.outputs()
    grads = b.gradients()

    def both():
        ctx.abs_attention(b.q, b.k, b.v, plan, o, lse, scale=b.scale)
        ctx.abs_attention_backward(b.do, b.q, b.k, b.v, o, lse, plan, *grads, scratch, scale=b.scale)

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        both()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            both()
    for lens in ([300, 212], [10, 502], [0, 512], [511, 1]):
        b.lens, b.start = lens, [0, lens[0], 512]
        ctx.attention_plan(torch.tensor(b.start, dtype=torch.int32, device="cuda"), b.total, plan=plan)
        b.fused.copy_(torch.randn_like(b.fused))
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        check_forward(b, o, lse)
        check_backward(b, o, lse, *grads)


def test_on_another_stream(ctx):
    b = Batch([600, 9], 2, 2, 64, "bf16", seed=11)
    plan, o, lse = run_forward(ctx, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2, lse2 = b.outputs()
    ctx.abs_attention(b.q, b.k, b.v, plan, o2, lse2, scale=b.scale, stream=side)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("table,lens,bad", [([5, 3, 40], [0, 35], 1), ([-4, 20, 90], [20, 20], 1), ([0, 7, 40], [7, 33], 0)])
def test_bad_offsets_are_put_right(ctx, table, lens, bad):
    b = Batch([40], 2, 1, 64, "bf16", seed=12)
    b.lens = lens
    b.start = [max(table[0], 0)]
    for n in lens:
        b.start.append(b.start[-1] + n)
    b.offsets = torch.tensor(table, dtype=torch.int32, device="cuda")
    plan, o, lse = run_forward(ctx, b)
    assert plan.words[2].item() == bad
    check_forward(b, o, lse)
    check_backward(b, o, lse, *run_backward(ctx, b, plan, o, lse))
    assert (o[b.outside()] == 7.0).all()


def test_plan_covers_every_tile_once(ctx):
    """Every tile of every sequence once; forward the most work first, backward the least."""
    gen = torch.Generator().manual_seed(13)
    lens = torch.randint(0, 1500, (700,), generator=gen)
    lens[::7] = 0
    start = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
    total = int(start[-1]) + 50
    plan = ctx.attention_plan(start.to(torch.int32).cuda(), total)
    words = plan.words.cpu()
    n = len(lens)
    fwd_cap, bwd_cap = total // 256 + n, total // 128 + n
    for kind, rows, at in ((0, 256, 16), (1, 128, 16 + 4 * fwd_cap)):
        count = int(words[kind])
        assert count <= (fwd_cap, bwd_cap)[kind]
        recs = [tuple(r.tolist()) for r in words[at:at + 4 * count].view(-1, 4)]
        slots = {(r[3] + r[2]) for r in recs}
        assert kind == 0 or (len(slots) == count and max(slots) < bwd_cap)
        recs = [r[:3] for r in recs]
        want = {(int(start[i]), int(start[i + 1]), t) for i in range(n) for t in range(-(-int(lens[i]) // rows))}
        assert len(recs) == len(want) and set(recs) == want
        work = [-t - 1 if kind == 0 else -(-(e - s) // rows) - t for s, e, t in recs]
        assert work == sorted(work)


def test_nothing_to_do(ctx):
    b = Batch([0, 0], 2, 2, 64, "bf16", tail=4)
    plan, o, lse = run_forward(ctx, b)
    grads = run_backward(ctx, b, plan, o, lse)
    assert (o == 7.0).all() and (lse == 7.0).all() and all((g == 7.0).all() for g in grads)
    empty = Batch([], 2, 2, 64, "bf16")
    plan, o, lse = run_forward(ctx, empty)
    run_backward(ctx, empty, plan, o, lse)


@pytest.mark.parametrize("hq,hk,parts", [(6, 2, 1), (6, 2, 3), (4, 1, 4)])
def test_groups_of_heads_whole_and_in_parts(ctx, hq, hk, parts):
    """Many tiles: a group's query heads are one tile's work; few: each part's dk and dv are summed at the end."""
    b = Batch([5, 131] * 300 if parts == 1 else [700, 129], hq, hk, 64, "bf16", seed=31)
    tiles = (b.total // 128 + len(b.lens)) * hk
    assert (tiles >= 8 * 148) == (parts == 1)
    plan, o, lse = run_forward(ctx, b)
    check_backward(b, o, lse, *run_backward(ctx, b, plan, o, lse))


@pytest.mark.parametrize("hd,pad", [(64, 8), (128, 8), (72, 0), (72, 8), (64, 16)])
def test_rows_that_are_no_whole_sectors(ctx, hd, pad):
    """Strides of 16 bytes that are not 32, and heads whose last sector is half: rows are stored 16 bytes at a time, nothing beside them."""
    b = Batch([3, 150, 300], 4, 2, hd, "bf16", seed=32, front=2, tail=3, pad=pad)
    plan = ctx.attention_plan(b.offsets, b.total)
    wide = torch.full((b.total, b.hq * hd + pad), 7.0, device="cuda", dtype=torch.bfloat16)
    o, lse = wide[:, :b.hq * hd].unflatten(1, (b.hq, hd)), torch.full((b.hq, b.total), 7.0, device="cuda")
    ctx.abs_attention(b.q, b.k, b.v, plan, o, lse, scale=b.scale)
    check_forward(b, o, lse)
    assert (wide[:, b.hq * hd:] == 7.0).all() and (o[b.outside()] == 7.0).all()
    width = (b.hq + 2 * b.hk) * hd
    grads = torch.full(b.fused.shape, 7.0, device="cuda", dtype=torch.bfloat16)
    heads = grads[:, :width].unflatten(1, (b.hq + 2 * b.hk, hd))
    dq, dk, dv = heads[:, :b.hq], heads[:, b.hq:b.hq + b.hk], heads[:, b.hq + b.hk:]
    scratch = ctx.attention_scratch(b.total, b.hq, b.hk, hd, len(b.lens))
    ctx.abs_attention_backward(b.do, b.q, b.k, b.v, o, lse, plan, dq, dk, dv, scratch, scale=b.scale)
    check_backward(b, o, lse, dq, dk, dv)
    assert (grads[:, width:] == 7.0).all() and (grads[b.outside()] == 7.0).all()


@pytest.mark.parametrize("hd,hq,hk", [(64, 4, 4), (128, 4, 4), (64, 6, 2)])
def test_a_wait_that_runs_out_leaves_nan_and_the_next_call_is_right(ctx, hd, hq, hk):
    b = Batch([300, 0, 1, 700], hq, hk, hd, "bf16", seed=33, front=1, tail=2)
    plan, o, lse = run_forward(ctx, b)
    grads = run_backward(ctx, b, plan, o, lse)
    ctx.set_tuning("stats_timeout_cycles", 200000)
    ctx.set_tuning("stats_fault_drop_loads", 1)
    try:
        _, lost, lost_lse = run_forward(ctx, b)
        lost_grads = run_backward(ctx, b, plan, o, lse)
        torch.cuda.synchronize()
    finally:
        ctx.set_tuning("stats_fault_drop_loads", 0)
        ctx.set_tuning("stats_timeout_cycles", 0)
    inside = ~b.outside()
    assert torch.isnan(lost[inside]).all() and torch.isnan(lost_lse[:, inside]).all()
    for g in lost_grads:
        assert torch.isnan(g[inside]).all() and (g[~inside] == 7.0).all()
    assert (lost[~inside] == 7.0).all()
    _, again, again_lse = run_forward(ctx, b)
    assert torch.equal(again, o) and torch.equal(again_lse, lse)
    for g, want in zip(run_backward(ctx, b, plan, o, lse), grads):
        assert torch.equal(g, want)


@pytest.mark.parametrize("scale", [0.0, -0.3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_of_zero_and_below(ctx, dtype, scale):
    b = Batch([1, 65, 200], 2, 1, 64, dtype, seed=34)
    b.scale = scale
    plan, o, lse = run_forward(ctx, b)
    check_forward(b, o, lse)
    check_backward(b, o, lse, *run_backward(ctx, b, plan, o, lse))


@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "bf16"), (64, "f32")])
def test_rows_far_apart(ctx, hd, dtype):
    """Elements behind the 2^31-st of a tensor: the same bits as from rows that lie together."""
    b = Batch([520, 30], 2, 1, hd, dtype, seed=35)
    plan, o, lse = run_forward(ctx, b)
    want = (o, *run_backward(ctx, b, plan, o, lse))
    heads, apart = b.hq + 2 * b.hk, 1 << 22
    far = torch.empty((b.total, apart), device="cuda", dtype=b.dtype)[:, -heads * hd:].unflatten(1, (heads, hd))
    assert b.total * apart > 2 ** 31
    far.copy_(b.fused.view(b.total, heads, hd))
    views = far.split((b.hq, b.hk, b.hk), dim=1)
    far_o = torch.empty((b.total, apart), device="cuda", dtype=b.dtype)[:, -b.hq * hd:].unflatten(1, (b.hq, hd))
    ctx.abs_attention(*views, plan, far_o, lse, scale=b.scale)
    grads = torch.empty((b.total, apart), device="cuda", dtype=b.dtype)[:, -heads * hd:].unflatten(1, (heads, hd)).split((b.hq, b.hk, b.hk), dim=1)
    scratch = ctx.attention_scratch(b.total, b.hq, b.hk, hd, 2)
    ctx.abs_attention_backward(b.do, *views, far_o, lse, plan, *grads, scratch, scale=b.scale)
    for got, ref in zip((far_o, *grads), want):
        assert torch.equal(got, ref)


def test_calls_on_two_streams_at_once(ctx):
    """Two batches' passes side by side, each with its own plan and scratch: the same bits as one after the other."""
    batches = [Batch([1000, 300, 77] * 8, 6, 2, 64, "bf16", seed=36), Batch([700, 2048], 4, 4, 128, "bf16", seed=37)]
    want, sides = [], [torch.cuda.Stream() for _ in batches]
    for b in batches:
        plan, o, lse = run_forward(ctx, b)
        want.append((o, *run_backward(ctx, b, plan, o, lse)))
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        outs = [(b.outputs(), b.gradients(), ctx.attention_scratch(b.total, b.hq, b.hk, b.hd, len(b.lens))) for b in batches]
        torch.cuda.synchronize()
        for b, side, ((o, lse), grads, scratch) in zip(batches, sides, outs):
            with torch.cuda.stream(side):
                plan = ctx.attention_plan(b.offsets, b.total)
                ctx.abs_attention(b.q, b.k, b.v, plan, o, lse, scale=b.scale)
                ctx.abs_attention_backward(b.do, b.q, b.k, b.v, o, lse, plan, *grads, scratch, scale=b.scale)
                got.append((plan, (o, *grads)))
        torch.cuda.synchronize()
        for (_, g), w in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(g, w))


@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "bf16"), (40, "f32")])
def test_heads_in_front_of_tokens_and_no_lse(ctx, hd, dtype):
    """Tensors [heads][total][hd], forward with and without lse: the same bits as from [total][heads][hd]."""
    b = Batch([140, 1, 300], 6, 3, hd, dtype, seed=38, front=1, tail=2)
    plan, o, lse = run_forward(ctx, b)
    want = (o, *run_backward(ctx, b, plan, o, lse))
    by_head = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    q, k, v, do = (by_head(t) for t in (b.q, b.k, b.v, b.do))
    got_o = by_head(torch.full_like(o, 7.0))
    ctx.abs_attention(q, k, v, plan, got_o, None, scale=b.scale)
    grads = tuple(by_head(torch.full_like(t, 7.0)) for t in (q, k, v))
    scratch = ctx.attention_scratch(b.total, b.hq, b.hk, hd, len(b.lens))
    ctx.abs_attention_backward(do, q, k, v, got_o, lse, plan, *grads, scratch, scale=b.scale)
    for got, ref in zip((got_o, *grads), want):
        assert torch.equal(got, ref)


@pytest.mark.parametrize("hq,hk,hd", [(64, 1, 64), (96, 96, 8), (30, 10, 128)])
def test_many_heads(ctx, hq, hk, hd):
    b = Batch([129, 70], hq, hk, hd, "bf16", seed=39)
    plan, o, lse = run_forward(ctx, b)
    check_forward(b, o, lse)
    check_backward(b, o, lse, *run_backward(ctx, b, plan, o, lse))


@pytest.mark.parametrize("steps", [1, 2, 3, 5, 10])
@pytest.mark.parametrize("lens,hd,hq,hk", [([300, 0, 1, 700, 129, 64, 1500, 17], 64, 6, 2), ([300, 0, 1, 700, 129, 64, 1500, 17], 128, 6, 2),
                                           ([5, 131, 400] * 200, 64, 2, 2), ([5, 131, 400] * 200, 128, 2, 2), ([2000, 1100], 64, 4, 1),
                                           ([2000, 1100], 128, 4, 1)])
def test_loads_that_stop_in_the_middle(ctx, lens, hd, hq, hk, steps):
    """Every other CTA's loads stop after some steps: waits run out in the middle of tiles, and in CTAs that wait for such a tile's part of dq
    while their own copies, whole and partial blocks', are under way.  What is not NaN has the undisturbed calls' bits, and the next
    calls are right.  (Groups of heads in parts and whole; one to sixteen tiles of keys a sequence.)"""
    b = Batch(lens, hq, hk, hd, "bf16", seed=40, front=1, tail=2)
    plan, o, lse = run_forward(ctx, b)
    grads = run_backward(ctx, b, plan, o, lse)
    ctx.set_tuning("stats_timeout_cycles", 200000)
    ctx.set_tuning("attention_fault_stop_after", steps)
    try:
        _, some_o, some_lse = run_forward(ctx, b)
        some_grads = run_backward(ctx, b, plan, o, lse)
        torch.cuda.synchronize()
    finally:
        ctx.set_tuning("attention_fault_stop_after", 0)
        ctx.set_tuning("stats_timeout_cycles", 0)
    inside = ~b.outside()
    lost = 0
    for got, want in ((some_o, o), (some_lse.t(), lse.t()), *zip(some_grads, grads)):
        nan = torch.isnan(got)
        assert torch.equal(got[~nan], want[~nan]) and (got[~inside] == 7.0).all()
        lost += nan.sum().item()
    assert lost > 0
    again_o, again_lse = run_forward(ctx, b)[1:]
    assert torch.equal(again_o, o) and torch.equal(again_lse, lse)
    for g, want in zip(run_backward(ctx, b, plan, o, lse), grads):
        assert torch.equal(g, want)


@pytest.mark.parametrize("hd,dtype,hq,hk", [(64, "bf16", 6, 2), (128, "bf16", 2, 2), (64, "f32", 4, 2), (24, "bf16", 3, 3)])
@pytest.mark.parametrize("change", ["sequences", "total", "zeros", "words"])
def test_a_plan_of_another_batch_gives_nan(ctx, hd, dtype, hq, hk, change):
    """Nothing of such a plan but its header is looked at."""
    b = Batch([300, 5, 200], hq, hk, hd, dtype, seed=41, front=1, tail=2, pad=1 if hd == 24 else 0)
    plan, o, lse = run_forward(ctx, b)
    grads = run_backward(ctx, b, plan, o, lse)
    n = len(b.lens)
    words = plan.words.clone()
    if change == "sequences":
        words = ctx.attention_plan(torch.tensor([1, 301, 306], dtype=torch.int32, device="cuda"), b.total).words
    elif change == "total":
        words = ctx.attention_plan(b.offsets, b.total + 1).words
    elif change == "zeros":
        words.zero_()
    elif change == "words":
        words = torch.randint(-2 ** 31, 2 ** 31 - 1, words.shape, device="cuda", dtype=torch.int32)
    other = pkg.AttentionPlan(words, n, b.total)
    wrong_o, wrong_lse = run_forward(ctx, b, plan=other)[1:]
    for t in (wrong_o, wrong_lse, *run_backward(ctx, b, other, o, lse)):
        assert torch.isnan(t).all()
    again_o, again_lse = run_forward(ctx, b, plan=plan)[1:]
    assert torch.equal(again_o, o) and torch.equal(again_lse, lse)
    for g, want in zip(run_backward(ctx, b, plan, o, lse), grads):
        assert torch.equal(g, want)


@pytest.mark.parametrize("scale", [2.5e38, -2.5e38, math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_that_overflow_are_refused(ctx, dtype, scale):
    """Scores are taken log2 e times in the exponent: a scale that is finite but overflows there would make every row NaN."""
    b = Batch([3], 2, 1, 64, dtype, seed=42)
    plan, o, lse = run_forward(ctx, b)
    b.scale = scale
    with pytest.raises(pkg.AbsError, match="scale"):
        run_forward(ctx, b, plan=plan)
    with pytest.raises(pkg.AbsError, match="scale"):
        run_backward(ctx, b, plan, o, lse)
