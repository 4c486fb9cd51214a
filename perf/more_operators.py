"""Cases for timing and checking attention, the root-mean-square norm and the token embedding.

Three operators, each with its backward pass: causal attention with grouped heads over packed sequences, the
root-mean-square norm with the residual's addition (and an 8-bit output), and the embedding lookup of M replicas.
`run` computes each in its plain form, elementary torch operations in fp32, or, where `own` is set, through the
package's Context.  Everything runs on cuda:0.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
RMS_EPS = 1e-6
E4M3_MAX = 448.0


# ---- cases ---------------------------------------------------------------------------------------
# lens: the packed sequences' lengths, "4*100,7" is four of 100 and one of 7; tail: rows behind the last sequence
def listed():
    return [
        # 8 workers, micro-batches of 16 sequences of 1024 tokens, one layer of the 12-layer, 768-wide language model
        dict(name="attn_fwd_lm", op="attn_fwd", lens="128*1024", tail=0, hq=12, hk=12, hd=64, dtype="bf16"),
        # two long documents of unequal length, grouped heads of 128
        dict(name="attn_fwd_long", op="attn_fwd", lens="8191,4097", tail=5, hq=8, hk=2, hd=128, dtype="bf16"),
        # backward of attn_fwd_lm
        dict(name="attn_bwd_lm", op="attn_bwd", lens="128*1024", tail=0, hq=12, hk=12, hd=64, dtype="bf16"),
        # a fine-tuning batch of short texts of all lengths, one of them a single token, grouped heads of 128
        dict(name="attn_bwd_ragged", op="attn_bwd", lens="700,1,129,0,333,64,1500,17,256", tail=72, hq=16, hk=2, hd=128, dtype="bf16"),
        # the norm in front of a layer of that model: the branch is added to the residual stream on the way
        dict(name="rms_fwd_lm", op="rms_fwd", M=8, rows=16384, d=768, pad=0, dtype="bf16", residual=True, quant=False),
        # input of an 8-bit product: rows in e4m3 with a scale each
        dict(name="rms_fwd_8bit", op="rms_fwd", M=1, rows=4099, d=4096, pad=0, dtype="bf16", residual=False, quant=True),
        # backward of rms_fwd_lm with one gradient row per sequence for the batch-size test
        dict(name="rms_bwd_lm", op="rms_bwd", M=8, S=16, T=1024, d=768, pad=0, dtype="bf16", residual=True, per_sample=True),
        # per-sample gradients of a classifier's norm (one row a sample), odd width: latency is all there is
        dict(name="rms_bwd_few_rows", op="rms_bwd", M=2, S=8, T=1, d=257, pad=0, dtype="f32", residual=False, per_sample=True),
        # the token embedding of that model: tables of 8 replicas, falling token frequencies
        dict(name="emb_fwd_lm", op="emb_fwd", M=8, rows=16384, vocab=50000, d=768, dtype="bf16"),
        # a handful of tokens of a small vocabulary, an odd width
        dict(name="emb_fwd_few_rows", op="emb_fwd", M=1, rows=7, vocab=1001, d=129, dtype="f32"),
        # its gradient: every row of the tables is written, those of absent tokens with zeros
        dict(name="emb_bwd_lm", op="emb_bwd", M=8, rows=16384, vocab=50000, d=768, dtype="bf16", add=False),
        # a short micro-batch added to a gradient that is there already (tied tables, accumulated batches)
        dict(name="emb_bwd_add", op="emb_bwd", M=2, rows=300, vocab=777, d=100, dtype="f32", add=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn_fwd", "attn_bwd", "rms_fwd", "rms_bwd", "emb_fwd", "emb_bwd"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op in ("attn_fwd", "attn_bwd"):
        hd = rng.choice([32, 64, 64, 80, 96, 128, 128])
        hk = rng.randint(1, 8)
        hq = hk * rng.choice([1, 1, 2, 4])
        longest = _log(rng, 1, 6000 if dtype == "bf16" else 1500)
        # the plain form holds [sequences, heads, longest, longest] values several times over
        most = max(1, min(64, int(4.0e8 / (hq * longest * longest))))
        lens = [longest] + [rng.randint(0, longest) for _ in range(rng.randint(0, most - 1))]
        rng.shuffle(lens)
        return dict(op=op, lens=",".join(map(str, lens)), tail=rng.choice([0, 0, 3, 100]), hq=hq, hk=hk, hd=hd, dtype=dtype)
    if op in ("rms_fwd", "rms_bwd"):
        d = _log(rng, 32, 8192)
        if rng.random() < 0.6:
            d = max(32, d // 8 * 8)
        M = rng.randint(1, 8)
        rows = _log(rng, 1, min(40000, max(2, 60_000_000 // (M * d))))
        case = dict(op=op, M=M, d=d, pad=rng.choice([0, 0, 8, 3]), dtype=dtype, residual=rng.random() < 0.6)
        if op == "rms_fwd":
            return dict(case, rows=rows, quant=rng.random() < 0.4)
        S = _log(rng, 1, min(64, rows))
        return dict(case, S=S, T=max(1, rows // S), per_sample=rng.random() < 0.5)
    d = _log(rng, 16, 4096)
    if rng.random() < 0.6:
        d = max(16, d // 8 * 8)
    M = rng.randint(1, 8)
    vocab = _log(rng, 16, min(130_000, 250_000_000 // (M * d)))
    rows = _log(rng, 1, min(60_000, max(2, 90_000_000 // (M * d))))
    case = dict(op=op, M=M, rows=rows, vocab=vocab, d=d, dtype=dtype)
    return case if op == "emb_fwd" else dict(case, add=rng.random() < 0.3)


def _lens(case):
    out = []
    for part in case["lens"].split(","):
        times, _, length = part.rpartition("*")
        out += [int(length)] * int(times or 1)
    return out


# ---- inputs --------------------------------------------------------------------------------------
def _rows(gen, M, rows, d, pad, dtype, scale, offset):
    """[M, rows, d] activations inside rows of d + pad: every row has a scale and an offset of its own."""
    full = torch.randn((M, rows, d + pad), device="cuda", generator=gen)
    s = torch.rand((M, rows, 1), device="cuda", generator=gen) + 0.5
    o = torch.randn((M, rows, 1), device="cuda", generator=gen)
    return (full * (scale * s) + offset * o).to(dtype)[:, :, :d]


def _sequences(st, gen):
    """Offsets of the packed sequences, and their rows' places in [sequences, longest]."""
    lens = _lens(st)
    st["n"], st["longest"] = len(lens), max(max(lens), 1)
    length = torch.tensor(lens)
    start = torch.cat([torch.zeros(1, dtype=torch.int64), length.cumsum(0)])
    st["total"] = int(start[-1]) + st["tail"]
    at = torch.arange(st["longest"])
    valid = at[None, :] < length[:, None]
    packed = (start[:-1, None] + at[None, :])[valid]
    st["offsets"] = start.to(torch.int32).cuda()
    st["packed"], st["padded"] = packed.cuda(), valid.view(-1).nonzero().view(-1).cuda()
    st["valid"] = valid.cuda()


def _prepare_attention(st, gen):
    _sequences(st, gen)
    total, hq, hk, hd, dt = st["total"], st["hq"], st["hk"], st["hd"], TYPES[st["dtype"]]
    # what one product of a layer gives: queries, keys and values side by side, every head with a scale of its own
    heads = hq + 2 * hk
    fused = torch.randn((total, heads, hd), device="cuda", generator=gen)
    fused *= 0.5 + 1.5 * torch.rand((1, heads, 1), device="cuda", generator=gen)
    st["QKV"] = fused.to(dt)
    st["O"] = torch.zeros((total, hq, hd), device="cuda", dtype=dt)
    st["lse"] = torch.zeros((hq, total), device="cuda")
    st["scale"] = hd ** -0.5
    if st["op"] == "attn_bwd":
        st["dO"] = (1e-2 * torch.randn((total, hq, hd), device="cuda", generator=gen)).to(dt)
        out = _plain_attn_fwd(st)
        st["O"], st["lse"] = out["O"], out["lse"]
        st["dQKV"] = torch.zeros((total, heads, hd), device="cuda", dtype=dt)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    st = dict(case)
    if op in ("attn_fwd", "attn_bwd"):
        _prepare_attention(st, gen)
        return st
    M, d, dt = case["M"], case["d"], TYPES[case["dtype"]]
    if op in ("rms_fwd", "rms_bwd"):
        rows = case["rows"] if op == "rms_fwd" else case["S"] * case["T"]
        # the replicas' parameter vectors: the norm's weight lies inside a longer flat vector
        st["weight"] = (1.0 + 0.1 * torch.randn((M, d + 64), device="cuda", generator=gen))[:, :d]
        shape = (M, rows, d)
        if op == "rms_fwd":
            st["X"] = _rows(gen, M, rows, d, case["pad"], dt, 0.5, 0.1)
            st["R"] = _rows(gen, M, rows, d, case["pad"], dt, 1.0, 0.5) if case["residual"] else None
            st["H"] = torch.empty(shape, device="cuda", dtype=dt) if case["residual"] else None
            st["rstd"] = torch.empty((M, rows), device="cuda")
            if case["quant"]:
                st["Y"], st["Q"] = None, torch.empty(shape, device="cuda", dtype=torch.float8_e4m3fn)
                st["scales"] = torch.empty((M, rows), device="cuda")
            else:
                st["Y"] = torch.empty(shape, device="cuda", dtype=dt)
            return st
        st["H"] = _rows(gen, M, rows, d, case["pad"], dt, 1.0, 0.5)
        st["rstd"] = (st["H"].double().square().mean(2) + RMS_EPS).rsqrt().float()
        st["dY"] = _rows(gen, M, rows, d, case["pad"], dt, 1e-3, 1e-4)
        st["dH"] = _rows(gen, M, rows, d, case["pad"], dt, 1e-3, 1e-4) if case["residual"] else None
        st["dX"] = torch.empty(shape, device="cuda", dtype=dt)
        st["dW"] = torch.empty((M, d), device="cuda")
        st["G"] = torch.empty((M, case["S"], d), device="cuda") if case["per_sample"] else None
        return st
    rows, vocab = case["rows"], case["vocab"]
    # falling frequencies: the k-th token about 1 / k of the first
    u = torch.rand((M, rows), device="cuda", generator=gen)
    st["tokens"] = (torch.exp(u * math.log(vocab + 1.0)) - 1.0).floor().clamp_(0, vocab - 1).to(torch.int32)
    st["scale"] = math.sqrt(d)
    # the table lies inside the replicas' flat parameter vectors, the gradient inside theirs
    flat = torch.empty((M, vocab * d + 64), device="cuda")
    table = flat[:, :vocab * d].view(M, vocab, d)
    if op == "emb_fwd":
        st["E"] = table
        for m in range(M):
            table[m].normal_(0.0, 0.02, generator=gen)
        st["Y"] = torch.empty((M, rows, d), device="cuda", dtype=dt)
        return st
    st["dY"] = (1e-3 * torch.randn((M, rows, d), device="cuda", generator=gen)).to(dt)
    st["dE"] = table
    if case["add"]:
        flat.normal_(0.0, 1e-3, generator=gen)
    return st


# ---- the plain forms -----------------------------------------------------------------------------
def _split(st, fused):
    hq, hk = st["hq"], st["hk"]
    return fused[:, :hq], fused[:, hq:hq + hk], fused[:, hq + hk:]


def _pad(st, x, kind=torch.float32):
    """[total, heads, hd] -> [sequences, heads, longest, hd], zeros behind a sequence's end."""
    out = torch.zeros((st["n"] * st["longest"], x.shape[1], x.shape[2]), device="cuda", dtype=kind)
    out[st["padded"]] = x[st["packed"]].to(kind)
    return out.view(st["n"], st["longest"], x.shape[1], x.shape[2]).transpose(1, 2)


def _unpad(st, x, into):
    """[sequences, heads, longest, hd] -> rows of `into` [total, heads, hd]; the rows behind the last sequence stay."""
    flat = x.transpose(1, 2).reshape(st["n"] * st["longest"], x.shape[1], x.shape[3])
    into[st["packed"]] = flat[st["padded"]].to(into.dtype)
    return into


def _scores(st, q, k):
    """[n, hk, group, longest, longest] scaled products with -inf where a row may not look."""
    n, hk, L, hd = k.shape
    s = q.reshape(n, hk, -1, L, hd) @ k.unsqueeze(2).transpose(3, 4)
    s *= st["scale"]
    later = torch.ones((L, L), device="cuda", dtype=torch.bool).triu_(1)
    return s.masked_fill_(later, -math.inf)


def _plain_attn_fwd(st):
    q, k, v = (_pad(st, x) for x in _split(st, st["QKV"]))
    n, hq, L, hd = q.shape
    s = _scores(st, q, k)
    top = s.amax(4, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(4, keepdim=True)
    o = (p @ v.unsqueeze(2)) / total
    lse = (top + total.log()).reshape(n, hq, L, 1)
    _unpad(st, o.reshape(n, hq, L, hd), st["O"])
    _unpad(st, lse, st["lse"].t().unsqueeze(2))
    return {"O": st["O"], "lse": st["lse"]}


def _plain_attn_bwd(st):
    q, k, v = (_pad(st, x) for x in _split(st, st["QKV"]))
    n, hq, L, hd = q.shape
    hk = k.shape[1]
    do, o = _pad(st, st["dO"]), _pad(st, st["O"])
    lse = _pad(st, st["lse"].t().unsqueeze(2))
    group = (n, hk, hq // hk, L, -1)
    do, q, delta = do.reshape(group), q.reshape(group), (do * o).sum(3).reshape(group)
    p = _scores(st, q, k).sub_(lse.reshape(group)).exp_()
    p.masked_fill_(~st["valid"].view(n, 1, 1, L, 1), 0.0)
    dv = (p.transpose(3, 4) @ do).sum(2)
    ds = (do @ v.unsqueeze(2).transpose(3, 4)).sub_(delta).mul_(p).mul_(st["scale"])
    dq = (ds @ k.unsqueeze(2)).reshape(n, hq, L, hd)
    dk = (ds.transpose(3, 4) @ q).sum(2)
    for x, into in zip((dq, dk, dv), _split(st, st["dQKV"])):
        _unpad(st, x, into)
    return {"dQKV": st["dQKV"]}


def _plain_rms_fwd(st):
    dt = st["X"].dtype
    out = {}
    h = st["X"].float()
    if st["R"] is not None:
        out["H"] = (h + st["R"].float()).to(dt)          # what the stream holds is what is normalised
        h = out["H"].float()
    rstd = torch.rsqrt((h * h).mean(2, keepdim=True) + RMS_EPS)
    y = h * rstd * st["weight"].unsqueeze(1)
    out["rstd"] = rstd.squeeze(2)
    if st["quant"]:
        top = y.abs().amax(2, keepdim=True)
        scale = torch.where(top == 0, torch.ones_like(top), top / E4M3_MAX)
        out["Q"] = (y / scale).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        out["scales"] = scale.squeeze(2)
    else:
        out["Y"] = y.to(dt)
    return out


def _plain_rms_bwd(st):
    h, dy = st["H"].float(), st["dY"].float()
    M, rows, d = h.shape
    rstd = st["rstd"].unsqueeze(2)
    xh = h * rstd
    a = dy * st["weight"].unsqueeze(1)
    dx = rstd * (a - xh * (a * xh).mean(2, keepdim=True))
    if st["dH"] is not None:
        dx = dx + st["dH"].float()
    out = {"dX": dx.to(st["H"].dtype)}
    gw = (dy * xh).view(M, st["S"], st["T"], d).sum(2)
    if st["per_sample"]:
        out["G"] = gw
    out["dW"] = gw.sum(1)
    return out


def _plain_emb_fwd(st):
    M, vocab, d = st["E"].shape
    at = st["tokens"].long()
    rows = st["E"][torch.arange(M, device="cuda")[:, None], at]
    return {"Y": (rows * st["scale"]).to(st["Y"].dtype)}


def _plain_emb_bwd(st):
    M, rows = st["tokens"].shape
    dE = st["dE"]
    if not st["add"]:
        dE.zero_()
    at = st["tokens"].long()
    dE.index_put_((torch.arange(M, device="cuda")[:, None].expand(M, rows), at), st["dY"].float() * st["scale"], accumulate=True)
    return {"dE": dE}


# ---- the package's operators ---------------------------------------------------------------------
_kept = {}


def _context():
    """The context that a program keeps from call to call."""
    if "ctx" not in _kept:
        import paper_2406_13936_b200 as pkg
        _kept["ctx"] = pkg.Context(0)
    return _kept["ctx"]


def _own(st):
    ctx = _context()
    op = st["op"]
    if op in ("attn_fwd", "attn_bwd"):
        if "plan" not in st:      # one a batch, which every layer's forward and backward pass takes
            st["plan"] = ctx.attention_plan(st["offsets"], st["total"])
            if op == "attn_bwd":
                st["scratch"] = ctx.attention_scratch(st["total"], st["hq"], st["hk"], st["hd"], st["n"])
        q, k, v = _split(st, st["QKV"])
        if op == "attn_fwd":
            ctx.abs_attention(q, k, v, st["plan"], st["O"], st["lse"], scale=st["scale"])
            return {"O": st["O"], "lse": st["lse"]}
        dq, dk, dv = _split(st, st["dQKV"])
        ctx.abs_attention_backward(st["dO"], q, k, v, st["O"], st["lse"], st["plan"], dq, dk, dv, st["scratch"],
                                   scale=st["scale"])
        return {"dQKV": st["dQKV"]}
    if op == "rms_fwd":
        if st["quant"]:
            ctx.abs_rms_norm(st["X"], st["weight"], RMS_EPS, None, residual=st["R"], summed=st["H"], rstd=st["rstd"],
                             Q=st["Q"], scales=st["scales"])
            out = {"rstd": st["rstd"], "Q": st["Q"], "scales": st["scales"]}
        else:
            ctx.abs_rms_norm(st["X"], st["weight"], RMS_EPS, st["Y"], residual=st["R"], summed=st["H"], rstd=st["rstd"])
            out = {"rstd": st["rstd"], "Y": st["Y"]}
        if st["R"] is not None:
            out["H"] = st["H"]
        return out
    if op == "rms_bwd":
        ctx.abs_rms_norm_backward(st["dY"], st["H"], st["rstd"], st["weight"], st["dX"], dH=st["dH"], dW=st["dW"],
                                  samples=st["S"], Gw=st["G"])
        out = {"dX": st["dX"], "dW": st["dW"]}
        if st["per_sample"]:
            out["G"] = st["G"]
        return out
    if op == "emb_fwd":
        ctx.abs_embedding(st["E"], st["tokens"], st["Y"], scale=st["scale"])
        return {"Y": st["Y"]}
    if "scratch" not in st:
        st["scratch"] = ctx.embedding_scratch(st["M"], st["rows"], st["vocab"], st["d"])
    ctx.abs_embedding_backward(st["dY"], st["tokens"], st["dE"], st["scratch"], scale=st["scale"], accumulate=st["add"])
    return {"dE": st["dE"]}


_PLAIN = {"attn_fwd": _plain_attn_fwd, "attn_bwd": _plain_attn_bwd, "rms_fwd": _plain_rms_fwd, "rms_bwd": _plain_rms_bwd,
          "emb_fwd": _plain_emb_fwd, "emb_bwd": _plain_emb_bwd}


def run(st):
    return _own(st) if own else _PLAIN[st["op"]](st)


# ---- what a pass cannot do without -----------------------------------------------------------------
def _distinct(vocab, rows):
    """How many tokens to expect among `rows` of them, each k with probability log((k + 2) / (k + 1)) / log(vocab + 1)."""
    norm, total, k = math.log(vocab + 1.0), 0.0, 0
    while k < vocab:                                     # in runs of nearly equal probability
        step = max(1, min(k // 16, vocab - k))
        p = math.log((k + step + 1.0) / (k + 1.0)) / norm / step
        total += step * (1.0 - (1.0 - p) ** rows)
        k += step
    return total


def work(case):
    op, es = case["op"], 4 if case["dtype"] == "f32" else 2
    if op in ("attn_fwd", "attn_bwd"):
        lens = _lens(case)
        pairs, rows = sum(n * (n + 1) // 2 for n in lens) * case["hq"], sum(lens)
        q, kv, lse = rows * case["hq"] * case["hd"] * es, rows * case["hk"] * case["hd"] * es, rows * case["hq"] * 4
        if op == "attn_fwd":
            return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * case["hd"] * pairs}
        return {"bytes": 4 * q + 4 * kv + lse, "flops": 10 * case["hd"] * pairs}
    M, d = case["M"], case["d"]
    if op in ("rms_fwd", "rms_bwd"):
        rows = case["rows"] if op == "rms_fwd" else case["S"] * case["T"]
        elems = M * rows * d
        if op == "rms_fwd":
            each = es + (2 * es if case["residual"] else 0) + (1 if case["quant"] else es)
            return {"bytes": elems * each + M * rows * (8 if case["quant"] else 4) + 4 * M * d, "flops": 5 * elems}
        each = 3 * es + (es if case["residual"] else 0)
        extra = 4 * M * case["S"] * d if case["per_sample"] else 0
        return {"bytes": elems * each + 4 * M * rows + 8 * M * d + extra, "flops": 9 * elems}
    elems, used = M * case["rows"] * d, int(M * d * _distinct(case["vocab"], case["rows"]))
    if op == "emb_fwd":
        return {"bytes": 4 * used + elems * es + 4 * M * case["rows"], "flops": elems}
    table = 8 * used if case["add"] else 4 * M * case["vocab"] * d
    return {"bytes": table + elems * es + 4 * M * case["rows"], "flops": 2 * elems}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _exact_attention(st):
    """Sequence by sequence and query head by query head."""
    q, k, v = (x.double() for x in _split(st, st["QKV"]))
    group = st["hq"] // st["hk"]
    backward = st["op"] == "attn_bwd"
    o, lse = st["O"].double(), st["lse"].double()
    dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v))
    start = 0
    for n in _lens(st):
        at = slice(start, start + n)
        start += n
        if n == 0:
            continue
        looks = torch.ones((n, n), device="cuda", dtype=torch.bool).tril()
        for h in range(st["hq"]):
            g = h // group
            w = (q[at, h] * st["scale"]) @ k[at, g].T
            if not backward:
                w = torch.where(looks, w, torch.full_like(w, -math.inf))
                total = torch.logsumexp(w, 1)
                o[at, h] = torch.exp(w - total[:, None]) @ v[at, g]
                lse[h, at] = total
                continue
            w = torch.where(looks, torch.exp(w - lse[h, at][:, None]), torch.zeros_like(w))
            do = st["dO"][at, h].double()
            dv[at, g] += w.T @ do
            w *= do @ v[at, g].T - torch.einsum("td,td->t", do, o[at, h])[:, None]
            w *= st["scale"]
            dq[at, h] = w @ k[at, g]
            dk[at, g] += w.T @ q[at, h]
    return {"dQKV": torch.cat([dq, dk, dv], 1)} if backward else {"O": o, "lse": lse}


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op in ("attn_fwd", "attn_bwd"):
        return _exact_attention(st)
    M, d = case["M"], case["d"]
    if op in ("rms_fwd", "rms_bwd"):
        w = st["weight"].double()[:, None, :]
        if op == "rms_fwd":
            h = st["X"].double()
            out = {}
            if case["residual"]:
                h = (h + st["R"].double()).to(st["X"].dtype).double()
                out["H"] = h
            norm = torch.linalg.vector_norm(h, dim=2, keepdim=True)
            root = 1.0 / torch.sqrt(norm * norm / d + RMS_EPS)
            y = w * (h * root)
            out["rstd"] = root.squeeze(2)
            if case["quant"]:
                scale = torch.linalg.vector_norm(y, ord=math.inf, dim=2, keepdim=True) / E4M3_MAX
                scale[scale == 0] = 1.0
                out["Q"], out["scales"] = None, scale.squeeze(2)
            else:
                out["Y"] = y
            return out
        h, dy, rstd = st["H"].double(), st["dY"].double(), st["rstd"].double()[:, :, None]
        c = torch.einsum("mrd,mrd,mrd->mr", dy, w.expand_as(dy), h)[:, :, None] / d
        dx = rstd * (w * dy) - rstd ** 3 * c * h
        if case["residual"]:
            dx = dx + st["dH"].double()
        seg = (M, case["S"], case["T"], d)
        gw = torch.einsum("mstd,mstd->msd", dy.reshape(seg), (h * rstd).reshape(seg))
        out = {"dX": dx, "dW": gw.sum(1)}
        if case["per_sample"]:
            out["G"] = gw
        return out
    if op == "emb_fwd":
        return {"Y": torch.stack([st["scale"] * st["E"][m].double().index_select(0, st["tokens"][m].long()) for m in range(M)])}
    out = []
    for m in range(M):
        into = st["dE"][m].double() if case["add"] else torch.zeros((case["vocab"], d), device="cuda", dtype=torch.float64)
        out.append(into.index_add_(0, st["tokens"][m].long(), st["scale"] * st["dY"][m].double()))
    return {"dE": torch.stack(out)}
