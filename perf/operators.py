"""Cases for timing and checking the layer-norm and matrix-optimiser operators.

Four operators: layer norm forward, layer norm backward (with the weight gradient per sample or in
total), orthogonalisation by Newton-Schulz products, and the local Muon step built on it.  `run`
computes each in its plain form, elementary torch operations in fp32, or, where `own` is set, through
the package's Context.  Everything runs on cuda:0.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NS = (3.4445, -4.7750, 2.0315)      # coefficients of the quintic that users of Muon take
NS_EPS = 1e-7
LN_EPS = 1e-5


# ---- cases ---------------------------------------------------------------------------------------
def listed():
    return [
        # a handful of token rows of the 768-wide language model: latency is all there is
        dict(name="ln_fwd_few_rows", op="ln_fwd", M=1, rows=4, d=768, pad=0, dtype="bf16", bias=True),
        # 8 workers, micro-batches of 16 sequences of 1024 tokens, one layer norm of that model
        dict(name="ln_fwd_lm", op="ln_fwd", M=8, rows=16384, d=768, pad=0, dtype="bf16", bias=True),
        # fp32 rows of an odd width inside wider rows, no bias: nothing is 16-byte aligned
        dict(name="ln_fwd_odd", op="ln_fwd", M=3, rows=2049, d=1021, pad=10, dtype="f32", bias=False),
        # per-sample gradients of a classifier's norm (one row a sample), a few samples a worker
        dict(name="ln_bwd_few_rows", op="ln_bwd", M=2, S=8, T=1, d=257, pad=0, dtype="f32", per_sample=True),
        # backward of ln_fwd_lm with one gradient row per sequence for the batch-size test
        dict(name="ln_bwd_lm", op="ln_bwd", M=8, S=16, T=1024, d=768, pad=0, dtype="bf16", per_sample=True),
        # a wide fp32 layer on a short run of ragged length, totals only
        dict(name="ln_bwd_wide", op="ln_bwd", M=1, S=1, T=6001, d=4096, pad=0, dtype="f32", per_sample=False),
        # the last layer of the 784-1024-1024-10 network, 8 replicas
        dict(name="orth_head", op="orth", batch=8, m=10, n=1024, src="bf16", dst="bf16", steps=5),
        # the first layer of that network (taller than wide), fp32 result to fp32 accuracy
        dict(name="orth_mlp_f32", op="orth", batch=8, m=1024, n=784, src="f32", dst="f32", steps=5),
        # one large square matrix
        dict(name="orth_large", op="orth", batch=1, m=4096, n=4096, src="bf16", dst="bf16", steps=5),
        # a small adapter matrix on 4 replicas
        dict(name="muon_small", op="muon", M=4, L=1, m=64, n=192, steps=5, nesterov=True, average=False),
        # the middle layer of the 784-1024-1024-10 network, 8 replicas, last local step of a round
        dict(name="muon_mlp", op="muon", M=8, L=1, m=1024, n=1024, steps=5, nesterov=False, average=True),
        # the attention output matrices of the 12-layer, 768-wide language model, 8 replicas
        dict(name="muon_lm", op="muon", M=8, L=12, m=768, n=768, steps=5, nesterov=True, average=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "orth", "muon"])
    if op in ("ln_fwd", "ln_bwd"):
        d = _log(rng, 32, 8192)
        if rng.random() < 0.6:
            d = max(32, d // 8 * 8)
        M = rng.randint(1, 8)
        rows = _log(rng, 1, min(40000, max(2, 80_000_000 // (M * d))))
        dtype = rng.choice(["f32", "bf16"])
        pad = rng.choice([0, 0, 8, 3])
        if op == "ln_fwd":
            return dict(op=op, M=M, rows=rows, d=d, pad=pad, dtype=dtype, bias=rng.random() < 0.8)
        S = _log(rng, 1, min(64, rows))
        return dict(op=op, M=M, S=S, T=max(1, rows // S), d=d, pad=pad, dtype=dtype, per_sample=rng.random() < 0.5)
    m, n = _log(rng, 16, 2500), _log(rng, 16, 2500)
    lo = min(m, n)
    most = max(1, int(2.0e10 / (3.0 * lo * lo * max(m, n) + lo ** 3)))
    if op == "orth":
        src, dst = rng.choice([("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        return dict(op=op, batch=rng.randint(1, min(8, most)), m=m, n=n, src=src, dst=dst, steps=rng.choice([3, 5, 6]))
    M = rng.randint(1, min(8, most))
    L = rng.randint(1, max(1, min(6, most // M)))
    return dict(op=op, M=M, L=L, m=m, n=n, steps=rng.choice([4, 5]), nesterov=rng.random() < 0.5,
                average=rng.random() < 0.5)


# ---- inputs --------------------------------------------------------------------------------------
def _rows(gen, M, rows, d, pad, dtype, scale, offset):
    """[M, rows, d] activations inside rows of d + pad: every row has a scale and an offset of its own."""
    full = torch.randn((M, rows, d + pad), device="cuda", generator=gen)
    s = torch.rand((M, rows, 1), device="cuda", generator=gen) + 0.5
    o = torch.randn((M, rows, 1), device="cuda", generator=gen)
    return (full * (scale * s) + offset * o).to(dtype)[:, :, :d]


def _gradients(gen, batch, m, n, scale):
    """[batch, m, n] matrices like a layer's gradient: outer products of falling weight, and noise."""
    r = max(1, min(m, n) // 8)
    w = torch.arange(1, r + 1, device="cuda", dtype=torch.float32).rsqrt()
    low = (torch.randn((batch, m, r), device="cuda", generator=gen) * w) @ torch.randn((batch, r, n), device="cuda", generator=gen)
    low = low / low.square().mean(dim=(1, 2), keepdim=True).sqrt()
    return scale * (low + 0.3 * torch.randn((batch, m, n), device="cuda", generator=gen))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    st = dict(case)
    if op in ("ln_fwd", "ln_bwd"):
        M, d, dt = case["M"], case["d"], TYPES[case["dtype"]]
        rows = case["rows"] if op == "ln_fwd" else case["S"] * case["T"]
        # the replicas' parameter vectors: the norm's weight and bias lie inside a longer flat vector
        params = torch.randn((M, 2 * d + 64), device="cuda", generator=gen) * 0.1
        params[:, :d] += 1.0
        st["weight"] = params[:, :d]
        st["bias"] = params[:, d:2 * d] if case.get("bias", True) else None
        st["X"] = _rows(gen, M, rows, d, case["pad"], dt, 1.0, 0.5)
        if op == "ln_fwd":
            st["Y"] = torch.empty((M, rows, d), device="cuda", dtype=dt)
            st["mean"], st["rstd"] = (torch.empty((M, rows), device="cuda") for _ in range(2))
            return st
        S = case["S"]
        x = st["X"].double()
        st["mean"] = x.mean(2).float()
        st["rstd"] = (x.var(2, unbiased=False) + LN_EPS).rsqrt().float()
        st["dY"] = _rows(gen, M, rows, d, case["pad"], dt, 1e-3, 1e-4)
        st["dX"] = torch.empty((M, rows, d), device="cuda", dtype=dt)
        st["dW"], st["dB"] = (torch.empty((M, d), device="cuda") for _ in range(2))
        st["G"] = torch.empty((M, S, 2 * d), device="cuda") if case["per_sample"] else None
        return st
    if op == "orth":
        st["G"] = _gradients(gen, case["batch"], case["m"], case["n"], 1e-3).to(TYPES[case["src"]])
        st["O"] = torch.empty(st["G"].shape, device="cuda", dtype=TYPES[case["dst"]])
        return st
    M, L, m, n = case["M"], case["L"], case["m"], case["n"]
    size = L * m * n
    # flat parameter vectors, one a replica; the L matrices are the first part of each
    view = (M, L, m, n)
    for name in ("X", "Buf", "Gb"):
        flat = torch.empty((M, size + 64), device="cuda")
        st[name] = flat[:, :size].view(view)
    x0 = torch.randn((L, m, n), device="cuda", generator=gen) * 0.02
    st["X"].copy_(x0 + 1e-4 * torch.randn(view, device="cuda", generator=gen))
    st["Gb"].copy_(_gradients(gen, M * L, m, n, 1e-3).view(view))
    st["Buf"].copy_(_gradients(gen, M * L, m, n, 5e-3).view(view))
    st["lr"], st["momentum"], st["wd"] = 3e-4, 0.95, 0.1
    st["scale"] = 0.2 * math.sqrt(max(m, n))
    return st


# ---- the plain forms -----------------------------------------------------------------------------
def _plain_ln_fwd(st):
    x = st["X"].float()
    mean = x.mean(2, keepdim=True)
    xc = x - mean
    rstd = torch.rsqrt((xc * xc).mean(2, keepdim=True) + LN_EPS)
    y = xc * rstd * st["weight"].unsqueeze(1)
    if st["bias"] is not None:
        y = y + st["bias"].unsqueeze(1)
    return {"Y": y.to(st["X"].dtype), "mean": mean.squeeze(2), "rstd": rstd.squeeze(2)}


def _plain_ln_bwd(st):
    x, dy = st["X"].float(), st["dY"].float()
    M, rows, d = x.shape
    rstd = st["rstd"].unsqueeze(2)
    xh = (x - st["mean"].unsqueeze(2)) * rstd
    a = dy * st["weight"].unsqueeze(1)
    dx = rstd * (a - a.mean(2, keepdim=True) - xh * (a * xh).mean(2, keepdim=True))
    p = dy * xh
    out = {"dX": dx.to(st["X"].dtype)}
    if st["per_sample"]:
        gw = p.view(M, st["S"], st["T"], d).sum(2)
        gb = dy.reshape(M, st["S"], st["T"], d).sum(2)
        out["G"] = torch.cat([gw, gb], 2)
        out["dW"], out["dB"] = gw.sum(1), gb.sum(1)
    else:
        out["dW"], out["dB"] = p.sum(1), dy.sum(1)
    return out


def _plain_newton_schulz(g, steps):
    """g [batch, m, n] fp32."""
    a, b, c = NS
    tall = g.shape[1] > g.shape[2]
    x = g.transpose(1, 2) if tall else g
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    for _ in range(steps):
        A = x @ x.transpose(1, 2)
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.transpose(1, 2) if tall else x


def _plain_muon(st):
    M, L, m, n = st["X"].shape
    buf = st["Buf"] * st["momentum"] + st["Gb"]
    u = st["Gb"] + st["momentum"] * buf if st["nesterov"] else buf
    o = _plain_newton_schulz(u.reshape(M * L, m, n), st["steps"]).reshape(M, L, m, n)
    x = st["X"] * (1.0 - st["lr"] * st["wd"]) - (st["lr"] * st["scale"]) * o
    if st["average"]:
        x = x.mean(0, keepdim=True).expand(M, L, m, n)
    st["Buf"].copy_(buf)
    st["X"].copy_(x)
    return {"X": st["X"], "Buf": st["Buf"]}


# ---- the package's operators ---------------------------------------------------------------------
_kept = {}


def _context():
    """The context and the scratch that a program keeps from call to call."""
    if "ctx" not in _kept:
        import paper_2406_13936_b200 as pkg
        _kept["pkg"], _kept["ctx"] = pkg, pkg.Context(0)
    return _kept["pkg"], _kept["ctx"]


def _own(st):
    pkg, ctx = _context()
    op = st["op"]
    if op == "ln_fwd":
        ctx.abs_layer_norm(st["X"], st["weight"], st["bias"], LN_EPS, st["Y"], st["mean"], st["rstd"])
        return {"Y": st["Y"], "mean": st["mean"], "rstd": st["rstd"]}
    if op == "ln_bwd":
        d, G = st["d"], st["G"]
        out = {"dX": st["dX"], "dW": st["dW"], "dB": st["dB"]}
        if G is not None:
            ctx.abs_layer_norm_backward(st["dY"], st["X"], st["mean"], st["rstd"], st["weight"], st["dX"], st["dW"],
                                        st["dB"], samples=st["S"], Gw=G[:, :, :d], Gb=G[:, :, d:])
            out["G"] = G
        else:
            ctx.abs_layer_norm_backward(st["dY"], st["X"], st["mean"], st["rstd"], st["weight"], st["dX"], st["dW"],
                                        st["dB"])
        return out
    if "cfg" not in st:      # what a program sets up once: options and scratch
        a, b, c = NS
        precision = "f32" if st.get("dst") == "f32" else "f16"
        ns = pkg.make_ns_cfg(steps=st["steps"], a=a, b=b, c=c, eps=NS_EPS, precision=precision)
        if op == "orth":
            st["cfg"] = ns
            st["scratch"] = ctx.ns_scratch(st["batch"], st["m"], st["n"], ns)
        else:
            st["cfg"] = pkg.make_muon_cfg(lr=st["lr"], momentum=st["momentum"], weight_decay=st["wd"],
                                          scale=st["scale"], nesterov=st["nesterov"], ns=ns)
            st["scratch"] = ctx.ns_scratch(st["M"] * st["L"], st["m"], st["n"], ns)
    if op == "orth":
        ctx.abs_orthogonalise(st["G"], st["O"], st["cfg"], st["scratch"])
        return {"O": st["O"]}
    ctx.local_muon_step(st["X"], st["Buf"], st["Gb"], st["cfg"], st["scratch"], average_after=st["average"])
    return {"X": st["X"], "Buf": st["Buf"]}


def run(st):
    if own:
        return _own(st)
    op = st["op"]
    if op == "ln_fwd":
        return _plain_ln_fwd(st)
    if op == "ln_bwd":
        return _plain_ln_bwd(st)
    if op == "orth":
        return {"O": _plain_newton_schulz(st["G"].float(), st["steps"]).to(TYPES[st["dst"]])}
    return _plain_muon(st)


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    op = case["op"]
    if op in ("ln_fwd", "ln_bwd"):
        es = 4 if case["dtype"] == "f32" else 2
        M, d = case["M"], case["d"]
        rows = case["rows"] if op == "ln_fwd" else case["S"] * case["T"]
        elems = M * rows * d
        if op == "ln_fwd":
            return {"bytes": 2 * elems * es + 8 * M * rows + (8 if case["bias"] else 4) * M * d, "flops": 7 * elems}
        extra = 8 * M * case["S"] * d if case["per_sample"] else 0
        return {"bytes": 3 * elems * es + 8 * M * rows + 12 * M * d + extra, "flops": 14 * elems}
    lo, hi = min(case["m"], case["n"]), max(case["m"], case["n"])
    batch = case["batch"] if op == "orth" else case["M"] * case["L"]
    # A = X X' and A A are symmetric: half of each product is enough
    flops = case["steps"] * batch * (lo * lo * hi + lo ** 3 + 2 * lo * lo * hi)
    if op == "orth":
        es = (4 if case["src"] == "f32" else 2) + (4 if case["dst"] == "f32" else 2)
        return {"bytes": batch * lo * hi * es, "flops": flops}
    return {"bytes": batch * lo * hi * 20, "flops": flops + 8 * batch * lo * hi}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _ns64(u, steps):
    """The iteration on the longer side's Gram matrix, (X'X) acting from the right, in Horner form."""
    a, b, c = NS
    tall = u.shape[-2] > u.shape[-1]
    y = u if tall else u.mT
    y = y / (torch.linalg.matrix_norm(y).reshape(*y.shape[:-2], 1, 1) + NS_EPS)
    eye = torch.eye(y.shape[-1], device=u.device, dtype=u.dtype)
    for _ in range(steps):
        gram = y.mT @ y
        y = y @ (a * eye + gram @ (b * eye + c * gram))
    return y if tall else y.mT


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op in ("ln_fwd", "ln_bwd"):
        x, w = st["X"].double(), st["weight"].double()[:, None, :]
        if op == "ln_fwd":
            mean = x.sum(2) / case["d"]
            var = ((x - mean[:, :, None]) ** 2).sum(2) / case["d"]
            rstd = 1.0 / torch.sqrt(var + LN_EPS)
            y = (x - mean[:, :, None]) * rstd[:, :, None] * w
            if st["bias"] is not None:
                y += st["bias"].double()[:, None, :]
            return {"Y": y, "mean": mean, "rstd": rstd}
        dy, rstd = st["dY"].double(), st["rstd"].double()[:, :, None]
        xh = (x - st["mean"].double()[:, :, None]) * rstd
        c1 = torch.einsum("mrd,mrd->mr", dy, w.expand_as(dy)) / case["d"]
        c2 = torch.einsum("mrd,mrd,mrd->mr", dy, w.expand_as(dy), xh) / case["d"]
        dx = rstd * (dy * w - c1[:, :, None] - xh * c2[:, :, None])
        seg = (case["M"], case["S"], case["T"], case["d"])
        gw = torch.einsum("mstd,mstd->msd", dy.reshape(seg), xh.reshape(seg))
        gb = torch.einsum("mstd->msd", dy.reshape(seg))
        out = {"dX": dx, "dW": gw.sum(1), "dB": gb.sum(1)}
        if case["per_sample"]:
            out["G"] = torch.cat([gw, gb], 2)
        return out
    if op == "orth":
        return {"O": _ns64(st["G"].double(), case["steps"])}
    g, mu = st["Gb"].double(), st["momentum"]
    buf = mu * st["Buf"].double() + g
    u = g + mu * buf if case["nesterov"] else buf
    x = (1.0 - st["lr"] * st["wd"]) * st["X"].double() - st["lr"] * st["scale"] * _ns64(u, case["steps"])
    if case["average"]:
        x = x.sum(0, keepdim=True).expand_as(x) / case["M"]
    return {"X": x, "Buf": buf}
