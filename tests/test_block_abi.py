"""Sizes, host-side answers and refusals of the attention, RMS norm and embedding entry points (no GPU needed)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2406_13936_b200 as pkg
from paper_2406_13936_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("abs_rms_norm", "abs_rms_norm_backward", "abs_attention_plan_bytes", "abs_attention_plan", "abs_attention_scratch_bytes",
         "abs_attention", "abs_attention_backward", "abs_embedding", "abs_embedding_scratch_bytes", "abs_embedding_backward")


def size(name, *args):
    out = ctypes.c_size_t()
    return getattr(binding.load_library(), name)(*args, ctypes.byref(out)), out.value


def test_declared_and_bound():
    text = open(os.path.join(ROOT, "include", "abs.h")).read()
    for name in NAMES:
        assert re.search(r"^int %s\(" % name, text, flags=re.M)
        assert name in binding.EXPORTS
    assert ctypes.sizeof(binding.Heads) == 24


@pytest.mark.parametrize("sequences,total", [(0, 0), (1, 1), (7, 1000), (1000, 1000), (3, 1 << 20)])
def test_plan_holds_every_tile(sequences, total):
    rc, got = size("abs_attention_plan_bytes", sequences, total)
    # tiles of 256 and of 128 rows, 16 bytes each, of sequences that share `total` rows
    assert rc == 0 and got >= 64 + 16 * (total // 256 + sequences) + 16 * (total // 128 + sequences)


@pytest.mark.parametrize("args", [(-1, 5), (5, -1), (1 << 25, 5), (1, (1 << 30) + 1)])
def test_plan_refusals(args):
    assert size("abs_attention_plan_bytes", *args)[0] < 0
    assert binding.load_library().abs_last_error(None)


@pytest.mark.parametrize("args", [(100, 3, 2, 64, 1), (100, 0, 1, 64, 1), (100, 4, 0, 64, 1), (100, 4, 2, 0, 1), (100, 4, 2, 129, 1),
                                  (-1, 4, 2, 64, 1), (100, 8192, 1, 64, 1), (1 << 30, 8, 1, 64, 1), (100, 4, 2, 64, -1)])
def test_attention_scratch_refusals(args):
    assert size("abs_attention_scratch_bytes", *args)[0] < 0
    assert size("abs_attention_scratch_bytes", 100, 4, 2, 64, 1)[0] == 0


@pytest.mark.parametrize("args", [(0, 5, 5, 5), (1, -1, 5, 5), (1, 5, 0, 5), (1, 5, 5, 0), (70000, 5, 5, 5), (1, (1 << 28) + 1, 5, 5),
                                  (1, 5, 1 << 24, 5), (1, 5, 5, (1 << 24) + 1), (60000, 1 << 20, 5, 5)])
def test_embedding_scratch_refusals(args):
    assert size("abs_embedding_scratch_bytes", *args)[0] < 0
    assert size("abs_embedding_scratch_bytes", 1, 5, 5, 5)[0] == 0


class _Library:
    """Takes every call, does nothing and remembers the last one."""

    def __getattr__(self, name):
        def call(*args):
            self.last = name, args
            return 0
        return call


class _Stream:
    cuda_stream = 0


def context():
    """A context whose library does nothing; its device is the CPU's, so its tensors may be there."""
    ctx = pkg.Context.__new__(pkg.Context)
    ctx._lib, ctx._h, ctx.device = _Library(), None, -1
    return ctx


S = _Stream()


def heads(total, n, hd, dtype=torch.float32):
    return torch.zeros((total, n, hd), dtype=dtype)


def plan(total, sequences=1):
    return pkg.AttentionPlan(torch.zeros(64, dtype=torch.int32), sequences, total)


def test_calls_return_the_tensor_that_they_were_given():
    ctx = context()
    for shape in ((4, 8), (2, 4, 8)):
        x, y = torch.zeros(shape), torch.zeros(shape)
        assert ctx.abs_rms_norm(x, None, 1e-5, y, stream=S) is y
        q, s = torch.zeros(shape, dtype=torch.uint8), torch.zeros(shape[:-1])
        assert ctx.abs_rms_norm(x, None, 1e-5, None, Q=q, scales=s, stream=S) is q
        tokens, table = torch.zeros(shape[:-1], dtype=torch.int32), torch.zeros(shape)
        assert ctx.abs_embedding(table, tokens, y, stream=S) is y
        assert ctx.abs_embedding_backward(y, tokens, table, torch.zeros(9, dtype=torch.uint8), stream=S) is table
    q, o = heads(6, 4, 8), heads(6, 4, 8)
    assert ctx.abs_attention(q, heads(6, 2, 8), heads(6, 2, 8), plan(6), o, stream=S) is o


def test_views_of_a_fused_tensor_are_passed_by_their_strides():
    ctx = context()
    fused = torch.zeros((6, 8 * 16))
    q, k, v = (t.unflatten(1, (-1, 16)) for t in (fused[:, :64], fused[:, 64:96], fused[:, 96:]))
    ctx.abs_attention(q, k, v, plan(6), heads(6, 4, 16), stream=S)
    name, args = ctx._lib.last
    assert name == "abs_attention"
    for t, view in zip(args[1:4], (q, k, v)):
        assert (t.data, t.row_stride, t.head_stride) == (view.data_ptr(), 128, 16)


@pytest.mark.parametrize("change", ["k_heads", "v_type", "o_shape", "plan", "lse_shape", "lse_type", "columns", "dims", "double"])
def test_attention_refuses(change):
    q, k, v, o, p = heads(6, 4, 8), heads(6, 2, 8), heads(6, 2, 8), heads(6, 4, 8), plan(6)
    lse = torch.zeros((4, 6))
    if change == "k_heads":
        k = heads(6, 3, 8)
    elif change == "v_type":
        v = v.to(torch.bfloat16)
    elif change == "o_shape":
        o = heads(5, 4, 8)
    elif change == "plan":
        p = plan(7)
    elif change == "lse_shape":
        lse = torch.zeros((6, 4))
    elif change == "lse_type":
        lse = lse.double()
    elif change == "columns":
        v = torch.zeros((6, 2, 16))[:, :, ::2]
    elif change == "dims":
        q = q[0]
    elif change == "double":
        q, k, v, o = (t.double() for t in (q, k, v, o))
    with pytest.raises(pkg.AbsError):
        context().abs_attention(q, k, v, p, o, lse, stream=S)
    with pytest.raises(pkg.AbsError):
        context().abs_attention_backward(o, q, k, v, o, lse, p, o, k, v, torch.zeros(9), stream=S)


def test_attention_backward_needs_lse():
    q, k = heads(6, 4, 8), heads(6, 2, 8)
    with pytest.raises(pkg.AbsError, match="lse"):
        context().abs_attention_backward(q, q, k, k, q, None, plan(6), q, k, k, torch.zeros(9), stream=S)


@pytest.mark.parametrize("offsets", [torch.zeros(3, dtype=torch.int64), torch.zeros((2, 2), dtype=torch.int32),
                                     torch.zeros(0, dtype=torch.int32), torch.zeros(6, dtype=torch.int32)[::2]])
def test_plan_refuses_other_offsets(offsets):
    with pytest.raises(pkg.AbsError, match="offsets"):
        context().attention_plan(offsets, 10, stream=S)


def test_plan_of_another_batch_is_refused():
    with pytest.raises(pkg.AbsError, match="plan is for"):
        context().attention_plan(torch.zeros(3, dtype=torch.int32), 10, plan=plan(10, 3), stream=S)


@pytest.mark.parametrize("change", ["residual_type", "summed_shape", "nothing", "scales", "q_type", "q_shape", "rstd", "weight", "columns"])
def test_rms_norm_refuses(change):
    kw = dict(residual=torch.zeros((2, 4, 8)), summed=torch.zeros((2, 4, 8)), rstd=torch.zeros((2, 4)),
              Q=torch.zeros((2, 4, 8), dtype=torch.uint8), scales=torch.zeros((2, 4)))
    x, y, w = torch.zeros((2, 4, 8)), torch.zeros((2, 4, 8)), torch.zeros((2, 8))
    if change == "residual_type":
        kw["residual"] = kw["residual"].to(torch.bfloat16)
    elif change == "summed_shape":
        kw["summed"] = torch.zeros((2, 4, 9))
    elif change == "nothing":
        y, kw["Q"], kw["scales"] = None, None, None
    elif change == "scales":
        kw["scales"] = None
    elif change == "q_type":
        kw["Q"] = kw["Q"].to(torch.int8)
    elif change == "q_shape":
        kw["Q"] = kw["Q"][:, :2]
    elif change == "rstd":
        kw["rstd"] = torch.zeros((2, 5))
    elif change == "weight":
        w = torch.zeros((2, 9))
    elif change == "columns":
        x = torch.zeros((2, 4, 16))[:, :, ::2]
    with pytest.raises(pkg.AbsError):
        context().abs_rms_norm(x, w, 1e-6, y, stream=S, **kw)


@pytest.mark.parametrize("samples", [0, -1, 3])
def test_rms_norm_backward_refuses_unequal_samples(samples):
    x = torch.zeros((1, 4, 8))
    with pytest.raises(pkg.AbsError, match="samples"):
        context().abs_rms_norm_backward(x, x, torch.zeros((1, 4)), None, samples=samples, stream=S)


@pytest.mark.parametrize("change", ["table_type", "tokens_type", "tokens_shape", "width", "workers"])
def test_embedding_refuses(change):
    E, tokens, Y = torch.zeros((2, 10, 8)), torch.zeros((2, 4), dtype=torch.int32), torch.zeros((2, 4, 8))
    if change == "table_type":
        E = E.to(torch.bfloat16)
    elif change == "tokens_type":
        tokens = tokens.long()
    elif change == "tokens_shape":
        tokens = tokens[:, :3]
    elif change == "width":
        Y = torch.zeros((2, 4, 9))
    elif change == "workers":
        Y = torch.zeros((3, 4, 8))
    with pytest.raises(pkg.AbsError):
        context().abs_embedding(E, tokens, Y, stream=S)
    with pytest.raises(pkg.AbsError):
        context().abs_embedding_backward(Y, tokens, E, torch.zeros(9), stream=S)
