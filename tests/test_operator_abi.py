"""Sizes and host-side answers of the layer-norm, orthogonalisation and Muon entry points (no GPU needed)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2406_13936_b200 as pkg
from paper_2406_13936_b200 import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def scratch(count, rows, cols, **kw):
    cfg, out = pkg.make_ns_cfg(**kw), ctypes.c_size_t()
    rc = binding.load_library().abs_ns_scratch_bytes(count, rows, cols, ctypes.byref(cfg), ctypes.byref(out))
    return rc, out.value


def test_struct_sizes():
    assert ctypes.sizeof(binding.NsCfg) == 24
    assert ctypes.sizeof(binding.MuonCfg) == 48


def test_declared_and_bound():
    text = open(os.path.join(ROOT, "include", "abs.h")).read()
    for name in ("abs_ns_scratch_bytes", "abs_orthogonalise", "local_muon_step", "abs_layer_norm", "abs_layer_norm_backward"):
        assert re.search(r"^int %s\(" % name, text, flags=re.M)
        assert name in binding.EXPORTS


@pytest.mark.parametrize("m,n", [(1, 1), (10, 1024), (128, 1000), (129, 300), (784, 1024), (2048, 2048)])
@pytest.mark.parametrize("precision", ["f16", "f32"])
def test_scratch_is_the_same_for_either_orientation_and_enough_for_one_matrix(m, n, precision):
    rc, one = scratch(1, m, n, precision=precision)
    assert rc == 0 and scratch(1, n, m, precision=precision) == (0, one)
    if min(m, n) > 128:                      # X twice (values) and once (remainders), A and B, two bytes each
        assert one >= 2 * (3 * m * n + 2 * min(m, n) ** 2)


def test_scratch_of_many_matrices_is_bounded():
    """Matrices are worked off in groups: past some number the scratch stops growing."""
    sizes = [scratch(count, 768, 768)[1] for count in (1, 8, 64, 512, 4096)]
    assert sizes[0] < sizes[1] < 300 << 20
    assert max(sizes) < 300 << 20


@pytest.mark.parametrize("count,rows,cols,kw", [
    (0, 8, 8, {}), (-1, 8, 8, {}), (1, 0, 8, {}), (1, 8, 0, {}), (1, -3, 8, {}), (1, 1 << 20, 8, {}),
    (1, 8, 8, dict(steps=0)), (1, 8, 8, dict(steps=1000)), (1, 8, 8, dict(a=float("nan"))), (1, 8, 8, dict(eps=-1.0))])
def test_scratch_refusals(count, rows, cols, kw):
    rc, _ = scratch(count, rows, cols, **kw)
    assert rc < 0
    assert binding.load_library().abs_last_error(None)


def test_unknown_precision():
    with pytest.raises(KeyError):
        pkg.make_ns_cfg(precision="f8")


@pytest.mark.parametrize("m,n,precision", [(300, 520, "f32"), (768, 768, "f16"), (18, 2474, "f16"), (10, 1024, "f32"), (4096, 4096, "f16"),
                                           (129, 129, "f16"), (86, 2085, "f32")])
def test_scratch_of_any_number_is_enough_for_one(m, n, precision):
    """... which is the least that a call takes: whatever scratch was made for, fewer matrices can use it."""
    one = scratch(1, m, n, precision=precision)[1]
    assert all(scratch(count, m, n, precision=precision)[1] >= one for count in list(range(1, 120)) + [1000, 1 << 20])


class _Library:
    """Takes every call and does nothing."""

    def __getattr__(self, name):
        return lambda *args: 0


def context():
    """A context whose library does nothing; its device is the CPU's, so its tensors may be there."""
    ctx = pkg.Context.__new__(pkg.Context)
    ctx._lib, ctx._h, ctx.device = _Library(), None, -1
    return ctx


class _Stream:
    cuda_stream = 0


def test_calls_return_the_tensor_that_they_were_given():
    ctx, s = context(), _Stream()
    for shape in ((4, 8), (2, 4, 8)):
        x, y = torch.zeros(shape), torch.zeros(shape)
        assert ctx.abs_layer_norm(x, None, None, 1e-5, y, stream=s) is y
        assert ctx.abs_orthogonalise(x, y, pkg.make_ns_cfg(), torch.zeros(10, dtype=torch.uint8), stream=s) is y


@pytest.mark.parametrize("shape", [(8, 8), (8,), (1, 2, 2, 4, 4)])
def test_muon_refuses_other_dimensions(shape):
    x = torch.zeros(shape)
    with pytest.raises(pkg.AbsError, match="M, L, rows, cols"):
        context().local_muon_step(x, x, x, pkg.make_muon_cfg(0.1), torch.zeros(10, dtype=torch.uint8), stream=_Stream())
