"""Host-side planning of the layer norm's backward pass (no GPU): every place that its CTAs write in the workspace lies
inside the workspace and has one writer, and the CTAs' runs cover all rows."""
import ctypes
import random

import pytest

import paper_2406_13936_b200 as pkg
from paper_2406_13936_b200 import binding

MIB = 1 << 20


def check(dtype, M, samples, tokens, d, gw, gb, totals, workspace_bytes, aligned=True, sm_count=148):
    p = pkg.plan_layer_norm_backward(dtype, M, samples, tokens, d, aligned, gw, gb, totals, sm_count, workspace_bytes)
    total, T, per = M * samples * tokens, p["tokens"], p["rows_per_cta"]
    assert p["samples"] * T == samples * tokens
    assert p["room"] * 2 * d * 4 <= workspace_bytes
    if total == 0:
        return p
    assert (p["ctas"] - 1) * per < total <= p["ctas"] * per          # every CTA has rows, every row has a CTA
    assert per < 1 << 31
    places = []
    for c in range(p["ctas"]):
        first, end = c * per, min((c + 1) * per, total)
        s, last = first // T, (end - 1) // T
        if p["direct"]:
            # segments that lie within the CTA need no place: at most the first and the last do
            for seg in sorted({s, last}):
                if seg * T >= first and (seg + 1) * T <= end:
                    continue
                places.append(2 * c + (1 if seg * T > first else 0))
        else:
            places.extend(range(c + s, c + last + 1))
    if gw or gb or totals:
        assert len(set(places)) == len(places)
        assert max(places, default=-1) < p["room"]
        assert len(places) == 0 or max(places) < p["used"]
        assert p["used"] <= p["room"]
        if totals and p["parts"] > 1:
            assert p["used"] + M * p["parts"] <= p["room"]
    return p


def outputs():
    return [(True, False, False), (False, True, False), (True, False, True), (True, True, False), (True, True, True), (False, False, True)]


def test_struct_size():
    assert ctypes.sizeof(binding.LnBackwardPlan) == 72


@pytest.mark.parametrize("samples,tokens", [(14738, 23), (14000, 4), (12345, 2), (15000, 3), (9001, 8), (13000, 16)])
def test_one_gradient_of_many_short_samples(samples, tokens):
    """Only Gw: a place for every sample and one for every CTA.  With fp32 rows of 512 the default workspace has 16384."""
    for d in (512, 768, 1024):
        try:
            check("f32", 1, samples, tokens, d, True, False, False, 64 * MIB)
        except pkg.AbsError:
            assert samples + 1 > 64 * MIB // (8 * d)


@pytest.mark.parametrize("spare", [1, 2, 3, 7, 40])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,samples,tokens", [(1, 64, 2), (3, 50, 5), (2, 1000, 11), (1, 300, 23), (4, 7, 1), (1, 9, 200), (8, 1, 3)])
def test_a_workspace_with_barely_enough_places(M, samples, tokens, dtype, spare):
    for d in (32, 96, 257, 768, 4096, 9000):
        for gw, gb, totals in outputs():
            for aligned in (True, False):
                needed = (2 if gw and gb else M * (samples if gw or gb else 1) + 1) + spare - 1
                p = check(dtype, M, samples, tokens, d, gw, gb, totals, needed * 8 * d, aligned)
                assert p["needed"] <= needed


def test_many_rows():
    """Past 2^30 rows a CTA's share is limited: the CTAs that this takes have places too, or the call is refused."""
    for rows in (1 << 30, (1 << 30) + 5, 1 << 31, (1 << 32) + 1, 3 << 32):
        for places in (1, 2, 3, 5, 8, 200):
            try:
                check("bf16", 1, 1, rows, 1, False, False, True, places * 8)
            except pkg.AbsError:
                assert places < 2 + (rows >> 30)
            try:
                check("bf16", 1, 1, rows, 1, True, True, True, places * 8)
            except pkg.AbsError:
                assert places < 2 + 2 * (rows >> 30)


def test_random_shapes():
    rng = random.Random(5)
    for _ in range(1500):
        d = int(2 ** rng.uniform(0, 14))
        M, tokens = rng.randint(1, 8), int(2 ** rng.uniform(0, 9))
        samples = int(2 ** rng.uniform(0, 12))
        gw, gb, totals = rng.choice(outputs())
        segments = M * (samples if gw or gb else 1)
        places = rng.choice([2, segments + 1, segments + rng.randint(1, 3000), 2 + rng.randint(0, 400)])
        try:
            check(rng.choice(["f32", "bf16"]), M, samples, tokens, d, gw, gb, totals, places * 8 * d, rng.random() < 0.5,
                  rng.choice([148, 132, 16, 1]))
        except pkg.AbsError:
            assert places < (2 if gw and gb else segments + 1)


def test_nothing_and_refusals():
    assert check("f32", 2, 3, 0, 64, True, True, True, 4096)["ctas"] == 0
    assert check("f32", 2, 0, 0, 64, False, False, True, 4096)["ctas"] == 0
    for bad in (dict(M=0), dict(d=0), dict(samples=-1), dict(tokens=-1), dict(samples=1 << 30, tokens=1 << 30)):
        with pytest.raises(pkg.AbsError):
            pkg.plan_layer_norm_backward("f32", **{**dict(M=1, samples=2, tokens=3, d=8), **bad})
