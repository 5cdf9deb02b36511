"""The cases of perf/more_operators.py at small sizes: the framework's calls and the plain forms against the 64-bit results, so that what is timed is known to be the operator.

Tolerances, of a tensor's error over its size (root of the sum of squares; u: half a unit in the last place of its type, relative):
  whole numbers, codes in 8 bits: equal.
  rounded once to 16 bits: u, which a rounding's own mean (u / sqrt 3 at most) and fp32's 2^-18 stay below; from 8-bit operands 2^-11 more, for what the instructions cut off: a
  product's part below 2^-13 of the largest of sixteen, always towards zero, of sums some of whose terms cancel.
  fp32: 2^-18."""
import importlib.util
import os
import random

import pytest
import torch

import gpu_util as G

pytestmark = pytest.mark.gpu

_path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "more_operators.py")
_spec = importlib.util.spec_from_file_location("perf_more_operators", _path)
P = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(P)
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -18}

CASES = [
    dict(kind="route", tokens=1, experts=64, top=6, score="softmax", bias=False, dtype="f32", padded=0), dict(kind="route", tokens=203, experts=256, top=8, score="sigmoid", bias=True, dtype="bf16", padded=3),
    dict(kind="quantize", rows=7, cols=1000, rows_of_block=1, dtype="f16"), dict(kind="quantize", rows=133, cols=300, rows_of_block=128, dtype="bf16"),
    dict(kind="product", rows=1, n_in=1024, n_out=96, gated=False, dtype="e4m3", scale="e8m0", out="f16"), dict(kind="product", rows=200, n_in=333, n_out=130, gated=True, dtype="e4m3", scale="f32", out="bf16"),
    dict(kind="product", rows=70, n_in=520, n_out=65, gated=True, dtype="f16", scale="none", out="f32"), dict(kind="product", rows=9, n_in=640, n_out=257, gated=False, dtype="e4m3", scale="f32", out="f32"),
    dict(kind="experts", tokens=8, top=4, experts=16, n_in=256, n_out=64, gathered=True, gated=True, dtype="e4m3", scale="e8m0", out="bf16"),
    dict(kind="experts", tokens=101, top=3, experts=7, n_in=500, n_out=127, gathered=False, gated=False, dtype="bf16", scale="none", out="bf16"),
    dict(kind="combine", tokens=5, top=4, cols=128, residual=True, dtype="bf16", dropped=0.1), dict(kind="combine", tokens=77, top=2, cols=75, residual=False, dtype="f16", dropped=0.0)]


def far(got, want):
    """Error over size."""
    if not want.numel():
        return 0.0
    return float(torch.linalg.norm(got.double() - want.double()) / torch.linalg.norm(want.double()).clamp(min=1e-300))


def look(case, seed, own):
    want = P.exact(case, seed)
    P.own = own
    try:
        got = P.run(P.prepare(case, seed))
        torch.cuda.synchronize()
    finally:
        P.own = False
    pairs = list(zip(got, want)) if isinstance(got, list) else [(got, want)]
    assert not isinstance(got, list) or len(got) == len(want)
    for i, (g, w) in enumerate(pairs):
        what, w = "%s, output %d of %s" % ("kernels" if own else "plain", i, case), w.to(g.device)
        assert g.shape == w.shape, what
        if not g.dtype.is_floating_point or g.dtype == torch.float8_e4m3fn:
            assert torch.equal(g.double(), w.double()), what
            continue
        most = U[g.dtype] + (2.0 ** -11 if case["dtype"] == "e4m3" and g.dtype != torch.float32 else 0)
        e = far(g, w)
        G.say("%s: %.3g of %.3g" % (what, e, most))
        assert e <= most, what


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d" % (c["kind"], c.get("tokens", c.get("rows"))))
def test_a_small_case(case, own):
    look(case, 11, own)


def test_cases_are_well_made():
    names = [c["name"] for c in P.listed()]
    assert len(set(names)) == len(names) and all({"bytes", "flops"} == set(P.work(c)) for c in P.listed())
    rng = random.Random(5)
    drawn = [P.draw(rng) for _ in range(100)]
    assert {c["kind"] for c in drawn} == {c["kind"] for c in P.listed()}
    most = [max(P.work(c)[k] for c in P.listed()) for k in ("bytes", "flops")]
    assert all(P.work(c)["bytes"] <= most[0] and P.work(c)["flops"] <= most[1] for c in drawn)
    # (the inputs are the seed's)
    case = P.listed()[2]
    assert torch.equal(P.prepare(case, 3)["x"], P.prepare(case, 3)["x"]) and not torch.equal(P.prepare(case, 3)["x"], P.prepare(case, 4)["x"])
