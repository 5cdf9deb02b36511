"""The cases of perf/operators.py at small sizes: the framework's calls and the plain forms against the 64-bit results, so that what is timed is known to be the operator.

Tolerances, of a tensor's error over its size (root of the sum of squares; u: half a unit in the last place of its type, relative):
  whole numbers (tables, slots, ids): equal.
  rounded once to 16 bits: u, which a rounding's own mean (u / sqrt 3 at most) and fp32's 2^-20 stay below.
  attention by the kernels, whose weights are fp16: 2^-10 more, of sum p |v|, which for values of both signs is some ten times the output's size at the longest case: 2^-7 in all.
  keys held in 4 bits: one in a thousand at most falls to the neighbouring code, a step of about half the values' size: 0.5 sqrt(0.001) = 0.016.  Held values, which get no norm: equal.
  fp32 statistics of log probabilities: 2^-18."""
import importlib.util
import os
import random

import pytest
import torch

import gpu_util as G

pytestmark = pytest.mark.gpu

_path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
_spec = importlib.util.spec_from_file_location("perf_operators", _path)
P = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(P)
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -18}

CASES = [
    dict(kind="tables", n_seq=7, cached=100, new_min=1, new_max=1, page=64), dict(kind="tables", n_seq=300, cached=90, new_min=0, new_max=8, page=32),
    dict(kind="rope", tokens=1, q_heads=4, kv_heads=4, dim=128, rot=128, interleaved=False, dtype="f16"), dict(kind="rope", tokens=37, q_heads=7, kv_heads=1, dim=256, rot=128, interleaved=True, dtype="bf16"),
    dict(kind="append", tokens=5, q_heads=4, kv_heads=2, dim=128, rot=128, interleaved=False, dtype="f16", page=64),
    dict(kind="append", tokens=203, q_heads=6, kv_heads=3, dim=64, rot=32, interleaved=True, dtype="bf16", page=32),
    dict(kind="attend", n_seq=1, q_min=1, q_max=1, kv_min=97, kv_max=97, q_heads=4, kv_heads=4, dim=128, page=64, dtype="f16"),
    dict(kind="attend", n_seq=1, q_min=1, q_max=1, kv_min=9001, kv_max=9001, q_heads=8, kv_heads=2, dim=128, page=64, dtype="f16"),
    dict(kind="attend", n_seq=9, q_min=1, q_max=9, kv_min=16, kv_max=300, q_heads=7, kv_heads=1, dim=64, page=32, dtype="bf16"),
    dict(kind="attend", n_seq=3, q_min=100, q_max=100, kv_min=100, kv_max=301, q_heads=4, kv_heads=2, dim=256, page=128, dtype="f16"),
    dict(kind="logprobs", rows=1, vocab=50257, top=20, dtype="bf16"), dict(kind="logprobs", rows=9, vocab=1001, top=5, dtype="f32"), dict(kind="logprobs", rows=700, vocab=3001, top=0, dtype="f16")]


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
        what = "%s, output %d of %s" % ("kernels" if own else "plain", i, case)
        assert g.shape == w.shape, what
        if not g.dtype.is_floating_point:
            assert torch.equal(g.long(), w.long()), what
            continue
        most = U[g.dtype]
        if case["kind"] == "attend" and own:
            most += 2.0 ** -7
        if case["kind"] == "append" and i > 0:
            most = 0.016 if i == 1 else 0.0
        e = far(g, w)
        G.say("%s: %.3g of %.3g" % (what, e, most))
        assert e <= most, what


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d" % (c["kind"], c.get("tokens", c.get("rows", c.get("n_seq")))))
def test_a_small_case(case, own):
    look(case, 11, own)


def test_cases_are_well_made():
    names = [c["name"] for c in P.listed()]
    assert len(set(names)) == len(names) and all({"bytes", "flops"} == set(P.work(c)) for c in P.listed())
    rng = random.Random(5)
    drawn = [P.draw(rng) for _ in range(200)]
    assert {c["kind"] for c in drawn} == {c["kind"] for c in P.listed()}
    most = [max(P.work(c)[k] for c in P.listed()) for k in ("bytes", "flops")]
    assert all(P.work(c)["bytes"] <= most[0] and P.work(c)["flops"] <= most[1] for c in drawn)
    # (the inputs are the seed's)
    case = P.listed()[2]
    assert torch.equal(P.prepare(case, 3)["qkv"], P.prepare(case, 3)["qkv"]) and not torch.equal(P.prepare(case, 3)["qkv"], P.prepare(case, 4)["qkv"])
