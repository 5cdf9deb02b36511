"""GPU tests of what stands between the layer products of a token pass -- block tables, norm and rotation, the cache in 4 bits and attention
over it, log probabilities -- against oracle/serve_oracle.py in 64 bits.

Tolerances (u = 2^-11 for fp16, 2^-8 for bf16: half a unit in the last place of the output, relative):
  tables, cache bytes of keys that get no norm and no rotation, values: equal.
  norm and rotation: u |y| for the rounding, and 2^-19 (|a| + |b|) for a handful of fp32 operations on the pair (a, b).
  codes behind them: a value may fall to a neighbouring code where fp32 and 64 bits lie on two sides of a boundary (a few 2^-22 of a step: less than
      1 in 1000 of the values), the scale to its neighbour likewise: s (1 + 2^-6) and 2^-6 of the value, at such places.
  attention: probabilities rounded to fp16 (2^-11 each, no subnormal ones that matter: 2^-24 of the largest), fp32 sums: 2^-10 sum p |v|, the output's
      rounding u |o|; scores in fp32: an error d of a score changes p by d: 2 d sum p |v|, d = 2^-18 sum |q k| scale.
  log probabilities: fp32 statistics: 2^-20 (1 + |x - max| + log of the number) each, entropies likewise.
An fp16 output below 2^-14 has an absolute spacing: 2^-25 more."""
import math
import random

import numpy as np
import pytest
import torch

import gpu_util as G
from oracle import serve_oracle as S
from paper_2505_11076_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"f16": (torch.float16, B.F16, 2.0 ** -11), "bf16": (torch.bfloat16, B.BF16, 2.0 ** -8), "f32": (torch.float32, B.F32, 2.0 ** -24)}


def ints(v):
    return torch.tensor(np.asarray(v, np.int64), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().cpu().double().numpy()


def ptr(t):
    return 0 if t is None else t.data_ptr()


def close(got, want, bound, what):
    with np.errstate(invalid="ignore"):
        _close(got, want, bound, what)


def _close(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound + 2.0 ** -25)
    bad &= ~(np.isnan(got) & np.isnan(want)) & ~(np.isinf(want) & (got == want))
    G.say("%s: %d values, worst %.3g of its bound" % (what, got.size, np.nanmax(np.abs(got - want) / (bound + 2.0 ** -25), initial=0)))
    assert not bad.any(), (what, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


# ---- block tables ------------------------------------------------------------------------------------------


def run_tables(cached, new, page, free, table, max_tokens):
    n, guard = len(cached), 16
    dev = [ints(cached), ints(new), ints(free) if len(free) else None, ints(table)]
    out = [torch.full((m + guard,), 777, dtype=torch.int32, device="cuda") for m in (n + 1, n, max_tokens, max_tokens, 2)]
    B.dbf_block_tables(ptr(dev[0]), ptr(dev[1]), n, page, ptr(dev[2]), len(free), ptr(dev[3]), dev[3].shape[1], max_tokens, *[ptr(o) for o in out], G.stream_handle())
    torch.cuda.synchronize()
    for o in out:
        assert (o[-guard:] == 777).all()
    return [dev[3].cpu().numpy()] + [o[:-guard].cpu().tolist() for o in out]


@pytest.mark.parametrize("n,page,new_range,short,slack,wide", [
    (1, 64, (1, 1), 0, 0, 2), (1, 32, (0, 0), 0, 5, 2), (5, 32, (0, 3), 0, 1, 1), (64, 128, (1, 1), 0, 0, 1), (63, 256, (0, 700), 0, 40, 1), (300, 64, (0, 1), 2, 3, 1),
    (1000, 32, (0, 70), 0, 0, 1), (1000, 32, (0, 70), 37, 9, 0), (4097, 64, (0, 9), 5, 11, 1), (3, 32, (4000, 6000), 0, 0, 1), (70000, 32, (0, 1), 3, 1, 1), (3, 32, (40, 99), 999, 0, 1)])
def test_block_tables(n, page, new_range, short, slack, wide):
    rng = random.Random(n * 1000 + page)
    cached = [rng.choice([0, page - 1, page, page + 1, rng.randint(0, 5 * page)]) for _ in range(n)]
    new = [rng.randint(*new_range) for _ in range(n)]
    if n > 4:
        cached[2], new[3] = -5, -1   # (count as 0)
    c0, n0 = [max(c, 0) for c in cached], [max(v, 0) for v in new]
    need = sum(-(-(c + v) // page) - -(-c // page) for c, v in zip(c0, n0))
    # (wide 0: a table that has no place for some requests' last pages)
    stride = max(1, max(-(-(c + v) // page) for c, v in zip(c0, n0)) + (wide if wide else -1))
    ids = rng.sample(range(10 * (need + n * stride) + 10), need + n * stride)
    table = np.array(ids[need:]).reshape(n, stride)
    free = ids[: max(0, need - short)]
    tokens = sum(n0) + slack
    got = run_tables(cached, new, page, free, table, tokens)
    want = S.block_tables(cached, new, page, free, table, tokens)
    assert np.array_equal(got[0], want[0])
    assert got[1:] == [list(map(int, w)) for w in want[1:]]


def test_block_tables_more_tokens_than_there_is_room_for():
    got = run_tables([10, 0, 31], [50, 2000, 40], 32, list(range(100)), np.full((3, 70), -1), 700)
    want = S.block_tables([10, 0, 31], [50, 2000, 40], 32, list(range(100)), np.full((3, 70), -1), 3000)
    # (pages of tokens that have no room are counted; their entries are not made)
    assert got[1:3] == list(want[1:3]) and got[3] == want[3][:700] and got[4] == want[4][:700] and got[5] == want[5]


# ---- norm and rotation -------------------------------------------------------------------------------------


def rope_table(n, rot):
    a = np.arange(n)[:, None] * np.exp(-np.arange(0, rot, 2) * math.log(10000.0) / rot)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def make_heads(g, T, hq, hk, D, dtype, pad=0, offset=0, large=1.0):
    """q, k, v as views of one buffer with `pad` values between rows and `offset` values in front."""
    row = (hq + 2 * hk) * D + pad
    buf = torch.randn(T * row + offset + 8, generator=g, device="cuda").mul_(large).to(DT[dtype][0])
    rows = buf[offset: offset + T * row].view(T, row)
    return buf, row, [rows[:, a * D: b * D].unflatten(1, (-1, D)) for a, b in ((0, hq), (hq, hq + hk), (hq + hk, hq + 2 * hk))]


ROPE = [  # tokens, q heads, kv heads, head size, rotated, interleaved, type, norm, pad, offset
    (1, 32, 32, 128, 128, False, "f16", True, 0, 0), (1, 1, 1, 64, 64, True, "bf16", True, 0, 0), (7, 3, 1, 128, 64, True, "bf16", True, 8, 0), (5, 4, 2, 96, 96, False, "f16", True, 0, 8),
    (33, 8, 1, 256, 256, False, "f16", False, 0, 0), (3, 2, 2, 80, 40, False, "bf16", True, 1, 3), (2, 5, 1, 2, 2, True, "f16", True, 0, 1), (4, 1, 1, 1024, 1024, False, "f16", True, 0, 0),
    (9, 2, 1, 64, 0, False, "f16", True, 0, 0), (130, 7, 1, 128, 128, True, "f16", True, 0, 0), (257, 2, 2, 64, 32, False, "bf16", True, 16, 0), (6, 2, 1, 130, 26, True, "f16", False, 5, 5),
    (64, 3, 3, 128, 16, False, "bf16", True, 0, 0), (11, 2, 2, 192, 192, True, "bf16", True, 0, 0), (12, 2, 2, 256, 64, False, "f16", True, 8, 16), (70000, 1, 1, 64, 64, False, "f16", True, 0, 0)]


@pytest.mark.parametrize("T,hq,hk,D,rot,inter,dtype,norm,pad,offset", ROPE)
@pytest.mark.parametrize("in_place", [False, True])
def test_qk_norm_rope(T, hq, hk, D, rot, inter, dtype, norm, pad, offset, in_place):
    g = torch.Generator(device="cuda").manual_seed(T * 7 + D)
    dt, code, u = DT[dtype]
    buf, row, (q, k, v) = make_heads(g, T, hq, hk, D, dtype, pad, offset)
    before = buf.clone()
    w = [(1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt) if norm else None for _ in range(2)]
    table = rope_table(500, rot) if rot else None
    pos = torch.randint(0, 500, (T,), generator=g, device="cuda", dtype=torch.int32)
    dev = torch.from_numpy(table).cuda() if rot else None
    want = []
    for x, weight in zip((q, k), w):
        cos, sin = (table[f64(pos).astype(int)][:, i * rot // 2:][:, : rot // 2].astype(np.float64) for i in (0, 1)) if rot else (None, None)
        args = (None if weight is None else f64(weight), 1e-5, cos, sin, inter)
        want.append((S.norm_rope(f64(x), *args), S.norm_rope(np.abs(f64(x)), args[0] if args[0] is None else np.abs(args[0]), 1e-5,
                                                             None if cos is None else np.abs(cos), None if sin is None else -np.abs(sin), inter)))
    outs = (q, k) if in_place else [torch.full((T, h * D + 24), 7.0, dtype=dt, device="cuda") for h in (hq, hk)]
    strides = (row, row) if in_place else (hq * D + 24, hk * D + 24)
    h = B.Heads(q=ptr(q), q_stride=row, k=ptr(k), k_stride=row, q_out=ptr(outs[0]), q_out_stride=strides[0], k_out=ptr(outs[1]), k_out_stride=strides[1], dtype=code, n_tokens=T,
                n_q_heads=hq, n_kv_heads=hk, head_dim=D, q_weight=ptr(w[0]), k_weight=ptr(w[1]), eps=1e-5, rope=ptr(dev), rope_len=500 if rot else 0, rot_dim=rot,
                interleaved=int(inter), positions=ptr(pos))
    B.dbf_qk_norm_rope(h, G.stream_handle())
    torch.cuda.synchronize()
    for o, n, (y, size), what in zip(outs, (hq, hk), want, "qk"):
        got = f64(o) if in_place else f64(o[:, : n * D]).reshape(T, n, D)
        # (`size`: the pair's parts in absolute value, |a| |cos| + |b| |sin|, at the first of a pair; the sum bounds both)
        pair = size.copy()
        if rot:
            pair = np.abs(y) + size.max(-1, keepdims=True)
        close(got, y, u * np.abs(y) + 2.0 ** -19 * (np.abs(pair) + np.abs(y)), "%s of %s" % (what, (T, hq, hk, D, rot, inter, dtype)))
        if not in_place:
            assert (o[:, n * D:] == 7).all()
    if in_place:   # nothing else of the buffer
        rows, old = (b[offset: offset + T * row].view(T, row)[:, (hq + hk) * D:] for b in (buf, before))
        assert torch.equal(rows, old) and torch.equal(buf[:offset], before[:offset]) and torch.equal(buf[offset + T * row:], before[offset + T * row:])
    else:
        assert torch.equal(buf, before)


def test_one_of_the_two_and_positions_outside_the_table():
    g = torch.Generator(device="cuda").manual_seed(3)
    buf, row, (q, k, v) = make_heads(g, 4, 2, 1, 64, "f16")
    dev = torch.from_numpy(rope_table(10, 32)).cuda()
    pos = ints([0, -1, 9, 10])
    out = torch.full((4, 64), 7.0, dtype=torch.float16, device="cuda")
    B.dbf_qk_norm_rope(B.Heads(k=ptr(k), k_stride=row, k_out=ptr(out), k_out_stride=64, dtype=B.F16, n_tokens=4, n_kv_heads=1, head_dim=64, rope=ptr(dev), rope_len=10, rot_dim=32,
                               positions=ptr(pos)), G.stream_handle())
    torch.cuda.synchronize()
    assert torch.equal(out[0], k[0, 0]) and torch.isfinite(out[2]).all()
    assert torch.isnan(out[[1, 3], :32]).all() and torch.equal(out[[1, 3], 32:], k[[1, 3], 0, 32:])


def test_zero_rows_and_infinities():
    g = torch.Generator(device="cuda").manual_seed(5)
    buf, row, (q, k, v) = make_heads(g, 3, 1, 1, 128, "f16")
    q[0] = 0
    q[1, 0, 3] = float("inf")
    w = torch.ones(128, dtype=torch.float16, device="cuda")
    out = torch.full((3, 128), 7.0, dtype=torch.float16, device="cuda")
    B.dbf_qk_norm_rope(B.Heads(q=ptr(q), q_stride=row, q_out=ptr(out), q_out_stride=128, dtype=B.F16, n_tokens=3, n_q_heads=1, head_dim=128, q_weight=ptr(w), eps=1e-6),
                       G.stream_handle())
    torch.cuda.synchronize()
    assert (out[0] == 0).all() and torch.isnan(out[1, 3]) and torch.isfinite(out[2]).all()


# ---- the cache ---------------------------------------------------------------------------------------------


CACHE = [  # tokens, q heads, kv heads, head size, page, type, pad, offset
    (1, 1, 1, 64, 32, "f16", 0, 0), (5, 4, 2, 128, 64, "bf16", 0, 0), (40, 2, 1, 256, 128, "f16", 8, 0), (33, 3, 3, 128, 256, "f16", 1, 3), (70, 2, 2, 64, 32, "bf16", 0, 1), (64, 8, 4, 128, 32, "f16", 0, 8)]


def slots_of(rng, T, pages, page):
    return rng.permutation(pages * page)[:T]


@pytest.mark.parametrize("T,hq,hk,D,page,dtype,pad,offset", CACHE)
def test_cache_append_without_norm_is_exact(T, hq, hk, D, page, dtype, pad, offset):
    g = torch.Generator(device="cuda").manual_seed(T + D)
    rng = np.random.default_rng(T + D)
    buf, row, (q, k, v) = make_heads(g, T, hq, hk, D, dtype, pad, offset)
    pages = -(-T // page) + 1
    slots = slots_of(rng, T, pages, page)
    # awkward heads: nothing but zeros, one sign, one value, beyond the range, no numbers, tiny
    for i, x in enumerate([0.0, 1.0, -2.5, 60000.0, 3e-8]):
        if i < T:
            k[i, 0] = x
            v[T - 1 - i, hk - 1] = x
    if T > 8:
        k[6, 0] = k[6, 0].abs()
        v[7, 0] = -v[7, 0].abs()
        k[8, 0, 5] = float("nan")
        v[9, hk - 1, 63] = float("-inf")
    if T > 20:
        slots[11], slots[12] = -1, pages * page
    ref = S.Cache(pages, page, hk, D, fill=0x5A)
    dev = torch.full((ref.data.size + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    kk, vv = f64(k), f64(v)
    for t, s in enumerate(slots):
        for h in range(hk):
            if 0 <= s < pages * page:
                ref.write(int(s), h, kk[t, h], vv[t, h])
    qo = torch.full((T, hq * D), 7.0, dtype=DT[dtype][0], device="cuda")
    cache = B.Cache(data=ptr(dev), n_pages=pages, page_tokens=page, n_kv_heads=hk, head_dim=D)
    heads = B.Heads(q=ptr(q), q_stride=row, k=ptr(k), k_stride=row, v=ptr(v), v_stride=row, q_out=ptr(qo), q_out_stride=hq * D, dtype=DT[dtype][1], n_tokens=T, n_q_heads=hq,
                    n_kv_heads=hk, head_dim=D)
    sl = ints(slots)
    B.dbf_cache_append(heads, cache, ptr(sl), G.stream_handle())
    torch.cuda.synchronize()
    assert torch.equal(qo.view(T, hq, D), q)
    got = dev.cpu().numpy()
    assert (got[ref.data.size:] == 0x5A).all()
    # bytes are equal; words too (as numbers: there is more than one that is none)
    codes = lambda d: d.reshape(-1, 36 * D)[:, : 32 * D]   # noqa: E731
    words = lambda d: np.ascontiguousarray(d.reshape(-1, 36 * D)[:, 32 * D:]).view(np.float16)   # noqa: E731
    assert np.array_equal(words(got[: ref.data.size]), words(ref.data), equal_nan=True)
    assert np.array_equal(codes(got[: ref.data.size]), codes(ref.data))
    # and read back
    for name in ("f16", "bf16", "f32"):
        ko, vo = (torch.full((T + 1, hk, D), 7.0, dtype=DT[name][0], device="cuda") for _ in range(2))
        B.dbf_cache_read(cache, ptr(sl), T, ptr(ko), ptr(vo), DT[name][1], G.stream_handle())
        torch.cuda.synchronize()
        assert (ko[T] == 7).all() and (vo[T] == 7).all()
        for t, s in enumerate(slots):
            for h in range(hk):
                a, b = ref.read(int(s), h) if 0 <= s < pages * page else (np.zeros(D), np.zeros(D))
                for x, o in ((a, ko), (b, vo)):
                    x = torch.from_numpy(x).to(DT[name][0]).double().numpy()
                    assert np.array_equal(f64(o[t, h]), x, equal_nan=True)


@pytest.mark.parametrize("hq,hk,D,page,dtype", [(3, 3, 128, 32, "f16"), (0, 5, 64, 64, "bf16"), (2, 3, 256, 32, "f16"), (9, 1, 64, 32, "f16"), (0, 8, 128, 64, "bf16")])
@pytest.mark.parametrize("shift", [0, 1, 2, 3])
def test_cache_append_of_rows_of_slots(shift, hq, hk, D, page, dtype):
    """Tokens whose slots follow each other, from any place of a word's four on, over the ends of pages, broken off by others, and backwards; and what lies
    beside them stays."""
    g = torch.Generator(device="cuda").manual_seed(shift + D)
    pages = 8
    rows = [range(shift, shift + 9), range(page - 2 + shift, page + 7), range(2 * page + 5, 2 * page + 5 + shift), [-1, 3 * page + shift], range(4 * page + 12 + shift, 4 * page + 8, -1),
            range(6 * page - 4, 6 * page + 13 + shift), [pages * page - 1, pages * page, pages * page + 1], range(7 * page + shift, 7 * page + shift + 4)]
    slots = [s for r in rows for s in r]
    T = len(slots)
    buf, row, (q, k, v) = make_heads(g, T, max(hq, 1), hk, D, dtype)
    k[3, 0], v[5, hk - 1, 2] = 0.0, float("nan")
    ref = S.Cache(pages, page, hk, D, fill=0x5A)
    dev = torch.full((ref.data.size + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    kk, vv = f64(k), f64(v)
    for t, s in enumerate(slots):
        for h in range(hk):
            if 0 <= s < pages * page:
                ref.write(s, h, kk[t, h], vv[t, h])
    qo = torch.full((T, max(hq, 1) * D), 7.0, dtype=DT[dtype][0], device="cuda")
    cache = B.Cache(data=ptr(dev), n_pages=pages, page_tokens=page, n_kv_heads=hk, head_dim=D)
    heads = B.Heads(q=ptr(q) if hq else 0, q_stride=row, k=ptr(k), k_stride=row, v=ptr(v), v_stride=row, q_out=ptr(qo), q_out_stride=max(hq, 1) * D, dtype=DT[dtype][1], n_tokens=T,
                    n_q_heads=hq, n_kv_heads=hk, head_dim=D)
    sl = ints(slots)
    B.dbf_cache_append(heads, cache, ptr(sl), G.stream_handle())
    torch.cuda.synchronize()
    assert torch.equal(qo.view(T, -1, D), q) if hq else (qo == 7).all()
    got = dev.cpu().numpy()
    assert (got[ref.data.size:] == 0x5A).all()
    codes = lambda d: d.reshape(-1, 36 * D)[:, : 32 * D]   # noqa: E731
    words = lambda d: np.ascontiguousarray(d.reshape(-1, 36 * D)[:, 32 * D:]).view(np.float16)   # noqa: E731
    assert np.array_equal(words(got[: ref.data.size]), words(ref.data), equal_nan=True)
    assert np.array_equal(codes(got[: ref.data.size]), codes(ref.data))


@pytest.mark.parametrize("T,hq,hk,D,page,rot,inter,dtype", [(1, 4, 4, 128, 64, 128, False, "f16"), (300, 4, 2, 128, 64, 64, True, "bf16"), (77, 0, 2, 64, 32, 64, False, "f16"),
                                                            (90, 3, 1, 256, 128, 256, True, "f16"), (50, 2, 1, 64, 32, 16, False, "bf16")])
def test_cache_append_with_norm_and_rotation(T, hq, hk, D, page, rot, inter, dtype):
    g = torch.Generator(device="cuda").manual_seed(T + D + 1)
    dt, code, u = DT[dtype]
    buf, row, (q, k, v) = make_heads(g, T, max(hq, 1), hk, D, dtype)
    pages = -(-T // page) + 1
    slots = slots_of(np.random.default_rng(1), T, pages, page)
    w = [(1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dt) for _ in range(2)]
    table, pos = rope_table(400, rot), torch.randint(0, 400, (T,), generator=g, device="cuda", dtype=torch.int32)
    dev = torch.from_numpy(table).cuda()
    data = torch.zeros(S.cache_bytes(pages, page, hk, D), dtype=torch.uint8, device="cuda")
    qo, sl = torch.full((T, max(hq, 1) * D), 7.0, dtype=dt, device="cuda"), ints(slots)
    cache = B.Cache(data=ptr(data), n_pages=pages, page_tokens=page, n_kv_heads=hk, head_dim=D)
    heads = B.Heads(q=ptr(q) if hq else 0, q_stride=row, k=ptr(k), k_stride=row, v=ptr(v), v_stride=row, q_out=ptr(qo), q_out_stride=max(hq, 1) * D, dtype=code, n_tokens=T,
                    n_q_heads=hq, n_kv_heads=hk, head_dim=D, q_weight=ptr(w[0]), k_weight=ptr(w[1]), eps=1e-6, rope=ptr(dev), rope_len=400, rot_dim=rot, interleaved=int(inter),
                    positions=ptr(pos))
    B.dbf_cache_append(heads, cache, ptr(sl), G.stream_handle())
    ko, vo = (torch.empty((T, hk, D), dtype=torch.float32, device="cuda") for _ in range(2))
    B.dbf_cache_read(cache, ptr(sl), T, ptr(ko), ptr(vo), B.F32, G.stream_handle())
    torch.cuda.synchronize()
    rows = table[f64(pos).astype(int)].astype(np.float64)
    cos, sin = rows[:, : rot // 2], rows[:, rot // 2:]
    y = S.norm_rope(f64(k), f64(w[1]), 1e-6, cos, sin, inter)
    want, got = S.held(y), f64(ko)
    assert np.array_equal(f64(vo), S.held(f64(v)))
    step = np.zeros_like(y)
    for t in range(T):
        for h in range(hk):
            s = S.quantise(y[t, h])[1]
            step[t, h] = [s[S.group_of(d, D)] for d in range(D)]
    off = np.abs(got - want)
    G.say("codes of %d keys: %d of other values" % (y.size, (off > 0).sum()))
    assert (off <= step * (1 + 2.0 ** -6) + 2.0 ** -6 * np.abs(want)).all() and (off > 0).mean() <= 1e-3 + 64 / y.size
    if hq:
        z = S.norm_rope(f64(q), f64(w[0]), 1e-6, cos, sin, inter)
        close(f64(qo).reshape(T, hq, D), z, u * np.abs(z) + 2.0 ** -18 * np.abs(z).max(-1, keepdims=True), "q")
    else:
        assert (qo == 7).all()


# ---- attention ---------------------------------------------------------------------------------------------


def make_cache(rng, kv, page, hk, D, extra=2, scale=(1.0, 1.0), poison=True):
    """A cache of random keys and values for requests of kv tokens, its block table, and the values held.  Where no token is held the bytes are 0xFF
    (codes 15, words that are no numbers) if poison."""
    each = [-(-n // page) for n in kv]
    pages = sum(each) + extra
    order = rng.permutation(pages)
    table = np.full((len(kv), max(each + [1]) + 1), -1)
    for i, n in enumerate(each):
        table[i, :n] = order[sum(each[:i]): sum(each[:i]) + n]
    n = D // 64
    codes = rng.integers(0, 16, (2, pages, hk, page, D))
    s = 2.0 ** -3 * rng.integers(64, 128, (2, pages, hk, page, n)) / 64 * np.array(scale).reshape(2, 1, 1, 1, 1)
    z = rng.integers(0, 16, (2, pages, hk, page, n))
    groups = [(d // 16) % n for d in range(D)]
    values = s[..., groups] * (codes - z[..., groups])
    assert np.array_equal(values.astype(np.float16).astype(np.float64), values)
    # the bytes, from the layout's description
    k4 = codes[0].reshape(pages, hk, page // 32, 32, D // 2, 2)
    kb = (k4[..., 0] | k4[..., 1] << 4).reshape(pages, hk, page // 32, -1)
    vb = np.zeros((pages, hk, page // 32, 16 * D), np.int64)
    ref = S.Cache(1, 32, 1, D)
    for t in range(32):
        for d, (_, _, at, half) in enumerate(ref.places(t)):
            vb[..., at - 16 * D] |= codes[1].reshape(pages, hk, page // 32, 32, D)[..., t, d] << 4 * half
    held = np.zeros((pages, page), bool)
    for i, m in enumerate(kv):
        for r in range(each[i]):
            held[table[i, r], : max(0, min(page, m - r * page))] = True
    words = []
    for x in range(2):
        w = np.stack([s[x], -s[x] * z[x]], -1).astype(np.float16)                       # pages, hk, page, n, 2
        if poison:
            w[~np.broadcast_to(held[:, None], w.shape[:3])] = np.float16(np.nan)
        words.append(np.ascontiguousarray(w.reshape(pages, hk, page // 32, 32, n, 2).transpose(0, 1, 2, 4, 3, 5)).view(np.uint8).reshape(pages, hk, page // 32, -1))
    data = np.concatenate([kb.astype(np.uint8), vb.astype(np.uint8)] + words, -1)
    assert data.size == S.cache_bytes(pages, page, hk, D)
    k, v = ([np.concatenate([values[x][table[i, r]].transpose(1, 0, 2) for r in range(each[i])] or [np.zeros((0, hk, D))])[: kv[i]] for i in range(len(kv))] for x in range(2))
    return torch.from_numpy(data.reshape(-1)).cuda(), pages, table, k, v


def run_attend(data, pages, table, kv, q_len, q, page, hk, D, dtype, scale, causal, max_q=None, max_kv=None, starts=True, out=None, pad=0, stream=None, n_tokens=None):
    T, hq = q.shape[:2]
    if out is None:
        out = torch.full((T + 1, hq * D + pad), 7.0, dtype=q.dtype, device="cuda")
    kvd, st, tab = ints(kv), ints(np.cumsum([0] + list(q_len))), ints(table)
    cache = B.Cache(data=ptr(data), n_pages=pages, page_tokens=page, n_kv_heads=hk, head_dim=D)
    a = B.Attend(q=ptr(q), q_stride=q.stride(0), out=ptr(out), out_stride=out.stride(0), dtype=DT[dtype][1], n_tokens=T if n_tokens is None else n_tokens, n_seq=len(kv),
                 n_q_heads=hq, max_q=max(q_len) if max_q is None else max_q, max_kv=max(kv) if max_kv is None else max_kv, q_start=ptr(st) if starts else 0, kv_len=ptr(kvd),
                 block_table=ptr(tab), table_stride=tab.shape[1], scale=scale, causal=int(causal))
    n = B.dbf_cache_attend_workspace_bytes(a, cache)
    ws = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    B.dbf_cache_attend(a, cache, ptr(ws), n, G.stream_handle() if stream is None else stream)
    torch.cuda.synchronize()
    assert (ws[n:] == 0xA5).all()
    return out


def check_attend(out, q, k, v, q_len, D, dtype, scale, causal, what):
    u, at = DT[dtype][2], 0
    T, hq = q.shape[:2]
    got, qq = f64(out[:T, : hq * D]).reshape(T, hq, D), f64(q)
    for i, n in enumerate(q_len):
        o, w, size = S.attend(qq[at: at + n], k[i], v[i], scale, causal)
        close(got[at: at + n], o, 2.0 ** -10 * w + u * np.abs(o) + 2 * 2.0 ** -18 * size[..., None] * w, "%s, request %d" % (what, i))
        at += n
    assert (out[T:] == 7).all() and (out[:, hq * D:] == 7).all()


ATTEND = [  # kv lengths, rows, q heads, kv heads, head size, page, type, causal
    ([1], [1], 1, 1, 64, 32, "f16", 1), ([333], [1], 4, 4, 128, 64, "f16", 1), ([31, 32, 33, 0, 64, 65, 1], [1] * 7, 8, 2, 128, 32, "bf16", 1),
    ([2000, 5, 700], [1, 1, 1], 16, 1, 128, 128, "f16", 1), ([1500, 130], [1, 1], 7, 1, 64, 256, "bf16", 1), ([900, 257], [1, 1], 4, 2, 256, 64, "f16", 1),
    ([50, 3, 0, 9], [4, 3, 2, 0], 4, 2, 128, 32, "f16", 1), ([600, 40], [5, 9], 8, 4, 64, 64, "bf16", 1), ([5000], [3], 8, 2, 128, 64, "f16", 1), ([100, 2], [2, 5], 2, 2, 128, 32, "f16", 1),
    ([300, 33, 64], [40, 33, 1], 8, 2, 128, 64, "f16", 1), ([129, 257], [129, 200], 2, 2, 64, 32, "bf16", 1), ([400, 31], [100, 31], 6, 2, 256, 128, "f16", 1),
    ([700], [17], 4, 4, 128, 64, "f16", 0), ([90, 5], [3, 8], 4, 2, 128, 32, "bf16", 0), ([70, 200], [70, 150], 3, 3, 128, 64, "f16", 0), ([20, 500], [64, 0], 2, 1, 64, 32, "f16", 1),
    ([3000], [130], 32, 8, 128, 64, "bf16", 1), ([17, 300], [1, 1], 40, 2, 128, 32, "f16", 1), ([260], [260], 1, 1, 128, 256, "f16", 1), ([100], [33], 5, 5, 256, 32, "bf16", 0)]


@pytest.mark.parametrize("kv,q_len,hq,hk,D,page,dtype,causal", ATTEND)
def test_cache_attend(kv, q_len, hq, hk, D, page, dtype, causal):
    rng = np.random.default_rng(sum(kv) + D + hq)
    data, pages, table, k, v = make_cache(rng, kv, page, hk, D)
    q = torch.from_numpy(rng.normal(size=(sum(q_len), hq, D))).cuda().to(DT[dtype][0])
    out = run_attend(data, pages, table, kv, q_len, q, page, hk, D, dtype, 1 / math.sqrt(D), causal)
    check_attend(out, q, k, v, q_len, D, dtype, 1 / math.sqrt(D), causal, "attend")


SHARED = [  # requests of which some are long and the items few: they are shared out among workgroups, cut anywhere
    ([5000, 0, 33, 1, 9000, 64], [1] * 6, 4, 2, 64, 32, "f16", 1), ([4200, 3, 2600], [2, 1, 4], 4, 2, 256, 128, "bf16", 1), ([20011], [1], 16, 1, 128, 64, "f16", 1),
    ([0, 0, 6000], [1, 1, 1], 7, 1, 128, 256, "bf16", 1), ([3000, 2999, 2, 7000], [3, 5, 5, 0], 4, 2, 128, 32, "f16", 0), ([70, 9, 2500, 0, 31] * 9, [1] * 45, 2, 1, 64, 32, "f16", 1),
    ([12000, 2], [4, 8], 2, 1, 128, 64, "f16", 1), ([2400] * 3, [1] * 3, 8, 8, 256, 64, "f16", 1)]


@pytest.mark.parametrize("kv,q_len,hq,hk,D,page,dtype,causal", SHARED)
def test_cache_attend_shared_out(kv, q_len, hq, hk, D, page, dtype, causal):
    assert max(kv) > 2048 + 8 * len(kv) * hk and max(q_len) * (hq // hk) <= 16
    test_cache_attend(kv, q_len, hq, hk, D, page, dtype, causal)


@pytest.mark.parametrize("kv,q_len,more", [([40, 300], [1, 1], 5000), ([40, 300], [30, 7], 3000), ([200], [200], 100)])
def test_cache_attend_with_larger_bounds_than_lengths(kv, q_len, more):
    """max_q and max_kv choose the launch (parts, rows of a workgroup): what is beyond the lengths adds nothing."""
    rng = np.random.default_rng(7)
    data, pages, table, k, v = make_cache(rng, kv, 64, 2, 128)
    table = np.concatenate([table, np.full((len(kv), 100), -1)], 1)
    q = torch.from_numpy(rng.normal(size=(sum(q_len), 8, 128))).cuda().half()
    out = run_attend(data, pages, table, kv, q_len, q, 64, 2, 128, "f16", 0.1, 1, max_q=max(q_len) + 40, max_kv=max(kv) + more)
    check_attend(out, q, k, v, q_len, 128, "f16", 0.1, 1, "larger bounds")


@pytest.mark.parametrize("scale", [(1.0, 1.0), (2.0 ** -15, 2.0 ** -15), (2.0 ** 11, 2.0 ** 11), (1.0, 2.0 ** -15), (2.0 ** -6, 2.0 ** 11)])
@pytest.mark.parametrize("kv,q_len", [([700, 40], [1, 1]), ([700, 40], [70, 40])])
def test_cache_attend_sizes_of_values(scale, kv, q_len):
    """Keys and values from fp16's smallest to its largest, queries and scales that make up for it: also scores that leave one token."""
    rng = np.random.default_rng(11)
    data, pages, table, k, v = make_cache(rng, kv, 32, 2, 128, scale=scale)
    q = torch.from_numpy(rng.normal(size=(sum(q_len), 4, 128)) * min(3.0, 0.5 / scale[0])).cuda().half()
    out = run_attend(data, pages, table, kv, q_len, q, 32, 2, 128, "f16", 1.0, 1)
    check_attend(out, q, k, v, q_len, 128, "f16", 1.0, 1, "values of %g" % scale[1])


@pytest.mark.parametrize("dtype,size", [("f16", 6e4), ("f16", 1e-7), ("bf16", 1e30), ("bf16", 1e-30)])
@pytest.mark.parametrize("q_len", [[1, 1], [60, 2]])
def test_cache_attend_sizes_of_queries(dtype, size, q_len):
    rng = np.random.default_rng(12)
    kv = [500, 70]
    data, pages, table, k, v = make_cache(rng, kv, 32, 2, 64)
    q = (torch.from_numpy(rng.normal(size=(sum(q_len), 2, 64))).clamp(-1, 1) * size).cuda().to(DT[dtype][0])
    q[0, 0] = 0
    out = run_attend(data, pages, table, kv, q_len, q, 32, 2, 64, dtype, 0.3 / size, 1)
    check_attend(out, q, k, v, q_len, 64, dtype, float(np.float32(0.3 / size)), 1, "queries of %g" % size)


@pytest.mark.parametrize("scale", [0.0, -0.2])
@pytest.mark.parametrize("q_len", [[1, 1], [60, 30]])
def test_cache_attend_other_scales(scale, q_len):
    rng = np.random.default_rng(19)
    kv = [500, 30]
    data, pages, table, k, v = make_cache(rng, kv, 32, 2, 64)
    q = torch.from_numpy(rng.normal(size=(sum(q_len), 4, 64))).cuda().half()
    out = run_attend(data, pages, table, kv, q_len, q, 32, 2, 64, "f16", scale, 1)
    check_attend(out, q, k, v, q_len, 64, "f16", float(np.float32(scale)), 1, "scale %g" % scale)


def test_cache_attend_lone_peak_and_equal_scores():
    """One token with all the weight, at each place of a record; and keys that are all alike (the mean of the values)."""
    rng = np.random.default_rng(13)
    kv = [97]
    data, pages, table, k, v = make_cache(rng, kv, 32, 1, 64, poison=False)
    for at in (0, 1, 15, 16, 31, 32, 63, 95, 96):
        q = torch.from_numpy(8.0 * k[0][at: at + 1] / np.abs(k[0][at]).max()).cuda().half().reshape(1, 1, 64)
        out = run_attend(data, pages, table, kv, [1], q, 32, 1, 64, "f16", 4.0, 1)
        check_attend(out, q, k, v, [1], 64, "f16", 4.0, 1, "a peak at %d" % at)
    q = torch.zeros((1, 1, 64), dtype=torch.float16, device="cuda")
    out = run_attend(data, pages, table, kv, [1], q, 32, 1, 64, "f16", 1.0, 1)
    close(f64(out[:1]), v[0].mean(0), 2.0 ** -10 * np.abs(v[0]).mean(0) + 2.0 ** -11, "equal scores")


@pytest.mark.parametrize("rows", [6, 80])
def test_tokens_that_are_no_numbers(rows):
    """A token held as no number makes the rows that see it no numbers, in its head only."""
    rng = np.random.default_rng(14)
    kv, D, hk = [100], 64, 2
    data, pages, table, k, v = make_cache(rng, kv, 32, hk, D)
    q = torch.from_numpy(rng.normal(size=(rows, 4, D))).cuda().half()
    want = run_attend(data, pages, table, kv, [rows], q, 32, hk, D, "f16", 0.1, 1)
    bad = 100 - rows + 3                                     # row 3 is the first to see it
    slot = int(table[0, bad // 32]) * 32 + bad % 32
    kk = torch.zeros((1, hk, D), dtype=torch.float16, device="cuda")
    vv = kk.clone()
    kk[:], vv[:] = torch.from_numpy(k[0][bad]).half(), torch.from_numpy(v[0][bad]).half()
    vv[0, 1, 9] = float("nan")
    cache = B.Cache(data=ptr(data), n_pages=pages, page_tokens=32, n_kv_heads=hk, head_dim=D)
    sl = ints([slot])
    B.dbf_cache_append(B.Heads(k=ptr(kk), k_stride=hk * D, v=ptr(vv), v_stride=hk * D, dtype=B.F16, n_tokens=1, n_kv_heads=hk, head_dim=D), cache, ptr(sl), G.stream_handle())
    got = run_attend(data, pages, table, kv, [rows], q, 32, hk, D, "f16", 0.1, 1)
    g, w = (f64(x[:rows]).reshape(rows, 4, D) for x in (got, want))
    assert np.isnan(g[3:, 2:]).all() and np.isfinite(g[:3]).all() and np.isfinite(g[:, :2]).all()
    assert np.array_equal(g[:3, 2:], w[:3, 2:])


@pytest.mark.parametrize("rows", [1, 40])
def test_requests_that_are_not_what_the_call_says(rows):
    """Lengths beyond max_kv, the table or max_q, negative ones, pages that the cache does not have: no numbers, in that request's rows only."""
    rng = np.random.default_rng(15)
    kv, D = [90, 90, 90, 90, 90], 64
    data, pages, table, k, v = make_cache(rng, kv, 32, 1, D)
    q = torch.from_numpy(rng.normal(size=(5 * rows, 2, D))).cuda().half()
    q_len = [rows] * 5
    lie = [91, -1, 90, 97, 90]
    table[2, 1], table[4, 2] = pages, -7
    table[3, 3:] = 0
    out = run_attend(data, pages, table, lie, q_len, q, 32, 1, D, "f16", 0.1, 1, max_kv=90)
    got = f64(out[: 5 * rows]).reshape(5, rows, 2, D)
    assert np.isnan(got[[0, 1, 3]]).all()
    last = 90 - rows + np.arange(rows)                        # the last token that a row sees
    assert (np.isnan(got[2]).all((-1, -2)) == (last >= 32)).all() and (np.isnan(got[4]).all((-1, -2)) == (last >= 64)).all()
    assert (np.isnan(got[2]).any((-1, -2)) == (last >= 32)).all() and (np.isnan(got[4]).any((-1, -2)) == (last >= 64)).all()
    if rows > 1:   # more rows than max_q: those below it are no numbers, the others are not written
        out = run_attend(data, pages, table, [90] * 5, [rows, 4, 4, 4, 4], q[: rows + 16], 32, 1, D, "f16", 0.1, 1, max_q=4)
        got = f64(out[: rows + 16])
        assert np.isnan(got[:4]).all() and (got[4:rows] == 7).all()
        assert np.isfinite(got[rows: rows + 4]).all()


def test_row_starts_that_are_out_of_range_stay_inside_the_tensor():
    rng = np.random.default_rng(16)
    data, pages, table, k, v = make_cache(rng, [90, 90], 32, 1, 64)
    q = torch.from_numpy(rng.normal(size=(6, 2, 64))).cuda().half()
    out = run_attend(data, pages, table, [90, 90], [3, 3], q, 32, 1, 64, "f16", 0.1, 1, n_tokens=4, max_q=3)
    assert (out[4:] == 7).all() and torch.isfinite(out[:3]).all()


@pytest.mark.parametrize("kv,q_len", [([700, 40, 1], [1, 1, 1]), ([90, 260], [50, 130])])
def test_strides_offsets_and_another_stream(kv, q_len):
    rng = np.random.default_rng(17)
    data, pages, table, k, v = make_cache(rng, kv, 64, 2, 128)
    T = sum(q_len)
    buf = torch.zeros(T * (4 * 128 + 5) + 3, dtype=torch.float16, device="cuda")
    q = buf[3:].view(T, 4 * 128 + 5)[:, : 512].unflatten(1, (4, 128))
    q.copy_(torch.from_numpy(rng.normal(size=(T, 4, 128))))
    base = torch.full(((T + 1) * 523 + 1,), 7.0, dtype=torch.float16, device="cuda")
    out = base[1:].view(T + 1, 523)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run_attend(data, pages, table, kv, q_len, q, 64, 2, 128, "f16", 0.09, 1, out=out)
    check_attend(out, q, k, v, q_len, 128, "f16", 0.09, 1, "strides")
    assert base[0] == 7
    if max(q_len) == 1:   # one row a request needs no starts
        again = run_attend(data, pages, table, kv, q_len, q, 64, 2, 128, "f16", 0.09, 1, starts=False)
        assert torch.equal(again[:T, :512], out[:T, :512])


def test_the_same_bits_every_time():
    rng = np.random.default_rng(18)
    for kv, q_len in (([3000, 700, 31], [1, 1, 1]), ([900, 64], [200, 33])):
        data, pages, table, k, v = make_cache(rng, kv, 64, 2, 128)
        q = torch.from_numpy(rng.normal(size=(sum(q_len), 8, 128))).cuda().half()
        outs = [run_attend(data, pages, table, kv, q_len, q, 64, 2, 128, "f16", 0.09, 1) for _ in range(4)]
        assert all(torch.equal(o, outs[0]) for o in outs)


def test_a_cache_past_32_bits_of_bytes():
    """A page whose bytes lie beyond 4 GiB: offsets are 64-bit in the write, the read and the attention."""
    D, hk, page = 128, 8, 256
    per = S.cache_bytes(1, page, hk, D)
    pages = (1 << 32) // per + 3
    data = torch.empty(pages * per, dtype=torch.uint8, device="cuda")
    assert data.numel() > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(5)
    T = 300
    k, v = (torch.randn(T, hk, D, generator=g, device="cuda").half() for _ in range(2))
    table = np.array([[pages - 1, pages - 2]])
    slots = [int(table[0, t // page]) * page + t % page for t in range(T)]
    cache = B.Cache(data=ptr(data), n_pages=pages, page_tokens=page, n_kv_heads=hk, head_dim=D)
    sl = ints(slots)
    B.dbf_cache_append(B.Heads(k=ptr(k), k_stride=hk * D, v=ptr(v), v_stride=hk * D, dtype=B.F16, n_tokens=T, n_kv_heads=hk, head_dim=D), cache, ptr(sl), G.stream_handle())
    ko, vo = (torch.empty(T, hk, D, device="cuda") for _ in range(2))
    B.dbf_cache_read(cache, ptr(sl), T, ptr(ko), ptr(vo), B.F32, G.stream_handle())
    torch.cuda.synchronize()
    assert float((ko - k.float()).abs().max()) < 0.4 and float((vo - v.float()).abs().max()) < 0.4
    for q_len in ([1], [50]):
        q = torch.randn(q_len[0], hk, D, generator=g, device="cuda").half()
        out = run_attend(data, pages, table, [T], q_len, q, page, hk, D, "f16", 0.1, 1)
        check_attend(out, q, [f64(ko)], [f64(vo)], q_len, D, "f16", 0.1, 1, "past 4 GiB")


# ---- log probabilities -------------------------------------------------------------------------------------


def run_logprobs(x, targets, top, stride=None, entropy=True):
    rows, vocab = x.shape
    code = {torch.float16: B.F16, torch.bfloat16: B.BF16, torch.float32: B.F32}[x.dtype]
    lp, h = (torch.full((rows + 1,), 7.0, device="cuda") for _ in range(2))
    ids, tops = torch.full((rows + 1, max(top, 1)), 77, dtype=torch.int32, device="cuda"), torch.full((rows + 1, max(top, 1)), 7.0, device="cuda")
    n = B.dbf_token_logprobs_workspace_bytes(rows, vocab, top)
    ws = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    t = None if targets is None else ints(targets)
    B.dbf_token_logprobs(ptr(x), code, x.stride(0) if rows > 1 else max(vocab, x.stride(0)), rows, vocab, ptr(t), top, ptr(lp) if t is not None else 0, ptr(h) if entropy else 0,
                         ptr(ids), ptr(tops), ptr(ws), n, G.stream_handle())
    torch.cuda.synchronize()
    assert (ws[n:] == 0xA5).all() and lp[rows] == 7 and h[rows] == 7 and (ids[rows] == 77).all() and (tops[rows] == 7).all()
    assert targets is not None or (lp == 7).all()
    assert entropy or (h == 7).all()
    return f64(lp[:rows]), f64(h[:rows]), ids[:rows, :top].cpu().numpy(), f64(tops[:rows, :top])


def check_logprobs(x, targets, top, what, **kw):
    lp, h, ids, tops = run_logprobs(x, targets, top, **kw)
    y = f64(x)
    want = S.token_logprobs(y, targets, top)
    with np.errstate(invalid="ignore"):
        width = np.where(np.isfinite(want[0]), np.abs(want[0]), 0)
        per = 2.0 ** -20 * (1 + math.log(x.shape[1]))
    close(lp, want[0], per + 2.0 ** -20 * width, what + " logprob")
    # (the mean of the scores and the logarithm of their sum: each to its own size)
    close(h, want[1], per + 2.0 ** -20 * np.nan_to_num(want[1]), what + " entropy")
    assert np.array_equal(ids, want[2]), what
    close(tops, want[3], per + 2.0 ** -20 * np.abs(np.nan_to_num(want[3], neginf=0)), what + " alternatives") if top else None


LOGPROBS = [(1, 1, 1, "f32"), (1, 2, 2, "f16"), (3, 63, 5, "bf16"), (2, 64, 64, "f32"), (5, 1000, 20, "f16"), (1, 32000, 20, "bf16"), (7, 32000, 0, "f16"), (300, 517, 3, "bf16"), (2, 50257, 64, "f32"),
            (1, 128256, 20, "bf16"), (33, 4099, 1, "f16"), (1, 150001, 5, "f32"), (600, 3000, 8, "f16"), (4, 8192, 33, "bf16"), (2, 8193, 64, "f16"), (1, 1000003, 20, "f16"), (65, 40000, 20, "bf16")]


@pytest.mark.parametrize("rows,vocab,top,dtype", LOGPROBS)
def test_token_logprobs(rows, vocab, top, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + vocab)
    x = (torch.randn(rows, vocab, generator=g, device="cuda") * 3).to(DT[dtype][0])
    targets = [int(v) for v in torch.randint(0, vocab, (rows,), generator=g, device="cuda")]
    if rows > 2:
        targets[1], targets[2] = -100, vocab
    check_logprobs(x, targets, top, "%d x %d %s" % (rows, vocab, dtype))


@pytest.mark.parametrize("vocab", [5, 64, 1000, 9000, 70000])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_token_logprobs_of_awkward_rows(vocab, dtype):
    """Ties everywhere, masks, rows of nothing, no numbers and infinities, large and equal logits, a lone peak, the largest at either end, rising and falling rows."""
    dt = DT[dtype][0]
    most = 6e4 if dtype == "f16" else 1e38
    g = torch.Generator(device="cuda").manual_seed(vocab)
    rows = [torch.zeros(vocab), torch.full((vocab,), -math.inf), torch.full((vocab,), most), torch.full((vocab,), -most), torch.arange(vocab) / vocab * 8, -torch.arange(vocab) / vocab * 8,
            torch.randint(0, 3, (vocab,)).float()]
    for v in (math.nan, math.inf):
        r = torch.randn(vocab)
        r[vocab // 2] = v
        r[vocab - 1] = v
        rows.append(r)
    for at in (0, vocab // 2, vocab - 1):
        r = torch.full((vocab,), -math.inf)
        r[at] = -3.0
        rows.append(r)
        r = torch.randn(vocab)
        r[at] = 200.0
        rows.append(r)
    r = torch.randn(vocab)
    r[torch.rand(vocab) < 0.7] = -math.inf
    r[vocab - 1] = 1
    rows.append(r)
    r = torch.randn(vocab)
    r[:] = torch.where(torch.rand(vocab) < 0.5, 0.0, -0.0)
    rows.append(r)
    r = torch.randn(vocab)
    r[torch.rand(vocab) < 0.5] = torch.finfo(dt).min
    rows.append(r)
    x = torch.stack(rows).cuda().to(dt)
    check_logprobs(x, [(7 * i) % vocab for i in range(len(rows))], min(vocab, 40), "awkward rows of %d" % vocab)


@pytest.mark.parametrize("rows,vocab,top,dtype", [(4, 53017, 20, "f16"), (9, 12345, 64, "bf16"), (2, 26000, 40, "f32")])
def test_token_logprobs_of_few_slices(rows, vocab, top, dtype):
    """Fewer slices than alternatives: spread over all of them, all in the first, all in the last, and in one that ends oddly."""
    g = torch.Generator(device="cuda").manual_seed(rows + vocab)
    x = torch.randn(rows, vocab, generator=g, device="cuda")
    x[0, : 2 * top] += 12
    x[1, vocab - 70:] += 12
    if rows > 2:
        x[2, 4080: 4100] += 12
    check_logprobs(x.to(DT[dtype][0]), [i * 77 % vocab for i in range(rows)], top, "%d x %d, %d alternatives" % (rows, vocab, top))


def test_token_logprobs_strides_and_what_may_be_left_out():
    g = torch.Generator(device="cuda").manual_seed(9)
    buf = torch.randn(50 * 1300 + 7, generator=g, device="cuda").bfloat16()
    for off, stride, vocab in ((0, 1300, 1300), (3, 1299, 777), (1, 1300, 1001), (7, 1300, 1300)):
        x = buf[off: off + 50 * stride].view(50, stride)[:, :vocab]
        check_logprobs(x, [i * 13 % vocab for i in range(50)], 7, "stride %d" % stride)
    x = torch.randn(4, 900, generator=g, device="cuda")
    a, b = run_logprobs(x, None, 5), run_logprobs(x, [1, 2, 3, 4], 5, entropy=False)
    c = run_logprobs(x, [1, 2, 3, 4], 5)
    assert np.array_equal(a[1], c[1]) and np.array_equal(a[2], c[2]) and np.array_equal(b[0], c[0]) and np.array_equal(b[3], c[3])


# ---- all of them in a captured graph -----------------------------------------------------------------------


def test_a_pass_in_a_graph():
    """Tables, write, attention and log probabilities of a decode step, captured once; lengths and tokens change between the replays, each of which
    equals the calls made one by one."""
    n, hq, hk, D, page, vocab = 3, 4, 2, 128, 32, 500
    g = torch.Generator(device="cuda").manual_seed(21)
    table, free = torch.full((n, 8), -1, dtype=torch.int32, device="cuda"), torch.arange(20, dtype=torch.int32, device="cuda")
    cached, new = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.ones(n, dtype=torch.int32, device="cuda")
    start, kv, pos, slots, status = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (n + 1, n, n, n, 2))
    qkv, q, out = torch.empty(n, (hq + 2 * hk) * D, dtype=torch.float16, device="cuda"), torch.empty(n, hq * D, dtype=torch.float16, device="cuda"), \
        torch.empty(n, hq * D, dtype=torch.float16, device="cuda")
    rope = torch.from_numpy(rope_table(300, D)).cuda()
    data = torch.zeros(S.cache_bytes(20, page, hk, D), dtype=torch.uint8, device="cuda")
    logits, target = torch.empty(n, vocab, dtype=torch.float16, device="cuda"), ints([3, 4, 5])
    lp, h, ids, tops = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 5, dtype=torch.int32, device="cuda"), torch.empty(n, 5, device="cuda")
    row, at = (hq + 2 * hk) * D, qkv.data_ptr()
    heads = B.Heads(q=at, q_stride=row, k=at + 2 * hq * D, k_stride=row, v=at + 2 * (hq + hk) * D, v_stride=row, q_out=ptr(q), q_out_stride=hq * D, dtype=B.F16, n_tokens=n,
                    n_q_heads=hq, n_kv_heads=hk, head_dim=D, rope=ptr(rope), rope_len=300, rot_dim=D, positions=ptr(pos))
    cache = B.Cache(data=ptr(data), n_pages=20, page_tokens=page, n_kv_heads=hk, head_dim=D)
    att = B.Attend(q=ptr(q), q_stride=hq * D, out=ptr(out), out_stride=hq * D, dtype=B.F16, n_tokens=n, n_seq=n, n_q_heads=hq, max_q=1, max_kv=8 * page, q_start=ptr(start),
                   kv_len=ptr(kv), block_table=ptr(table), table_stride=8, scale=0.09, causal=1)
    ws = torch.empty(max(256, B.dbf_cache_attend_workspace_bytes(att, cache)), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(max(256, B.dbf_token_logprobs_workspace_bytes(n, vocab, 5)), dtype=torch.uint8, device="cuda")

    def one():
        s = torch.cuda.current_stream().cuda_stream
        B.dbf_block_tables(ptr(cached), ptr(new), n, page, ptr(free), 20, ptr(table), 8, n, ptr(start), ptr(kv), ptr(pos), ptr(slots), ptr(status), s)
        B.dbf_cache_append(heads, cache, ptr(slots), s)
        B.dbf_cache_attend(att, cache, ptr(ws), ws.numel(), s)
        B.dbf_token_logprobs(ptr(logits), B.F16, vocab, n, vocab, ptr(target), 5, ptr(lp), ptr(h), ptr(ids), ptr(tops), ptr(ws2), ws2.numel(), s)

    outputs = (table, start, kv, pos, slots, status, q, out, data, lp, h, ids, tops)
    qkv.normal_(generator=g)
    logits.normal_(generator=g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    taken = 0
    for step in range(70):
        qkv.normal_(generator=g)
        logits.normal_(generator=g)
        cached.copy_(ints([step, step + 40, max(0, step - 9)]))
        if step == 0:
            table[1, :2] = ints([18, 19])
            free.copy_(torch.arange(20, dtype=torch.int32))
            taken = 0
        torch.cuda.synchronize()
        if step % 10 == 0:
            keep = [t.clone() for t in (table, data)]
            one()
            torch.cuda.synchronize()
            want = [t.clone() for t in outputs]
            table.copy_(keep[0])
            data.copy_(keep[1])
            for t in outputs[1:8] + outputs[9:]:
                t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        if step % 10 == 0:
            for t, w in zip(outputs, want):
                assert torch.equal(t, w), step
            assert torch.isfinite(out).all()
        took = int(status[0])
        assert int(status[1]) == 0
        taken += took
        free.copy_(torch.roll(free, -took))
    assert taken <= 18
