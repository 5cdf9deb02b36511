"""GPU tests of what stands between the layer products at the ends of its ranges, against oracle/serve_oracle.py in 64 bits.

Tolerances (u: half a unit in the last place of the output, relative, as in tests/test_serve_gpu.py):
  attention with scores so far apart that one token has all the weight: scores are fp32, an error d = 2^-18 sum |q k| scale each.  Where the largest of a row, in 64 bits,
      is ahead of all others by more than 2 d + 40 it is so in fp32 too and e^-40 of the rest is nothing: the row is that token's values, with the weight's rounding to fp16
      (2^-10) and the output's (u).  Elsewhere the weights may fall to any of the tokens, but they are weights: the row lies between its tokens' values, and values
      that are the same for all tokens come back, to the same roundings.
  log probabilities: as there, 2^-20 (1 + |x - max| + log of the number)."""
import math

import numpy as np
import pytest
import torch

import gpu_util as G
import test_serve_gpu as T
from oracle import serve_oracle as S
from paper_2505_11076_amd import binding as B

pytestmark = pytest.mark.gpu


# ---- attention: large scores ------------------------------------------------------------------------------


def write_cache(rng, k, v, page):
    """A cache of one request's keys and values [tokens, heads, D] (on the GPU), its table, and what it holds."""
    n, hk, D = k.shape
    each = -(-n // page)
    table = rng.permutation(each + 2)[:each][None]
    slots = T.ints([int(table[0, t // page]) * page + t % page for t in range(n)])
    data = torch.full((S.cache_bytes(each + 2, page, hk, D),), 0xFF, dtype=torch.uint8, device="cuda")
    cache = B.Cache(data=T.ptr(data), n_pages=each + 2, page_tokens=page, n_kv_heads=hk, head_dim=D)
    B.dbf_cache_append(B.Heads(k=T.ptr(k), k_stride=hk * D, v=T.ptr(v), v_stride=hk * D, dtype=B.F16, n_tokens=n, n_kv_heads=hk, head_dim=D), cache, T.ptr(slots), G.stream_handle())
    ko, vo = (torch.empty(n, hk, D, device="cuda") for _ in range(2))
    B.dbf_cache_read(cache, T.ptr(slots), n, T.ptr(ko), T.ptr(vo), B.F32, G.stream_handle())
    torch.cuda.synchronize()
    return data, each + 2, table, T.f64(ko), T.f64(vo)


def check_far_apart(out, q, k, v, dtype, scale, what):
    """Rows of one request, causal; see the tolerances above."""
    u, (rows, hq, D), n, hk = T.DT[dtype][2], q.shape, len(k), k.shape[1]
    got, qq, decided = T.f64(out[:rows]).reshape(rows, hq, D), T.f64(q), 0
    assert np.isfinite(got).all(), (what, np.argwhere(~np.isfinite(got))[:5])
    assert (out[rows:] == 7).all()
    for t in range(rows):
        seen = n - rows + t + 1
        for h in range(hq):
            K, V = k[:seen, h * hk // hq], v[:seen, h * hk // hq]
            x = K @ qq[t, h] * scale
            d = 2.0 ** -18 * (np.abs(K) @ np.abs(qq[t, h])).max() * abs(scale)
            order = np.sort(x)
            low, high = V.min(0), V.max(0)
            if seen == 1 or order[-1] - order[-2] > 2 * d + 40:
                low = high = V[x.argmax()]
                decided += 1
            slack = (2.0 ** -10 + u) * np.abs(V).max(0) + 2.0 ** -25
            bad = ~((got[t, h] >= low - slack) & (got[t, h] <= high + slack))
            assert not bad.any(), (what, t, h, np.argwhere(bad)[:3], got[t, h][bad][:3], low[bad][:3], high[bad][:3])
    G.say("%s: %d of %d rows have one token" % (what, decided, rows * hq))


def far_keys(rng, n, hk, D):
    """Keys of the size 2e4 and values of which the first half is 1 for all tokens."""
    k = torch.from_numpy(rng.choice([-1.0, 1.0], (n, hk, D)) * rng.uniform(0.5, 1.0, (n, hk, D)) * 2e4).cuda().half()
    v = torch.from_numpy(rng.uniform(0, 1, (n, hk, D))).cuda().half()
    v[:, :, : D // 2] = 1
    return k, v


@pytest.mark.parametrize("power", [12, 18, 20, 22, 24, 26, 27, 28, 29, 30, 31, 33, 40, 70, 110])
@pytest.mark.parametrize("rows,n,hq,hk,D", [(1, 300, 4, 2, 64), (3, 200, 8, 2, 128), (60, 300, 2, 1, 64), (130, 257, 2, 2, 128), (40, 150, 1, 1, 256), (20, 2500, 2, 1, 128)])
def test_cache_attend_of_scores_far_apart(rows, n, hq, hk, D, power):
    """Scores of about 2^power (to base 2), up to where fp32 tells none apart that lie near each other."""
    rng = np.random.default_rng(power * 1000 + rows)
    k, v = far_keys(rng, n, hk, D)
    data, pages, table, kk, vv = write_cache(rng, k, v, 64)
    q = torch.from_numpy(rng.choice([-1.0, 1.0], (rows, hq, D)) * rng.uniform(0.5, 1.0, (rows, hq, D)) * 2e4).cuda().half()
    scale = float(np.float32(2.0 ** power / (2e4 * 2e4 * math.sqrt(D))))
    out = T.run_attend(data, pages, table, [n], [rows], q, 64, hk, D, "f16", scale, 1)
    check_far_apart(out, q, kk, vv, "f16", scale, "scores of 2^%d" % power)


@pytest.mark.parametrize("rows,D", [(2, 128), (70, 128), (70, 64)])
@pytest.mark.parametrize("falling", [False, True])
@pytest.mark.parametrize("power", [24, 30, 34])
def test_cache_attend_of_scores_that_grow_along_the_tokens(rows, D, falling, power):
    """From 2^(power - 24) to 2^power, or back: tiles of ordinary scores before and behind those of very large ones."""
    rng = np.random.default_rng(power + rows)
    n = 900
    k, v = far_keys(rng, n, 1, D)
    size = torch.exp2(torch.linspace(-14, 0, n, device="cuda"))
    k = (k.float() * (size.flip(0) if falling else size)[:, None, None]).half()
    data, pages, table, kk, vv = write_cache(rng, k, v, 32)
    sizes = 2.0 ** rng.uniform(-10, 0, (rows, 2, 1))
    q = torch.from_numpy(rng.normal(size=(rows, 2, D)) * sizes * 1e4).cuda().half()
    scale = float(np.float32(2.0 ** power / (2e4 * 2e4 * math.sqrt(D))))
    out = T.run_attend(data, pages, table, [n], [rows], q, 32, 1, D, "f16", scale, 1)
    check_far_apart(out, q, kk, vv, "f16", scale, "growing to 2^%d" % power)


@pytest.mark.parametrize("size", [1e30, 1e34, 1e36, 1e38, 3e38])
@pytest.mark.parametrize("scale", [0.125, -0.125, 3.0, 1e-30])
@pytest.mark.parametrize("rows", [2, 50])
def test_cache_attend_of_the_largest_queries(rows, scale, size):
    """bfloat16 queries up to the type's largest with ordinary keys: a score may be beyond fp32, its row still is its likeliest token's."""
    rng = np.random.default_rng(rows)
    n, D = 120, 64
    k = torch.from_numpy(rng.normal(size=(n, 1, D)) * 3).cuda().half()
    v = torch.from_numpy(rng.uniform(0, 1, (n, 1, D))).cuda().half()
    v[:, :, : D // 2] = 1
    data, pages, table, kk, vv = write_cache(rng, k, v, 32)
    q = torch.from_numpy(rng.uniform(-1, 1, (rows, 2, D)) * size).cuda().bfloat16()
    scale = float(np.float32(scale))
    out = T.run_attend(data, pages, table, [n], [rows], q, 32, 1, D, "bf16", scale, 1)
    check_far_apart(out, q, kk, vv, "bf16", scale, "queries of %g times %g" % (size, scale))


# ---- attention: row starts --------------------------------------------------------------------------------


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("starts,fine", [([0, 3, 6], [0, 1]), ([-2, 3, 6], [1]), ([0, 3, 8], [0]), ([0, 6, 3], [0]), ([-4, -1, 6], []), ([3, 6, 2147483647], [0]), ([-2147483648, 2, 6], [1])])
def test_row_starts_outside_the_tensor(starts, fine, few):
    """Starts below 0 or beyond the tokens: which token a row is would be a guess, so what such a request has of the tensor's rows comes out as no numbers, and no others."""
    rng = np.random.default_rng(16)
    n_rows = 6 if few else 6 * 20
    starts = [s if abs(s) > 1000 else s * (n_rows // 6) for s in starts]
    kv = [190, 170]
    data, pages, table, k, v = T.make_cache(rng, kv, 32, 1, 64)
    q = torch.from_numpy(rng.normal(size=(n_rows, 2, 64))).cuda().half()
    out = torch.full((n_rows + 1, 2 * 64), 7.0, dtype=torch.float16, device="cuda")
    st, kvd, tab = T.ints(starts), T.ints(kv), T.ints(table)
    cache = B.Cache(data=T.ptr(data), n_pages=pages, page_tokens=32, n_kv_heads=1, head_dim=64)
    a = B.Attend(q=T.ptr(q), q_stride=128, out=T.ptr(out), out_stride=128, dtype=B.F16, n_tokens=n_rows, n_seq=2, n_q_heads=2, max_q=n_rows, max_kv=190, q_start=T.ptr(st),
                 kv_len=T.ptr(kvd), block_table=T.ptr(tab), table_stride=tab.shape[1], scale=0.1, causal=1)
    ws = torch.empty(max(256, B.dbf_cache_attend_workspace_bytes(a, cache)), dtype=torch.uint8, device="cuda")
    B.dbf_cache_attend(a, cache, T.ptr(ws), ws.numel(), G.stream_handle())
    torch.cuda.synchronize()
    got, mine = T.f64(out), np.full(n_rows + 1, 7.0)
    for i in range(2):
        at, end = max(starts[i], 0), min(starts[i + 1], n_rows)
        if i in fine:
            o, w, size = S.attend(T.f64(q[at: end]), k[i], v[i], 0.1, True)
            T.close(got[at: end].reshape(-1, 2, 64), o, 2.0 ** -10 * w + 2.0 ** -11 * np.abs(o) + 2 * 2.0 ** -18 * size[..., None] * w, "request %d of %s" % (i, starts))
            mine[at: end] = 0
        elif end > at:
            assert np.isnan(got[at: end]).all(), (i, starts)
            mine[at: end] = 0
    assert (got[mine == 7] == 7).all(), starts


# ---- attention: more items than shares ---------------------------------------------------------------------


@pytest.mark.parametrize("D,n,dtype,hq", [(256, 300, "f16", 2), (256, 260, "bf16", 6), (128, 400, "f16", 8), (64, 520, "bf16", 2)])
def test_cache_attend_of_more_items_than_shares(D, n, dtype, hq):
    """Shared out where there are at least as many items as workgroups (a record is kept for each share, not for each item): requests mostly short, some empty, some without rows,
    some longer than a share, one much longer."""
    rng = np.random.default_rng(D + n)
    hk, page = 2, 32
    shares = {64: 1024, 128: 768, 256: 512}[D]
    longest = 1200 + 11 * n * hk + 700
    assert n * hk >= shares
    kv = [int(x) for x in rng.choice([0, 1, 31, 32, 33, 64, 90, 500, 1111], n, p=[0.1, 0.1, 0.1, 0.1, 0.1, 0.2, 0.2, 0.07, 0.03])]
    kv[n // 3], kv[n - 1] = longest, 2222
    q_len = [int(x) for x in rng.choice([0, 1, 2], n, p=[0.1, 0.8, 0.1])]
    q_len[n // 3] = q_len[n - 1] = 1
    data, pages, table, k, v = T.make_cache(rng, kv, page, hk, D)
    q = torch.from_numpy(rng.normal(size=(sum(q_len), hq, D))).cuda().to(T.DT[dtype][0])
    a = B.Attend(dtype=T.DT[dtype][1], n_tokens=len(q), n_seq=n, n_q_heads=hq, max_q=2, max_kv=longest, table_stride=table.shape[1], scale=0.1, causal=1)
    assert B.dbf_cache_attend_workspace_bytes(a, B.Cache(data=T.ptr(data), n_pages=pages, page_tokens=page, n_kv_heads=hk, head_dim=D)) > 0
    out = T.run_attend(data, pages, table, kv, q_len, q, page, hk, D, dtype, 1 / math.sqrt(D), 1)
    u, got, qq, at, worst = T.DT[dtype][2], T.f64(out[:-1]).reshape(-1, hq, D), T.f64(q), 0, 0.0
    for i, m in enumerate(q_len):
        o, w, size = S.attend(qq[at: at + m], k[i], v[i], 1 / math.sqrt(D), True)
        bound = 2.0 ** -10 * w + u * np.abs(o) + 2 * 2.0 ** -18 * size[..., None] * w + 2.0 ** -25
        off = np.abs(got[at: at + m] - o)
        assert (off <= bound).all(), (i, kv[i], m)
        worst = max(worst, float((off / bound).max(initial=0)))
        at += m
    G.say("%d items on %d shares: worst %.3g of its bound" % (n * hk, shares, worst))
    assert (out[-1] == 7).all()


# ---- log probabilities -------------------------------------------------------------------------------------


@pytest.mark.parametrize("vocab", [5, 8, 64, 1000, 9000, 70000])
def test_token_logprobs_of_the_largest_logits(vocab):
    """fp32 logits up to the type's largest are numbers like others."""
    top = float(np.finfo(np.float32).max)
    g = torch.Generator().manual_seed(vocab)
    rows = []
    for value, at in ((top, 0), (top, vocab - 1), (3.401e38, vocab // 2), (-top, 3), (-3.401e38, vocab - 2)):
        r = torch.randn(vocab, generator=g)
        r[at] = value
        rows.append(r)
    rows += [torch.full((vocab,), top), torch.full((vocab,), -top), torch.full((vocab,), 3.4015e38)]
    r = torch.full((vocab,), top)
    r[vocab // 2:] = -top
    rows.append(r)
    r = torch.full((vocab,), -math.inf)
    r[1] = top
    rows.append(r)
    r = torch.randn(vocab, generator=g)
    r[2], r[vocab // 2] = top, math.inf
    rows.append(r)
    x = torch.stack(rows).cuda()
    for targets, n in (([(3 * i) % vocab for i in range(len(rows))], 20), ([0, vocab - 1, vocab // 2, 3, vocab - 2, 1, 1, 2, 0, 1, 2], 3)):
        got, want = T.run_logprobs(x, targets, min(vocab, n)), S.token_logprobs(T.f64(x), targets, min(vocab, n))
        assert np.array_equal(got[2], want[2])
        per = 2.0 ** -20 * (1 + math.log(vocab))
        for i, what in ((0, "logprob"), (1, "entropy"), (3, "alternatives")):
            with np.errstate(over="ignore"):
                w = want[i].astype(np.float32).astype(np.float64)   # (-max less max is -infinity in fp32)
            T.close(got[i], w, per + 2.0 ** -20 * np.abs(np.nan_to_num(w, neginf=0)), "largest logits of %d, %s" % (vocab, what))


# ---- calls of more threads than a launch takes ---------------------------------------------------------------


def test_calls_of_more_rows_than_a_launch_takes():
    """A launch takes fewer than 2^32 threads."""
    n = (1 << 24) + 5
    x = torch.empty(n, 8, dtype=torch.float16, device="cuda").normal_()
    lp, h = (torch.full((n + 1,), 7.0, device="cuda") for _ in range(2))
    t = torch.randint(0, 8, (n,), device="cuda", dtype=torch.int32)
    ids, tops = torch.full((n + 1, 2), 77, dtype=torch.int32, device="cuda"), torch.full((n + 1, 2), 7.0, device="cuda")
    B.dbf_token_logprobs(T.ptr(x), B.F16, 8, n, 8, T.ptr(t), 2, T.ptr(lp), T.ptr(h), T.ptr(ids), T.ptr(tops), 0, 0, G.stream_handle())
    torch.cuda.synchronize()
    want = torch.log_softmax(x.double(), 1)
    assert float((lp[:n] - want.gather(1, t.long()[:, None])[:, 0]).abs().max()) <= 2.0 ** -20 * 40
    assert float((h[:n] + (want.exp() * want).sum(1)).abs().max()) <= 2.0 ** -20 * 40
    best = want.sort(dim=1, descending=True, stable=True)
    assert torch.equal(ids[:n].long(), best.indices[:, :2]) and float((tops[:n] - best.values[:, :2]).abs().max()) <= 2.0 ** -20 * 40
    assert lp[n] == 7 and h[n] == 7 and (ids[n] == 77).all() and (tops[n] == 7).all()


@pytest.mark.parametrize("D", [2, 64])
def test_heads_of_more_tokens_than_a_launch_takes(D):
    """(a token's head is a wavefront's)"""
    n, heads = (1 << 26) + 9, 1
    q = torch.empty(n, heads * D, dtype=torch.float16, device="cuda")
    q.view(torch.int16).random_(0, 1 << 14)
    out = torch.full((n + 1, heads * D), 7.0, dtype=torch.float16, device="cuda")
    pos = torch.arange(n, device="cuda", dtype=torch.int32) % 4
    rope = torch.tensor([[1.0] * (D // 2) + [0.0] * (D // 2), [0.0] * (D // 2) + [1.0] * (D // 2)] * 2, device="cuda")   # as it is, a quarter of a turn, ...
    B.dbf_qk_norm_rope(B.Heads(q=T.ptr(q), q_stride=heads * D, q_out=T.ptr(out), q_out_stride=heads * D, dtype=B.F16, n_tokens=n, n_q_heads=heads, head_dim=D, rope=T.ptr(rope),
                               rope_len=4, rot_dim=D, positions=T.ptr(pos)), G.stream_handle())
    torch.cuda.synchronize()
    x, y = q.view(n, heads, D), out[:n].view(n, heads, D)
    assert torch.equal(y[0::2], x[0::2])
    assert torch.equal(y[1::2, :, : D // 2], -x[1::2, :, D // 2:]) and torch.equal(y[1::2, :, D // 2:], x[1::2, :, : D // 2])
    assert (out[n] == 7).all()


def test_a_cache_read_of_more_tokens_than_a_launch_takes():
    n = (1 << 26) + 3
    rng = np.random.default_rng(1)
    data = torch.empty(S.cache_bytes(1, 32, 1, 64), dtype=torch.uint8, device="cuda")
    cache = B.Cache(data=T.ptr(data), n_pages=1, page_tokens=32, n_kv_heads=1, head_dim=64)
    k, v = (torch.from_numpy(rng.normal(size=(32, 64))).cuda().half() for _ in range(2))
    slots = torch.arange(n, device="cuda", dtype=torch.int32) % 33
    B.dbf_cache_append(B.Heads(k=T.ptr(k), k_stride=64, v=T.ptr(v), v_stride=64, dtype=B.F16, n_tokens=32, n_kv_heads=1, head_dim=64), cache, T.ptr(slots), G.stream_handle())
    ko, vo = (torch.full((n + 1, 64), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
    B.dbf_cache_read(cache, T.ptr(slots), n, T.ptr(ko), T.ptr(vo), B.F16, G.stream_handle())
    torch.cuda.synchronize()
    for o in (ko, vo):
        assert (o[n] == 7).all() and (o[32] == 0).all() and (o[:32] != 7).all()
        whole = (n // 33) * 33
        assert torch.equal(o[:whole].view(-1, 33, 64), o[:33].expand(whole // 33, 33, 64)) and torch.equal(o[whole: n], o[: n - whole])


# ---- log probabilities: long sums ---------------------------------------------------------------------------


@pytest.mark.parametrize("rows,vocab,dtype", [(800, 32000, "bf16"), (800, 150000, "f16"), (800, 1 << 22, "f16"), (1, 1 << 24, "f32"), (5, 1 << 24, "f16"), (800, 128256, "f32")])
def test_token_logprobs_of_many_equal_logits(rows, vocab, dtype):
    """A few tokens at 0 and all others alike, further down by another amount in each row: equal terms are rounded the same way each time they are added, so what is lost grows with their number
    unless sums are kept short or what they lose is kept."""
    d = torch.linspace(0.03, 9.5, rows, device="cuda").to(T.DT[dtype][0])
    ones = torch.arange(vocab, device="cuda") % (1 << 18) < 2048
    x = torch.where(ones, torch.zeros((), dtype=d.dtype, device="cuda"), -d[:, None])
    lp, h = (torch.full((rows + 1,), 7.0, device="cuda") for _ in range(2))
    t = torch.where(torch.arange(rows, device="cuda") % 2 == 0, 0, vocab - 1).to(torch.int32)
    ws = torch.empty(max(256, B.dbf_token_logprobs_workspace_bytes(rows, vocab, 0)), dtype=torch.uint8, device="cuda")
    B.dbf_token_logprobs(T.ptr(x), T.DT[dtype][1], vocab, rows, vocab, T.ptr(t), 0, T.ptr(lp), T.ptr(h), 0, 0, T.ptr(ws), ws.numel(), G.stream_handle())
    torch.cuda.synchronize()
    n, at = int(ones.sum()), T.f64(d)
    assert not ones[vocab - 1]
    z = n + (vocab - n) * np.exp(-at)
    want = np.where(np.arange(rows) % 2 == 0, 0.0, -at) - np.log(z)
    entropy = np.log(z) + (vocab - n) * np.exp(-at) / z * at
    per = 2.0 ** -20 * (1 + math.log(vocab))
    T.close(T.f64(lp[:rows]), want, per + 2.0 ** -20 * np.abs(want), "logprob of %d x %d" % (rows, vocab))
    T.close(T.f64(h[:rows]), entropy, per + 2.0 ** -20 * entropy, "entropy of %d x %d" % (rows, vocab))
    assert lp[rows] == 7 and h[rows] == 7


# ---- attention: launches that share work out, in a captured graph ---------------------------------------------


def test_shared_and_cut_calls_in_a_graph():
    """Single tokens in equal shares and rows on a long axis in parts, captured once: lengths and queries change between the replays, each of which equals the calls made one by one."""
    rng = np.random.default_rng(8)
    kv, page, hk, D = [6000, 900, 64, 2500], 32, 2, 128
    data, pages, table, k, v = T.make_cache(rng, kv, page, hk, D)
    tab, cache = T.ints(table), B.Cache(data=T.ptr(data), n_pages=pages, page_tokens=page, n_kv_heads=hk, head_dim=D)
    g = torch.Generator(device="cuda").manual_seed(4)
    calls = []
    for rows in (1, 20):
        n = 4 * rows
        q, out = (torch.empty(n, 4 * D, dtype=torch.float16, device="cuda") for _ in range(2))
        start, length = T.ints([i * rows for i in range(5)]), T.ints(kv)
        a = B.Attend(q=T.ptr(q), q_stride=4 * D, out=T.ptr(out), out_stride=4 * D, dtype=B.F16, n_tokens=n, n_seq=4, n_q_heads=4, max_q=rows, max_kv=6000, q_start=T.ptr(start),
                     kv_len=T.ptr(length), block_table=T.ptr(tab), table_stride=tab.shape[1], scale=0.09, causal=1)
        size = B.dbf_cache_attend_workspace_bytes(a, cache)
        assert size > 0
        calls.append((a, q, out, start, length, torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")))

    def both():
        for a, _, _, _, _, ws in calls:
            B.dbf_cache_attend(a, cache, T.ptr(ws), ws.numel(), torch.cuda.current_stream().cuda_stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for step in range(12):
        for _, q, out, start, length, _ in calls:
            q.normal_(generator=g)
            rows = len(q) // 4
            length.copy_(T.ints([int(rng.integers(0, n + 1)) for n in kv]) if step else T.ints(kv))
            start.copy_(T.ints(np.cumsum([0, rows, int(rng.integers(0, rows + 1)), rows, rows])))
            out.fill_(7)
        both()
        torch.cuda.synchronize()
        want = [c[2].clone() for c in calls]
        for c in calls:
            c[2].fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for c, w in zip(calls, want):
            assert torch.equal(c[2], w), step
            at = T.f64(c[3]).astype(int)
            for i in range(4):
                n = int(c[4][i])
                o, weight, size = S.attend(T.f64(c[1][at[i]: at[i + 1]]).reshape(-1, 4, D), k[i][:n], v[i][:n], 0.09, True)
                T.close(T.f64(w[at[i]: at[i + 1]]).reshape(-1, 4, D), o, 2.0 ** -10 * weight + 2.0 ** -11 * np.abs(o) + 2 * 2.0 ** -18 * size[..., None] * weight, "step %d" % step)
