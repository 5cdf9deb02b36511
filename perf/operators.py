"""What stands between the layer products of a decoder's token pass, as cases: page tables for new tokens, norms and rotation of
queries and keys, the write to a cache held in 4 bits, attention over it, and log probabilities of given tokens.

`run` is one call as a serving program makes it (`own`), or the same in elementary torch operations in 32 bits.  `exact` is the
operator's definition in 64 bits, from the inputs as they were made.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 64   # values of a token and head that share a scale
BLOCK = 32   # tokens of a record of the cache


# ---- cases -------------------------------------------------------------------------------------------------


def listed():
    return [
        # a decode step of a batch: every request gets one token, now and then a page
        dict(name="tables_decode", kind="tables", n_seq=61, cached=4000, new_min=1, new_max=1, page=64),
        # admission of many requests with prompts of all lengths, some with nothing new
        dict(name="tables_prompts", kind="tables", n_seq=4096, cached=900, new_min=0, new_max=63, page=32),
        # one token's heads, as many keys as queries (a 4096-wide layer in heads of 128)
        dict(name="rope_token", kind="rope", tokens=1, q_heads=32, kv_heads=32, dim=128, rot=128, interleaved=False, dtype="f16"),
        # a prompt, shared key heads, part of each head rotated, neighbouring pairs
        dict(name="rope_prompt", kind="rope", tokens=8191, q_heads=32, kv_heads=8, dim=128, rot=64, interleaved=True, dtype="bf16"),
        # a decode step of a batch into the cache
        dict(name="append_decode", kind="append", tokens=48, q_heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, dtype="f16", page=64),
        # a prompt into the cache, every query head with keys of its own
        dict(name="append_prompt", kind="append", tokens=2047, q_heads=32, kv_heads=32, dim=128, rot=128, interleaved=False, dtype="f16", page=64),
        # one request at a time, a short conversation: latency
        dict(name="attend_token", kind="attend", n_seq=1, q_min=1, q_max=1, kv_min=333, kv_max=333, q_heads=32, kv_heads=32, dim=128, page=64, dtype="f16"),
        # one request over a long document: a long axis and few rows
        dict(name="attend_long", kind="attend", n_seq=1, q_min=1, q_max=1, kv_min=131071, kv_max=131071, q_heads=32, kv_heads=8, dim=128, page=64, dtype="f16"),
        # a serving batch of all lengths
        dict(name="attend_ragged", kind="attend", n_seq=64, q_min=1, q_max=1, kv_min=1, kv_max=8192, q_heads=32, kv_heads=8, dim=128, page=32, dtype="bf16"),
        # prompts of a few requests, causal
        dict(name="attend_prompt", kind="attend", n_seq=3, q_min=2048, q_max=2048, kv_min=2048, kv_max=3001, q_heads=32, kv_heads=32, dim=128, page=64, dtype="f16"),
        # the next token of one request, with alternatives
        dict(name="logprobs_token", kind="logprobs", rows=1, vocab=128256, top=20, dtype="bf16"),
        # a text judged by a compressed model
        dict(name="logprobs_text", kind="logprobs", rows=2048, vocab=32000, top=0, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "rope", "append", "attend", "attend", "attend", "logprobs"])
    page, dtype = rng.choice([32, 64, 128]), rng.choice(["f16", "bf16"])
    if kind == "tables":
        new_min, new_max = rng.choice([(1, 1), (0, 8), (0, 63), (1, 300)])
        return dict(kind=kind, n_seq=_log(rng, 1, 4096 if new_max < 64 else 400), cached=_log(rng, 50, 4000), new_min=new_min, new_max=new_max, page=page)
    if kind == "logprobs":
        vocab = _log(rng, 1000, 150000)
        return dict(kind=kind, rows=_log(rng, 1, min(2048, 65000000 // vocab)), vocab=vocab, top=rng.choice([0, 1, 5, 20]), dtype=rng.choice(["f16", "bf16", "f32"]))
    dim = rng.choice([64, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    q_heads = kv_heads * rng.choice([1, 2, 4, 7, 8])
    if kind in ("rope", "append"):
        c = dict(kind=kind, tokens=_log(rng, 1, max(1, min(8000, 24000000 // ((q_heads + 2 * kv_heads) * dim)))), q_heads=q_heads, kv_heads=kv_heads, dim=dim,
                 rot=rng.choice([dim, dim, dim // 2]), interleaved=rng.random() < 0.5, dtype=dtype)
        return dict(c, page=page) if kind == "append" else c
    form = rng.choice(["one", "batch", "few", "chunk", "prompt"])
    kv = dict(one=(1, 100000), batch=(1, 8000), few=(16, 8000), chunk=(1000, 16000), prompt=(100, 2000))[form]
    kv_max = _log(rng, *kv)
    n_seq = 1 if form == "one" else rng.randint(1, max(1, min(48, 4000000 // (kv_max * kv_heads * dim // 128))))
    q_min, q_max = dict(one=(1, 1), batch=(1, 1), few=(1, 9), chunk=(100, 500), prompt=(kv_max // 2, kv_max))[form]
    q_max = min(q_max, kv_max)
    q_min = min(max(1, q_min), q_max)
    c = dict(kind=kind, n_seq=n_seq, q_min=q_min, q_max=q_max, kv_min=max(q_max, rng.choice([1, kv_max // 2, kv_max])), kv_max=kv_max, q_heads=q_heads,
             kv_heads=kv_heads, dim=dim, page=page, dtype=dtype)
    # (no more bytes, products or scores than the largest of the listed ones have)
    while work(c)["bytes"] > 3.2e8 or work(c)["flops"] > 1.6e11 or c["n_seq"] * c["q_max"] * q_heads * kv_max > 800000000:
        if c["n_seq"] > 1:
            c["n_seq"] -= 1
        else:
            c["q_max"] = c["q_max"] * 3 // 4
            c["q_min"] = min(c["q_min"], c["q_max"])
    return c


def _lengths(case):
    """The lengths of a case's requests, the same for every seed."""
    rng = random.Random(",".join("%s=%s" % kv for kv in sorted(case.items()) if kv[0] != "name"))
    n = case["n_seq"]
    if case["kind"] == "tables":
        return [rng.randint(0, 2 * case["cached"]) for _ in range(n)], [rng.randint(case["new_min"], case["new_max"]) for _ in range(n)]
    kv = [rng.randint(case["kv_min"], case["kv_max"]) for _ in range(n)]
    kv[rng.randrange(n)] = case["kv_max"]
    q = [min(rng.randint(case["q_min"], case["q_max"]), k) for k in kv]
    return kv, q


# ---- inputs ------------------------------------------------------------------------------------------------


def _rng(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _pages(lengths, page):
    return [-(-n // page) for n in lengths]


def _heads(case, g):
    """A projection's output [tokens][q, k and v heads], norm weights and positions of a prompt that goes on at some place."""
    T, hq, hk, D = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"]
    dt = DTYPES[case["dtype"]]
    qkv = (_normal(g, T, hq + 2 * hk, D) * torch.exp(0.5 * _normal(g, D))).to(dt)
    w = [(1 + 0.2 * _normal(g, D)).to(dt) for _ in range(2)]
    pos = torch.arange(T, device=DEV, dtype=torch.int32) + torch.randint(0, 100, (1,), generator=g, device=DEV, dtype=torch.int32)
    return qkv, w, pos


def _rope_table(n, rot):
    f = torch.exp(torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) * (-math.log(10000.0) / rot))
    a = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _append_slots(case, g):
    n = -(-case["tokens"] // case["page"]) + 3
    pages = torch.randperm(n, generator=g, device=DEV)
    t = torch.arange(case["tokens"], device=DEV) + torch.randint(0, case["page"], (1,), generator=g, device=DEV)
    return n, (pages[t // case["page"]] * case["page"] + t % case["page"]).to(torch.int32)


def _up7(x):
    """x >= 0 rounded up to 7 significant bits, and to a multiple of 2^-24."""
    x = ((x.contiguous().view(torch.int32) + 0x1FFFF) & ~0x1FFFF).view(torch.float32)
    return torch.ceil(x * 16777216.0) * (1 / 16777216.0)


def _quantise(x):
    """Codes, scales and zero points of x [..., D]: a group is the values of every D/64-th run of 16."""
    n = x.shape[-1] // GROUP
    y = x.clamp(-57344, 57344).unflatten(-1, (4, n, 16))
    lo, hi = y.amin((-3, -1), keepdim=True).clamp(max=0), y.amax((-3, -1), keepdim=True).clamp(min=0)
    s = _up7((hi - lo) / torch.full_like(hi, 15))   # (a division by a plain number would be a product with its rounded reciprocal)
    d = torch.where(s > 0, s, 1)
    z = torch.round(-lo / d)
    return (torch.round(y / d) + z).clamp(0, 15), s, z


def _values(codes, s, z):
    return (s * (codes - z)).flatten(-3)


def _cache(case, g):
    """What the cache of an attention case holds, (codes, scales, zero points) of keys and values [pages][heads][page][4][D/64][16], and the
    block table: pages of all requests in one random order, and a few that are nobody's."""
    kv, _ = _lengths(case)
    each = _pages(kv, case["page"])
    n = sum(each) + 2
    order = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    table = torch.full((case["n_seq"], max(each) + 1), -1, dtype=torch.int32, device=DEV)
    seq = torch.repeat_interleave(torch.arange(case["n_seq"], device=DEV), torch.tensor(each, device=DEV))
    first = torch.tensor([sum(each[:i]) for i in range(len(each))], device=DEV)
    table[seq, torch.arange(sum(each), device=DEV) - first[seq]] = order[: sum(each)]
    shape = (n, case["kv_heads"], case["page"], case["dim"])
    channels = torch.exp(0.4 * _normal(g, case["kv_heads"], 1, case["dim"]))
    k = _quantise(_normal(g, *shape) * channels)
    v = _quantise(_normal(g, *shape) * 0.7)
    return k, v, table


def _words(s, z):
    """A group's scale and -scale * zero point, both exact in fp16: [..., page, 1, n, 1] -> bytes [..., page/32][n][32][4]."""
    w = torch.stack([s, -s * z], -1).to(torch.float16).flatten(-5, -2)                  # ..., page * n, 2
    w = w.unflatten(-2, (-1, BLOCK, s.shape[-2])).transpose(-2, -3).contiguous()         # ..., blocks, n, 32, 2
    return w.view(torch.uint8).flatten(-3)


def _pack(k, v):
    """The cache's bytes: records of 32 tokens of a page and head.  Keys by tokens, two neighbouring values a byte; values in words of
    four tokens, a byte the values of two runs of 16 of the group; then the groups' words."""
    kc, vc = (x[0].to(torch.uint8) for x in (k, v))
    n = kc.shape[-2]
    pages, heads, page = kc.shape[:3]
    kc = kc.view(pages, heads, page // BLOCK, BLOCK, 32 * n, 2)
    kc = (kc[..., 0] | kc[..., 1] << 4).flatten(-2)
    vc = vc.view(pages, heads, page // BLOCK, 2, 4, 4, 2, 2, n, 16)   # tile, g, i, q, half, group, lane
    vc = vc[..., 0, :, :] | vc[..., 1, :, :] << 4                     # tile, g, i, q, group, lane
    vc = vc.permute(0, 1, 2, 7, 4, 8, 6, 3, 5).flatten(3)             # group, g, lane, q, tile, i
    return torch.cat([kc, vc, _words(k[1], k[2]), _words(v[1], v[2])], -1).contiguous()


def _logits(case, g):
    x = (_normal(g, case["rows"], case["vocab"]) * 2.5).to(DTYPES[case["dtype"]])
    # (an even share of texts' tokens are the likely ones)
    t = torch.randint(0, case["vocab"], (case["rows"],), generator=g, device=DEV)
    best = x.argmax(1)
    return x, torch.where(torch.rand(case["rows"], generator=g, device=DEV) < 0.5, best, t).to(torch.int32)


def _bytes(n):
    return torch.empty(max(int(n), 256), dtype=torch.uint8, device=DEV)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(n):
    return _ints([sum(n[:i]) for i in range(len(n) + 1)])


def _tables_inputs(case, g):
    cached, new = _lengths(case)
    have, total = _pages(cached, case["page"]), _pages([c + n for c, n in zip(cached, new)], case["page"])
    order = torch.randperm(sum(total) + 5, generator=g, device=DEV).to(torch.int32)
    table = torch.full((case["n_seq"], max(max(total), 1) + 2), -1, dtype=torch.int32, device=DEV)
    seq = torch.repeat_interleave(torch.arange(case["n_seq"], device=DEV), torch.tensor(have, device=DEV))
    first = torch.tensor([sum(have[:i]) for i in range(len(have))], device=DEV)
    table[seq, torch.arange(sum(have), device=DEV) - first[seq]] = order[: sum(have)]
    return _ints(cached), _ints(new), order[sum(have):].contiguous(), table


def prepare(case, seed):
    g, kind = _rng(seed), case["kind"]
    s = dict(case=case)
    empty = lambda *shape, dtype=torch.int32: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    if kind == "tables":
        s["cached"], s["new"], s["free"], s["table"] = _tables_inputs(case, g)
        n = sum(_lengths(case)[1])
        s |= dict(tokens=n, start=empty(case["n_seq"] + 1), kv=empty(case["n_seq"]), pos=empty(max(n, 1)), slots=empty(max(n, 1)), status=empty(2))
    elif kind in ("rope", "append"):
        T, hq, hk, D = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"]
        s["qkv"], s["w"], s["pos"] = _heads(case, g)
        s["rope"] = _rope_table(T + 100, case["rot"])
        s["q"] = empty(T, hq, D, dtype=DTYPES[case["dtype"]])
        s["k"] = empty(T, hk, D, dtype=DTYPES[case["dtype"]] if kind == "rope" else torch.float16)
        if kind == "append":
            s["v"] = empty(T, hk, D, dtype=torch.float16)
            s["pages"], s["slots"] = _append_slots(case, g)
            s["cache"] = torch.zeros(s["pages"] * case["page"] * hk * D * 36 // 32, dtype=torch.uint8, device=DEV)
    elif kind == "attend":
        kv, q = _lengths(case)
        k, v, s["table"] = _cache(case, g)
        s["cache"] = _pack(k, v)
        s["q"] = _normal(g, sum(q), case["q_heads"], case["dim"]).to(DTYPES[case["dtype"]])
        s["out"] = torch.empty_like(s["q"])
        s["kv"], s["start"] = _ints(kv), _starts(q)
        s["max_q"], s["max_kv"], s["scale"] = max(q), max(kv), 1 / math.sqrt(case["dim"])
    else:
        s["x"], s["target"] = _logits(case, g)
        n, top = case["rows"], case["top"]
        s |= dict(lp=empty(n, dtype=torch.float32), h=empty(n, dtype=torch.float32), ids=empty(n, top), tops=empty(n, top, dtype=torch.float32))
    if own:
        _describe(s)
    return s


def _describe(s):
    """The descriptors and workspaces that a program makes once."""
    from paper_2505_11076_amd import binding as B

    case, kind = s["case"], s["case"]["kind"]
    dtypes = {"f16": B.F16, "bf16": B.BF16, "f32": B.F32}
    if kind in ("rope", "append"):
        hq, hk, D = case["q_heads"], case["kv_heads"], case["dim"]
        row, at = (hq + 2 * hk) * D, s["qkv"].data_ptr()
        size = s["qkv"].element_size()
        s["heads"] = B.Heads(q=at, q_stride=row, k=at + hq * D * size, k_stride=row, v=at + (hq + hk) * D * size, v_stride=row, q_out=s["q"].data_ptr(),
                             q_out_stride=hq * D, k_out=s["k"].data_ptr() if kind == "rope" else 0, k_out_stride=hk * D, dtype=dtypes[case["dtype"]],
                             n_tokens=case["tokens"], n_q_heads=hq, n_kv_heads=hk, head_dim=D, q_weight=s["w"][0].data_ptr(),
                             k_weight=s["w"][1].data_ptr(), eps=1e-6, rope=s["rope"].data_ptr(), rope_len=s["rope"].shape[0], rot_dim=case["rot"],
                             interleaved=int(case["interleaved"]), positions=s["pos"].data_ptr())
        if kind == "append":
            s["desc"] = B.Cache(data=s["cache"].data_ptr(), n_pages=s["pages"], page_tokens=case["page"], n_kv_heads=hk, head_dim=D)
    elif kind == "attend":
        hq, D = case["q_heads"], case["dim"]
        s["desc"] = B.Cache(data=s["cache"].data_ptr(), n_pages=s["cache"].shape[0], page_tokens=case["page"], n_kv_heads=case["kv_heads"], head_dim=D)
        s["attend"] = B.Attend(q=s["q"].data_ptr(), q_stride=hq * D, out=s["out"].data_ptr(), out_stride=hq * D, dtype=dtypes[case["dtype"]],
                               n_tokens=s["q"].shape[0], n_seq=case["n_seq"], n_q_heads=hq, max_q=s["max_q"], max_kv=s["max_kv"], q_start=s["start"].data_ptr(),
                               kv_len=s["kv"].data_ptr(), block_table=s["table"].data_ptr(), table_stride=s["table"].shape[1], scale=s["scale"], causal=1)
        s["ws"] = _bytes(B.dbf_cache_attend_workspace_bytes(s["attend"], s["desc"]))
    elif kind == "logprobs":
        s["ws"] = _bytes(B.dbf_token_logprobs_workspace_bytes(case["rows"], case["vocab"], case["top"]))
        s["type"] = dtypes[case["dtype"]]


# ---- one pass: the framework's calls -----------------------------------------------------------------------


def _own(s):
    from paper_2505_11076_amd import binding as B

    case, kind, stream = s["case"], s["case"]["kind"], torch.cuda.current_stream().cuda_stream
    if kind == "tables":
        B.dbf_block_tables(s["cached"].data_ptr(), s["new"].data_ptr(), case["n_seq"], case["page"], s["free"].data_ptr(), s["free"].numel(), s["table"].data_ptr(),
                           s["table"].shape[1], s["tokens"], s["start"].data_ptr(), s["kv"].data_ptr(), s["pos"].data_ptr(), s["slots"].data_ptr(),
                           s["status"].data_ptr(), stream)
        return [s["table"], s["start"], s["kv"], s["pos"], s["slots"], s["status"]]
    if kind == "rope":
        B.dbf_qk_norm_rope(s["heads"], stream)
        return [s["q"], s["k"]]
    if kind == "append":
        B.dbf_cache_append(s["heads"], s["desc"], s["slots"].data_ptr(), stream)
        B.dbf_cache_read(s["desc"], s["slots"].data_ptr(), case["tokens"], s["k"].data_ptr(), s["v"].data_ptr(), B.F16, stream)
        return [s["q"], s["k"], s["v"]]
    if kind == "attend":
        B.dbf_cache_attend(s["attend"], s["desc"], s["ws"].data_ptr(), s["ws"].numel(), stream)
        return s["out"]
    B.dbf_token_logprobs(s["x"].data_ptr(), s["type"], case["vocab"], case["rows"], case["vocab"], s["target"].data_ptr(), case["top"], s["lp"].data_ptr(),
                         s["h"].data_ptr(), s["ids"].data_ptr() if case["top"] else 0, s["tops"].data_ptr() if case["top"] else 0, s["ws"].data_ptr(),
                         s["ws"].numel(), stream)
    return [s["lp"], s["h"], s["ids"], s["tops"]]


# ---- one pass: the plain forms -----------------------------------------------------------------------------


def _plain_tables(s):
    case, P = s["case"], s["case"]["page"]
    cached, new, free, table = s["cached"].long(), s["new"].long(), s["free"], s["table"]
    kv, have = cached + new, (cached + P - 1) // P
    need = (kv + P - 1) // P - have
    end, off = new.cumsum(0), need.cumsum(0) - need
    # the new pages' entries, then the tokens'
    r = torch.arange(table.shape[1], device=DEV)
    at = r - have[:, None]
    index = (off[:, None] + at).clamp(0, free.numel() - 1)
    s["table"].copy_(torch.where((at >= 0) & (at < need[:, None]), free[index], table))
    t = torch.arange(s["tokens"], device=DEV)
    seq = torch.searchsorted(end, t, right=True)
    pos = cached[seq] + t - (end - new)[seq]
    slots = s["table"][seq, pos // P].long() * P + pos % P
    start = torch.cat([torch.zeros_like(end[:1]), end])
    status = torch.stack([need.sum(), torch.zeros_like(end[0])])
    return [s["table"]] + [x.to(torch.int32) for x in (start, kv, pos, slots, status)]


def _plain_rope(x, w, rope, pos, case, eps=1e-6):
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w.float()
    rot, half = case["rot"], case["rot"] // 2
    cos, sin = rope[pos.long()].unsqueeze(1).split(half, -1)
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_heads(s):
    case = s["case"]
    q, k, v = s["qkv"].split([case["q_heads"], case["kv_heads"], case["kv_heads"]], 1)
    q, k = (_plain_rope(x, w, s["rope"], s["pos"], case) for x, w in ((q, s["w"][0]), (k, s["w"][1])))
    q = q.to(DTYPES[case["dtype"]])
    if case["kind"] == "rope":
        return [q, k.to(DTYPES[case["dtype"]])]
    return [q] + [_values(*_quantise(x.float())).to(torch.float16) for x in (k, v)]


def _unpack(rec, D):
    """Keys and values [..., 32, D] in 32 bits of records [..., 36 D] of bytes."""
    n = D // GROUP
    kc, vc, kw, vw = rec.split([16 * D, 16 * D, 2 * D, 2 * D], -1)
    kc = torch.stack([kc & 15, kc >> 4], -1).flatten(-2).unflatten(-1, (BLOCK, 4, n, 16))
    vc = vc.unflatten(-1, (n, 4, 16, 2, 2, 4))                          # group, g, lane, q, tile, i
    vc = torch.stack([vc & 15, vc >> 4], -1)
    d = vc.dim() - 7
    vc = vc.permute(*range(d), d + 4, d + 1, d + 5, d + 3, d + 6, d, d + 2).flatten(d, d + 2).flatten(d + 1, d + 2)
    out = []
    for c, w in ((kc, kw), (vc, vw)):
        w = w.contiguous().view(torch.float16).unflatten(-1, (n, BLOCK, 2)).transpose(-2, -3).float()
        out.append((c.float() * w[..., 0][..., None, :, None] + w[..., 1][..., None, :, None]).flatten(-3))
    return out


def _plain_attend(s):
    case = s["case"]
    hq, hk, D, P = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    n, G, table = case["n_seq"], hq // hk, s["table"][:, : -(-s["max_kv"] // P)]
    k, v = _unpack(s["cache"][table.clamp(min=0).long()], D)                # n, pages, heads, blocks, 32, D
    k, v = (x.transpose(1, 2).reshape(n, hk, -1, D) for x in (k, v))
    start, kv = s["start"].long(), s["kv"].long()
    ql = start[1:] - start[:-1]
    t = torch.arange(s["max_q"], device=DEV)
    rows = (start[:-1, None] + t).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float().unflatten(2, (hk, G)).permute(0, 2, 3, 1, 4).reshape(n, hk, -1, D)
    x = torch.matmul(q, k.transpose(2, 3)).view(n, hk, G, s["max_q"], -1) * s["scale"]
    seen = torch.arange(x.shape[-1], device=DEV) <= ((kv - ql)[:, None] + t)[..., None]
    x = x.masked_fill(~seen[:, None, None], float("-inf"))
    x = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e30))
    total = x.sum(-1, keepdim=True)
    x = x / torch.where(total > 0, total, 1)
    v = v.masked_fill((torch.arange(v.shape[2], device=DEV) >= kv[:, None])[:, None, :, None], 0)
    y = torch.matmul(x.view(n, hk, -1, x.shape[-1]), v).view(n, hk, G, s["max_q"], D).permute(0, 3, 1, 2, 4).reshape(n, s["max_q"], hq, D)
    live = (t < ql[:, None]).flatten()
    return y.flatten(0, 1)[live.nonzero()[:, 0]].to(DTYPES[case["dtype"]])


def _plain_logprobs(s):
    x = s["x"].float()
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    lse = (m + torch.log(total))[:, 0]
    lp = x.gather(1, s["target"].long()[:, None])[:, 0] - lse
    h = lse - (e * x).sum(1) / total[:, 0]
    top = s["case"]["top"]
    # the largest by value, then by the lowest index: the values' bits in their order, over the indexes in reverse
    bits = (x + 0.0).view(torch.int32).long()   # (-0 is 0)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 32) - torch.arange(x.shape[1], device=DEV)
    ids = torch.topk(key, top, 1).indices if top else s["ids"].long()
    return [lp, h, ids.to(torch.int32), x.gather(1, ids) - lse[:, None] if top else s["tops"]]


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    if kind == "tables":
        return _plain_tables(s)
    if kind in ("rope", "append"):
        return _plain_heads(s)
    return _plain_attend(s) if kind == "attend" else _plain_logprobs(s)


# ---- what a pass cannot do without --------------------------------------------------------------------------


def work(case):
    kind = case["kind"]
    if kind == "tables":
        cached, new = _lengths(case)
        P = case["page"]
        pages = sum(_pages([c + n for c, n in zip(cached, new)], P)) - sum(_pages(cached, P))
        return dict(bytes=8 * case["n_seq"] + 8 * pages + 8 * sum(new) + 8 * case["n_seq"] + 12, flops=0)
    if kind == "logprobs":
        e = case["rows"] * case["vocab"]
        size = 4 if case["dtype"] == "f32" else 2
        return dict(bytes=e * size + case["rows"] * (12 + 8 * case["top"]), flops=4 * e)
    hq, hk, D = case["q_heads"], case["kv_heads"], case["dim"]
    if kind in ("rope", "append"):
        T = case["tokens"]
        common = T * (4 + 4 * case["rot"]) + 4 * D
        if kind == "rope":
            return dict(bytes=common + T * (hq + hk) * D * 4, flops=T * (hq + hk) * D * 8)
        # (the written values come back as fp16)
        return dict(bytes=common + T * (hq * 4 + hk * 2 * (2 + 2 * 36 / 64 + 2)) * D + 4 * T, flops=T * (hq + 3 * hk) * D * 8)
    kv, q = _lengths(case)
    pairs = sum(b * (2 * a - b + 1) // 2 for a, b in zip(kv, q))
    return dict(bytes=sum(kv) * hk * D * 2 * 36 / 64 + sum(q) * hq * D * 4 + 4 * sum(_pages(kv, case["page"])) + 8 * case["n_seq"], flops=4.0 * pairs * hq * D)


# ---- the same in 64 bits ------------------------------------------------------------------------------------


def _exact_turn(x, w, case, pos):
    x = x.double()
    x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + 1e-6) * w.double()
    rot = case["rot"]
    table = _rope_table(case["tokens"] + 100, rot).double()[pos.long()]
    turn = torch.complex(table[:, : rot // 2], table[:, rot // 2:])[:, None]
    if case["interleaved"]:
        y = torch.view_as_real(torch.view_as_complex(x[..., :rot].reshape(*x.shape[:2], -1, 2).contiguous()) * turn).reshape(*x.shape[:2], rot)
    else:
        c = torch.complex(x[..., : rot // 2].contiguous(), x[..., rot // 2: rot].contiguous()) * turn
        y = torch.cat([c.real, c.imag], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _exact_held(x):
    """What the cache holds of x [T, heads, D], group by group."""
    x = x.double()
    out, n = torch.zeros_like(x), x.shape[-1] // GROUP
    for p in range(n):
        dims = [d for d in range(x.shape[-1]) if d // 16 % n == p]
        y = x[..., dims]
        lo, hi = y.amin(-1, keepdim=True).clamp(max=0), y.amax(-1, keepdim=True).clamp(min=0)
        m, e = np.frexp(((hi - lo).cpu().numpy()) / 15)
        s = np.ceil(np.ldexp(np.ceil(np.ldexp(m, 7)), e - 7 + 24))
        s = torch.from_numpy(np.ldexp(s, -24)).to(DEV)
        safe = torch.where(s > 0, s, 1)
        z = torch.round(-lo / safe)
        out[..., dims] = s * ((torch.round(y / safe) + z).clamp(0, 15) - z)
    return out


def exact(case, seed):
    g, kind = _rng(seed), case["kind"]
    if kind == "tables":
        _, _, free, table = (x.cpu().tolist() for x in _tables_inputs(case, g))
        cached, new = _lengths(case)
        P, taken, start, pos, slots = case["page"], 0, [0], [], []
        for i, (c, n) in enumerate(zip(cached, new)):
            for t in range(c, c + n):
                if t % P == 0:
                    table[i][t // P] = free[taken]
                    taken += 1
                pos.append(t)
                slots.append(table[i][t // P] * P + t % P)
            start.append(start[-1] + n)
        return [_ints(v) for v in (table, start, [c + n for c, n in zip(cached, new)], pos, slots, [taken, 0])]
    if kind in ("rope", "append"):
        qkv, w, pos = _heads(case, g)
        hq, hk = case["q_heads"], case["kv_heads"]
        q, k = _exact_turn(qkv[:, :hq], w[0], case, pos), _exact_turn(qkv[:, hq: hq + hk], w[1], case, pos)
        return [q, k] if kind == "rope" else [q, _exact_held(k), _exact_held(qkv[:, hq + hk:])]
    if kind == "attend":
        (kc, ks, kz), (vc, vs, vz), table = _cache(case, g)
        kv, ql = _lengths(case)
        hq, hk, D, P = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
        q = _normal(g, sum(ql), hq, D).to(DTYPES[case["dtype"]]).double()
        out, at = [], 0
        for i in range(case["n_seq"]):
            pages = table[i, : -(-kv[i] // P)].long()
            rows, n = q[at: at + ql[i]], kv[i]
            at += ql[i]
            heads = []
            for h in range(hk):
                K, V = ((s[pages, h].double() * (c[pages, h].double() - z[pages, h].double())).reshape(-1, D)[:n] for c, s, z in ((kc, ks, kz), (vc, vs, vz)))
                x = rows[:, h * (hq // hk): (h + 1) * (hq // hk)] @ K.T / math.sqrt(D)
                last = n - ql[i] + torch.arange(ql[i], device=DEV)
                x = x.masked_fill((torch.arange(n, device=DEV) > last[:, None])[:, None], float("-inf"))
                heads.append(torch.softmax(x, -1) @ V)
            out.append(torch.cat(heads, 1))
        return torch.cat(out)
    x, target = _logits(case, g)
    x = x.double()
    lp = torch.log_softmax(x, 1)
    h = -(lp.exp() * lp).sum(1)
    ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, : case["top"]]
    return [lp.gather(1, target.long()[:, None])[:, 0], h, ids.to(torch.int32), lp.gather(1, ids)]
