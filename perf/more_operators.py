"""Products with weights that are not DBF layers, as cases: a router's choice of experts, the rounding of activations to 8 bits, products in 8 bits with a scale
for each block of 128 (and in 16 bits), the same by experts with ragged numbers of rows, and the weighted sum that brings experts' rows back to their tokens.

`run` is one call as a serving program makes it (`own`), or the same in elementary torch operations in 32 bits (a router's scores in 64: places in an order hang on
them).  `exact` is the operator's definition in 64 bits, from the inputs as they were made.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 128
E4M3_MOST = 448.0


# ---- cases -------------------------------------------------------------------------------------------------


def listed():
    return [
        # the next token of one request: 64 experts, 6 of them
        dict(name="route_token", kind="route", tokens=1, experts=64, top=6, score="softmax", bias=False, dtype="f32", padded=0),
        # a prompt, many experts, chosen with a bias that evens their loads out; the batch is padded
        dict(name="route_prompt", kind="route", tokens=8191, experts=256, top=8, score="sigmoid", bias=True, dtype="f32", padded=100),
        # a decode step's activations
        dict(name="quantize_token", kind="quantize", rows=7, cols=4096, rows_of_block=1, dtype="f16"),
        # a prompt's, the wide side of an MLP
        dict(name="quantize_prompt", kind="quantize", rows=8191, cols=11008, rows_of_block=1, dtype="bf16"),
        # one token through a square layer
        dict(name="product_token", kind="product", rows=1, n_in=4096, n_out=4096, gated=False, dtype="e4m3", scale="e8m0", out="f16"),
        # a decode batch's logits: the head, which stays uncompressed, with scales of 32 bits as weights come with
        dict(name="product_head", kind="product", rows=13, n_in=4096, n_out=128256, gated=False, dtype="e4m3", scale="f32", out="f16"),
        # a prompt through the gate and up layers of an MLP
        dict(name="product_prompt", kind="product", rows=2047, n_in=4096, n_out=11008, gated=True, dtype="e4m3", scale="e8m0", out="bf16"),
        # a decode batch of 8 tokens, 8 experts each, of 64: some experts have none
        dict(name="experts_decode", kind="experts", tokens=8, top=8, experts=64, n_in=2048, n_out=1024, gathered=True, gated=True, dtype="e4m3", scale="e8m0", out="bf16"),
        # a prompt through the gate and up layers of its experts, rows gathered from its tokens
        dict(name="experts_prompt", kind="experts", tokens=4096, top=4, experts=32, n_in=4096, n_out=2048, gathered=True, gated=True, dtype="e4m3", scale="f32", out="bf16"),
        # the way down of small experts that were left in 16 bits, odd sizes
        dict(name="experts_16bit", kind="experts", tokens=1021, top=6, experts=60, n_in=1000, n_out=2047, gathered=False, gated=False, dtype="bf16", scale="none", out="bf16"),
        # a decode batch's rows back to its tokens
        dict(name="combine_decode", kind="combine", tokens=8, top=8, cols=2048, residual=True, dtype="bf16", dropped=0.0),
        # a prompt's, some choices without a row
        dict(name="combine_prompt", kind="combine", tokens=4095, top=4, cols=4096, residual=True, dtype="f16", dropped=0.01),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "quantize", "product", "product", "product", "experts", "experts", "experts", "combine"])
    if kind == "route":
        experts = rng.choice([8, 16, 33, 60, 64, 128, 160, 256])
        tokens = _log(rng, 1, 8191)
        return dict(kind=kind, tokens=tokens, experts=experts, top=rng.choice([1, 2, 4, 6, 8]), score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5,
                    dtype=rng.choice(["f16", "bf16", "f32"]), padded=rng.randint(0, tokens // 8))
    if kind == "quantize":
        cols = _log(rng, 64, 16384)
        return dict(kind=kind, rows=_log(rng, 1, min(16384, 90000000 // cols)), cols=cols, rows_of_block=rng.choice([1, 1, 128]), dtype=rng.choice(["f16", "bf16", "f32"]))
    if kind == "combine":
        cols = _log(rng, 64, 8192)
        top = rng.choice([1, 2, 4, 6, 8])
        return dict(kind=kind, tokens=_log(rng, 1, min(8192, 60000000 // (cols * top))), top=top, cols=cols, residual=rng.random() < 0.5,
                    dtype=rng.choice(["f16", "bf16", "f32"]), dropped=rng.choice([0.0, 0.0, 0.1]))
    dtype = rng.choice(["e4m3", "e4m3", "e4m3", "f16", "bf16"])
    c = dict(kind=kind, n_in=_log(rng, 64, 11008), gated=rng.random() < 0.5, dtype=dtype, scale=rng.choice(["e8m0", "f32"]) if dtype == "e4m3" else "none",
             out=rng.choice(["f16", "bf16", "f32"]))
    if kind == "product":
        c |= dict(rows=_log(rng, 1, 2048), n_out=_log(rng, 64, 32000))
    else:
        c |= dict(tokens=_log(rng, 1, 4096), top=rng.choice([1, 2, 4, 6, 8]), experts=rng.choice([8, 16, 32, 60, 64]), n_out=_log(rng, 64, 4096), gathered=rng.random() < 0.5)
    # (no more bytes and products than the largest of the listed ones have)
    while work(c)["bytes"] > 6.0e8 or work(c)["flops"] > 5.0e11:
        if c.get("tokens", c.get("rows")) > 64:
            c["tokens" if kind == "experts" else "rows"] //= 2
        else:
            c["n_out"] = max(64, c["n_out"] * 3 // 4)
    return c


def _case_rng(case):
    return np.random.default_rng(abs(int.from_bytes(",".join("%s=%s" % kv for kv in sorted(case.items()) if kv[0] != "name").encode(), "little")) % (1 << 63))


def _choices(case):
    """The experts [tokens][top] of a case's tokens, the same for every seed: some experts are liked more than others."""
    rng = _case_rng(case)
    score = rng.gumbel(size=(case["tokens"], case["experts"])) + 0.7 * rng.normal(size=case["experts"])
    return np.argsort(-score, 1, kind="stable")[:, : case["top"]]


def _sizes(case):
    """Rows of each expert."""
    return np.bincount(_choices(case).reshape(-1), minlength=case["experts"])


# ---- inputs ------------------------------------------------------------------------------------------------


def _rng(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _up(n, to):
    return -(-n // to) * to


def _activations(g, rows, cols):
    """Values of a few loud channels and rows of different sizes."""
    return _normal(g, rows, cols) * torch.exp(0.7 * _normal(g, cols)) * torch.exp(0.5 * _normal(g, rows, 1))


def _pow2(e):
    """2^e of whole e in 64 bits, by its bits: powers and exponentials need not be exact."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _blocks(x, rows_of_block):
    """x [rows][cols] filled up with zeros to whole blocks, [row blocks][rows of a block][column blocks][128]."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, _up(cols, BLOCK) - cols, 0, _up(rows, rows_of_block) - rows))
    return x.view(-1, rows_of_block, x.shape[1] // BLOCK, BLOCK)


def _quantise(x, rows_of_block):
    """(codes as float8, bytes of the scales): a block's scale is the smallest 2^(byte - 127) that leaves no value above 448; of zeros 1."""
    rows, cols = x.shape
    b = _blocks(x.float(), rows_of_block)
    most = b.abs().amax((1, 3), keepdim=True)
    m, e = torch.frexp(most)                                   # m 2^e, m in [1/2, 1); 448 is 7/8 of 2^9
    e = torch.where(most > 0, (e - 9 + (m > 0.875)).clamp(-127, 127), 0)
    fine = torch.isfinite(most)
    q = torch.where(fine, b, 0) * _pow2(-e).float()
    codes = torch.where(fine, q, float("nan")).flatten(2).flatten(0, 1)[:rows, :cols].to(torch.float8_e4m3fn)
    return codes.contiguous(), (torch.where(fine, e, 0) + 127)[:, 0, :, 0].to(torch.uint8).contiguous()


def _weights(g, n, k, dtype, scale):
    """A layer's weights [n][k] and the scales of its blocks."""
    if dtype != "e4m3":
        return (_normal(g, n, k) / math.sqrt(k)).to(DTYPES[dtype]), None
    codes, scales = [], []
    for at in range(0, n, 16384):
        w = _normal(g, min(16384, n - at), k) / math.sqrt(k)
        if scale == "e8m0":
            c, s = _quantise(w, BLOCK)
        else:
            b = _blocks(w, BLOCK)
            s = b.abs().amax((1, 3), keepdim=True) / E4M3_MOST
            c = (b / s).flatten(2).flatten(0, 1)[: w.shape[0], :k].to(torch.float8_e4m3fn)
            s = s[:, 0, :, 0]
        codes.append(c)
        scales.append(s)
    return torch.cat(codes), torch.cat(scales).contiguous()


def _padded(x, size):
    """Rows of x at a stride of whole 16 bytes."""
    stride = _up(x.shape[-1], 16 // size)
    if stride == x.shape[-1]:
        return x.contiguous()
    y = torch.zeros(*x.shape[:-1], stride, dtype=x.dtype, device=DEV)
    y.view(torch.uint8 if size == 1 else torch.int16)[..., : x.shape[-1]] = x.view(torch.uint8 if size == 1 else torch.int16)
    return y


def prepare(case, seed):
    g, kind = _rng(seed), case["kind"]
    s = dict(case=case)
    empty = lambda *shape, dtype=torch.int32: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    if kind == "route":
        T, E, n = case["tokens"], case["experts"], case["top"]
        x = 1.5 * _normal(g, T, E) + _normal(g, E)
        x[torch.rand(T, E, generator=g, device=DEV) < 0.001] = float("-inf")     # (experts that a token may not have)
        x[T - case["padded"]:] = float("-inf")                                   # (rows of the batch that hold no token)
        s["x"] = x.to(DTYPES[case["dtype"]])
        s["bias"] = 0.1 * _normal(g, E) if case["bias"] else None
        s |= dict(ids=empty(T, n), weights=empty(T, n, dtype=torch.float32), starts=empty(E + 1), row_token=empty(T * n), token_rows=empty(T, n))
    elif kind == "quantize":
        rows, cols, R = case["rows"], case["cols"], case["rows_of_block"]
        s["x"] = _activations(g, rows, cols).to(DTYPES[case["dtype"]])
        s["codes"] = empty(rows, _up(cols, 16), dtype=torch.float8_e4m3fn)
        s["scales"] = empty(-(-rows // R), _up(-(-cols // BLOCK), 4), dtype=torch.uint8)
    elif kind == "combine":
        T, n, cols, dt = case["tokens"], case["top"], case["cols"], DTYPES[case["dtype"]]
        at = torch.randperm(T * n, generator=g, device=DEV).view(T, n)
        s["rows"] = _normal(g, T * n, cols).to(dt)
        s["token_rows"] = torch.where(torch.rand(T, n, generator=g, device=DEV) < case["dropped"], -1, at).to(torch.int32)
        s["weights"] = torch.rand(T, n, generator=g, device=DEV) / n
        s["residual"] = _normal(g, T, cols).to(dt) if case["residual"] else None
        s["out"] = torch.empty(T, cols, dtype=dt, device=DEV)
    else:
        _product_inputs(s, g)
    if own:
        _describe(s)
    return s


def _product_inputs(s, g):
    case = s["case"]
    n, k, dtype = case["n_out"], case["n_in"], case["dtype"]
    size = 1 if dtype == "e4m3" else 2
    rows, groups = case.get("rows"), 1
    if case["kind"] == "experts":
        each, groups = _sizes(case), case["experts"]
        rows = int(each.sum())
        s["sizes"] = [int(m) for m in each]
        s["starts"] = torch.tensor([0] + list(np.cumsum(each)), dtype=torch.int32, device=DEV)
        if case["gathered"]:
            order = np.argsort(_choices(case).reshape(-1), kind="stable")
            s["x_rows"] = torch.from_numpy((order // case["top"]).astype(np.int32)).to(DEV)
    x = _activations(g, case["tokens"] if case.get("gathered") else rows, k)
    if dtype == "e4m3":
        codes, scales = _quantise(x, 1)
        s["x"] = _padded(codes, 1)
        s["x_scale"] = torch.nn.functional.pad(scales, (0, _up(scales.shape[1], 4) - scales.shape[1])).contiguous()
    else:
        s["x"] = _padded(x.to(DTYPES[dtype]), 2)
    # (weights of all experts, gate and up apart)
    for name in ("w", "w_up") if case["gated"] else ("w",):
        s[name] = torch.zeros(groups, n, _up(k, 16 // size), dtype=torch.float8_e4m3fn if size == 1 else DTYPES[dtype], device=DEV)
        if dtype == "e4m3":
            s[name + "_scale"] = torch.empty(groups, -(-n // BLOCK), -(-k // BLOCK), dtype=torch.uint8 if case["scale"] == "e8m0" else torch.float32, device=DEV)
        for i in range(groups):
            w, scale = _weights(g, n, k, dtype, case["scale"])
            s[name][i] = _padded(w, size)
            if scale is not None:
                s[name + "_scale"][i] = scale
    s["y"] = torch.empty(rows, n, dtype=DTYPES[case["out"]], device=DEV)


def _bytes(n):
    return torch.empty(max(int(n), 256), dtype=torch.uint8, device=DEV)


def _address(t):
    return 0 if t is None else t.data_ptr()


def _describe(s):
    """The descriptors and workspaces that a program makes once."""
    from paper_2505_11076_amd import binding as B

    case, kind = s["case"], s["case"]["kind"]
    dtypes = {"f16": B.F16, "bf16": B.BF16, "f32": B.F32, "e4m3": B.E4M3, "e8m0": B.E8M0, "none": 0}
    if kind == "route":
        s["desc"] = B.Router(logits=s["x"].data_ptr(), row_stride=case["experts"], bias=_address(s["bias"]), dtype=dtypes[case["dtype"]], n_tokens=case["tokens"],
                             n_experts=case["experts"], n_top=case["top"], score=B.SCORE_SIGMOID if case["score"] == "sigmoid" else B.SCORE_SOFTMAX, renormalise=1, scale=1.0,
                             expert_ids=s["ids"].data_ptr(), weights=s["weights"].data_ptr(), starts=s["starts"].data_ptr(), row_token=s["row_token"].data_ptr(),
                             token_rows=s["token_rows"].data_ptr())
        s["ws"] = _bytes(B.dbf_route_workspace_bytes(s["desc"]))
    elif kind in ("product", "experts"):
        s["desc"] = B.Dense(x=s["x"].data_ptr(), x_stride=s["x"].shape[1], x_scale=_address(s.get("x_scale")), x_scale_stride=s["x_scale"].shape[1] if "x_scale" in s else 0,
                            n_x_rows=s["x"].shape[0], x_rows=_address(s.get("x_rows")), w=s["w"].data_ptr(), w_stride=s["w"].shape[2], w_group_stride=s["w"].stride(0),
                            w_scale=_address(s.get("w_scale")), w_scale_stride=-(-case["n_in"] // BLOCK), w_scale_group_stride=-(-case["n_in"] // BLOCK) * -(-case["n_out"] // BLOCK),
                            w_scale_type=dtypes[case["scale"]], w_up=_address(s.get("w_up")), w_up_scale=_address(s.get("w_up_scale")), y=s["y"].data_ptr(), y_stride=case["n_out"],
                            dtype=dtypes[case["dtype"]], out_dtype=dtypes[case["out"]], n_rows=s["y"].shape[0], n_in=case["n_in"], n_out=case["n_out"],
                            n_groups=case.get("experts", 0), starts=_address(s.get("starts")))
        size = B.dbf_grouped_gemm_workspace_bytes if kind == "experts" else B.dbf_dense_gemm_workspace_bytes
        s["ws"] = _bytes(size(s["desc"]))
    elif kind == "combine":
        s["desc"] = B.Combine(rows=s["rows"].data_ptr(), row_stride=case["cols"], n_rows=s["rows"].shape[0], token_rows=s["token_rows"].data_ptr(), weights=s["weights"].data_ptr(),
                              residual=_address(s["residual"]), residual_stride=case["cols"], out=s["out"].data_ptr(), out_stride=case["cols"], dtype=dtypes[case["dtype"]],
                              n_tokens=case["tokens"], n_top=case["top"], n_cols=case["cols"])
    else:
        s["type"] = dtypes[case["dtype"]]


# ---- one pass: the framework's calls -----------------------------------------------------------------------


def _own(s):
    from paper_2505_11076_amd import binding as B

    case, kind, stream = s["case"], s["case"]["kind"], torch.cuda.current_stream().cuda_stream
    if kind == "route":
        B.dbf_route(s["desc"], s["ws"].data_ptr(), s["ws"].numel(), stream)
        return [s["ids"], s["weights"], s["starts"], s["row_token"], s["token_rows"]]
    if kind == "quantize":
        B.dbf_quantize(s["x"].data_ptr(), s["type"], case["cols"], case["rows"], case["cols"], case["rows_of_block"], s["codes"].data_ptr(), s["codes"].shape[1],
                           s["scales"].data_ptr(), s["scales"].shape[1], stream)
        return [s["codes"][:, : case["cols"]], s["scales"][:, : -(-case["cols"] // BLOCK)]]
    if kind == "combine":
        B.dbf_combine(s["desc"], stream)
        return s["out"]
    if kind == "product":
        B.dbf_dense_gemm(s["desc"], s["ws"].data_ptr(), s["ws"].numel(), stream)
    else:
        B.dbf_grouped_gemm(s["desc"], s["ws"].data_ptr(), s["ws"].numel(), stream)
    return s["y"]


# ---- one pass: the plain forms -----------------------------------------------------------------------------


def _plain_route(s):
    case = s["case"]
    E, n, x = case["experts"], case["top"], s["x"].double()
    none = float("-inf")
    x = torch.where(torch.isnan(x), none, x)
    if case["score"] == "sigmoid":
        score = 1 / (1 + torch.exp(-x))
    else:
        e = torch.exp(x - x.amax(1, keepdim=True).clamp(min=-1e300))
        total = e.sum(1, keepdim=True)
        score = e / torch.where(total > 0, total, 1)
    by = x if s["bias"] is None else torch.where(x > none, score + s["bias"].double(), none)
    by, ids = torch.sort(by, dim=1, descending=True, stable=True)       # (ties to the lowest index)
    live, ids = by[:, :n] > none, ids[:, :n]
    w = torch.where(live, score.gather(1, ids), 0)
    total = w.sum(1, keepdim=True)
    w = (w / torch.where(total > 0, total, 1)).float()
    expert = torch.where(live, ids, E).flatten()
    expert, order = torch.sort(expert, dim=0, stable=True)
    starts = torch.searchsorted(expert, torch.arange(E + 1, device=DEV))
    token_rows = torch.empty_like(order)
    token_rows[order] = torch.arange(order.numel(), device=DEV)
    row_token = torch.where(expert < E, order // n, -1)
    out = [torch.where(live, ids, -1), w, starts, row_token, torch.where(live, token_rows.view(-1, n), -1)]
    return [t if t.dtype == torch.float32 else t.to(torch.int32) for t in out]


def _plain_weights(s, name, i):
    """Weights of group i in 32 bits."""
    k = s["case"]["n_in"]
    w = s[name][i][:, :k].float()
    if name + "_scale" not in s:
        return w
    scale = s[name + "_scale"][i]
    scale = _pow2(scale.long() - 127).float() if scale.dtype == torch.uint8 else scale
    return w * scale.repeat_interleave(BLOCK, 0)[: w.shape[0]].repeat_interleave(BLOCK, 1)[:, :k]


def _plain_product(s):
    case = s["case"]
    k = case["n_in"]
    x = s["x"][:, :k].float()
    if "x_scale" in s:
        x = x * _pow2(s["x_scale"].long() - 127).float().repeat_interleave(BLOCK, 1)[:, :k]
    if "x_rows" in s:
        x = x[s["x_rows"].long()]
    out = []
    for i, part in enumerate(x.split(s["sizes"]) if "sizes" in s else [x]):
        if not part.shape[0]:
            continue
        y = torch.matmul(part, _plain_weights(s, "w", i).t())
        if case["gated"]:
            y = y / (1 + torch.exp(-y)) * torch.matmul(part, _plain_weights(s, "w_up", i).t())
        out.append(y.to(DTYPES[case["out"]]))
    return torch.cat(out)


def _plain_combine(s):
    at = s["token_rows"].long()
    y = s["residual"].float() if s["residual"] is not None else torch.zeros(s["out"].shape, device=DEV)
    for j in range(s["case"]["top"]):
        row = s["rows"][at[:, j].clamp(min=0)].float()
        y = y + torch.where(at[:, j, None] >= 0, s["weights"][:, j, None] * row, 0)
    return y.to(s["out"].dtype)


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    if kind == "route":
        return _plain_route(s)
    if kind == "quantize":
        return list(_quantise(s["x"], s["case"]["rows_of_block"]))
    return _plain_combine(s) if kind == "combine" else _plain_product(s)


# ---- what a pass cannot do without --------------------------------------------------------------------------


def work(case):
    kind = case["kind"]
    size = {"f16": 2, "bf16": 2, "f32": 4, "e4m3": 1}[case["dtype"]]
    if kind == "route":
        e, n = case["tokens"] * case["experts"], case["tokens"] * case["top"]
        return dict(bytes=e * size + 16 * n + 4 * case["experts"], flops=10 * e)
    if kind == "quantize":
        e = case["rows"] * case["cols"]
        return dict(bytes=e * (size + 1) + e // (BLOCK * case["rows_of_block"]), flops=2 * e)
    if kind == "combine":
        e = case["tokens"] * case["cols"]
        return dict(bytes=e * size * (case["top"] + 1 + case["residual"]) + 8 * case["tokens"] * case["top"], flops=2 * e * case["top"])
    k, n, gates = case["n_in"], case["n_out"], 2 if case["gated"] else 1
    rows, used, x_rows = case.get("rows"), 1, case.get("rows")
    if kind == "experts":
        each = _sizes(case)
        rows, used = int(each.sum()), int((each > 0).sum())
        x_rows = case["tokens"] if case["gathered"] else rows
    scales = 0
    if case["dtype"] == "e4m3":
        blocks = -(-k // BLOCK)
        scales = x_rows * blocks + used * gates * blocks * -(-n // BLOCK) * (4 if case["scale"] == "f32" else 1)
    out = {"f16": 2, "bf16": 2, "f32": 4}[case["out"]]
    return dict(bytes=(x_rows + used * gates * n) * k * size + scales + rows * n * out, flops=2.0 * rows * n * k * gates)


# ---- the definition in 64 bits -----------------------------------------------------------------------------


def _e4m3_table():
    """The value of each code: sign, 4 bits of exponent (bias 7), 3 of mantissa; exponent 0 without the leading one; all ones is no number."""
    out = []
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = float("nan") if c & 127 == 127 else math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        out.append(-v if c > 127 else v)
    return torch.tensor(out, dtype=torch.float64, device=DEV)


def _exact_values(codes, cols):
    """Rows of codes or of 16-bit values, in 64 bits."""
    if codes.dtype != torch.float8_e4m3fn:
        return codes[:, :cols].double()
    return _e4m3_table()[codes.view(torch.uint8)[:, :cols].int()]


def _exact_scales(scale):
    return torch.from_numpy(np.ldexp(1.0, scale.cpu().numpy().astype(np.int64) - 127)).to(DEV) if scale.dtype == torch.uint8 else scale.double()


def _exact_route(s):
    case = s["case"]
    x, n, E = s["x"].double().cpu().numpy(), case["top"], case["experts"]
    bias = None if s["bias"] is None else s["bias"].double().cpu().numpy()
    ids, weights = np.full((len(x), n), -1), np.zeros((len(x), n))
    members = [[] for _ in range(E)]
    for t, row in enumerate(x):
        able = np.flatnonzero(row > -np.inf)
        if not len(able):
            continue
        v = row[able]
        if case["score"] == "sigmoid":
            p = np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))
        else:
            p = np.exp(v - v.max())
            p /= p.sum()
        rank = v if bias is None else p + bias[able]
        take = np.lexsort((able, -rank))[:n]
        ids[t, : len(take)] = able[take]
        weights[t, : len(take)] = p[take] / p[take].sum()
        for j, e in enumerate(able[take]):
            members[e].append((t, j))
    starts = np.concatenate([[0], np.cumsum([len(m) for m in members])])
    row_token, token_rows = np.full(ids.size, -1), np.full(ids.shape, -1)
    for r, (t, j) in enumerate(m for part in members for m in part):
        row_token[r] = t
        token_rows[t, j] = r
    return [torch.from_numpy(a) for a in (ids, weights, starts, row_token, token_rows)]


def _exact_quantize(s):
    case = s["case"]
    rows, cols, R = case["rows"], case["cols"], case["rows_of_block"]
    codes = torch.empty(rows, cols, dtype=torch.float64, device=DEV)
    scales = []
    for r in range(0, rows, 1024):
        part, here = s["x"][r: r + 1024].double(), []
        for c in range(0, cols, BLOCK):
            x = part[:, c: c + BLOCK]
            most = torch.cat([a.abs().max().view(1) for a in x.split(R)]) if R > 1 else x.abs().amax(1)
            # the smallest power of two that is at least most / 448: by its neighbours, whatever the logarithm's last bit is
            e = torch.ceil(torch.log2(torch.where(most > 0, most, 448.0) / 448)).clamp(-127, 127)
            pow2 = lambda e: torch.from_numpy(np.ldexp(1.0, e.cpu().numpy().astype(np.int64))).to(DEV)  # noqa: E731
            e = torch.where(most > 448 * pow2(e), e + 1, e)
            e = torch.where((most > 0) & (most <= 448 * pow2(e - 1)), e - 1, e).clamp(min=-127)
            here.append(e + 127)
            y = x / pow2(e).repeat_interleave(R)[: x.shape[0], None]
            step = pow2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20))).clamp(min=-6) - 3)
            codes[r: r + 1024, c: c + BLOCK] = torch.round(y / step) * step
        scales.append(torch.stack(here, 1))
    return [codes, torch.cat(scales)]


def _exact_product(s):
    case = s["case"]
    k, n = case["n_in"], case["n_out"]
    x = _exact_values(s["x"], k)
    if "x_scale" in s:
        x = x * _exact_scales(s["x_scale"]).repeat_interleave(BLOCK, 1)[:, :k]
    if "x_rows" in s:
        x = x[s["x_rows"].long()]
    y = torch.empty(x.shape[0], n, dtype=torch.float64, device=DEV)
    at = 0
    for i, m in enumerate(s.get("sizes", [x.shape[0]])):
        for c in range(0, n if m else 0, 64 * BLOCK):
            parts = []
            for name in ("w", "w_up") if case["gated"] else ("w",):
                w = _exact_values(s[name][i][c: c + 64 * BLOCK], k)
                if name + "_scale" in s:
                    scale = _exact_scales(s[name + "_scale"][i][c // BLOCK: c // BLOCK + 64])
                    w = w * scale.repeat_interleave(BLOCK, 0)[: w.shape[0]].repeat_interleave(BLOCK, 1)[:, :k]
                parts.append(x[at: at + m] @ w.T.contiguous())
            y[at: at + m, c: c + 64 * BLOCK] = parts[0] * torch.sigmoid(parts[0]) * parts[1] if case["gated"] else parts[0]
        at += m
    return y


def _exact_combine(s):
    at, w = s["token_rows"].cpu(), s["weights"].double()
    y = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV) if s["residual"] is None else s["residual"].double()
    for j in range(at.shape[1]):
        have = (at[:, j] >= 0).nonzero()[:, 0].to(DEV)
        y[have] += s["rows"][s["token_rows"][have, j].long()].double() * w[have, j][:, None]
    return y


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return dict(route=_exact_route, quantize=_exact_quantize, combine=_exact_combine).get(case["kind"], _exact_product)(s)
