"""Oracle of products with ordinary weights, in numpy and 64 bits: the type in 8 bits and its scales, products of one matrix or by groups, a router's choice and order, the sum that
brings rows back.  Written from the definitions in include/dbf.h, by loops where those are plainer."""
import math

import numpy as np

BLOCK, MOST = 128, 448.0


def _table():
    out = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = math.nan if c & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = -v if c & 128 else v
    return out


E4M3 = _table()


def encode(v):
    """The code nearest to each value (at most 448 in size), ties to the even code."""
    v = np.asarray(v, np.float64)
    values = E4M3[:127]                                   # 0 .. 448, ascending
    a = np.abs(v)
    hi = np.clip(np.searchsorted(values, a), 0, 126)      # the first that is at least a
    lo = np.maximum(hi - 1, 0)
    up, down = values[hi] - a, a - values[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code + np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def scale_byte(most):
    """The smallest b >= 0 with most <= 448 * 2^(b - 127); 127 for 0."""
    if most == 0:
        return 127
    b = 0
    while most > math.ldexp(MOST, b - 127):
        b += 1
    return b


def quantize(x, block_rows):
    """(codes, scale bytes) of x [rows][cols]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    codes = np.zeros((rows, cols), np.uint8)
    scales = np.zeros((-(-rows // block_rows), -(-cols // BLOCK)), np.uint8)
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            at = np.s_[i * block_rows: (i + 1) * block_rows, j * BLOCK: (j + 1) * BLOCK]
            if not np.all(np.isfinite(x[at])):
                codes[at], scales[i, j] = 0x7F, 127
                continue
            b = scale_byte(float(np.max(np.abs(x[at]))))
            codes[at], scales[i, j] = encode(x[at] * math.ldexp(1.0, 127 - b)), b
    return codes, scales


def scales_of(s):
    """Numbers that scales stand for: bytes 2^(b - 127) (255: no number), or themselves."""
    s = np.asarray(s)
    return np.where(s == 255, np.nan, np.ldexp(1.0, s.astype(np.int64) - 127)) if s.dtype == np.uint8 else s.astype(np.float64)


def values(codes, scales, block_rows):
    """What codes with scales stand for."""
    v = E4M3[codes]
    s = np.repeat(np.repeat(scales_of(scales), block_rows, 0)[: v.shape[0]], BLOCK, 1)[:, : v.shape[1]]
    return v * s


def silu(g):
    return g / (1 + np.exp(-g))


def route(logits, n_top, sigmoid, bias=None, renormalise=True, scale=1.0):
    """(ids, weights, starts, row_token, token_rows) by loops."""
    T, E = logits.shape
    ids, weights = np.full((T, n_top), -1), np.zeros((T, n_top))
    rows_of = [[] for _ in range(E)]
    for t in range(T):
        x = [float(v) for v in logits[t]]
        live = [e for e in range(E) if x[e] > -math.inf]
        top = max((x[e] for e in live), default=0.0)
        if sigmoid:
            s = {e: 1 / (1 + math.exp(-x[e])) if x[e] > -700 else 0.0 for e in live}
        else:
            s = {e: 1.0 if x[e] == top else math.exp(x[e] - top) if x[e] - top > -740 else 0.0 for e in live}
            total = sum(s.values())
            s = {e: v / total for e, v in s.items()}
        by = {e: x[e] if bias is None else s[e] + float(bias[e]) for e in live}
        order = sorted((e for e in live if by[e] > -math.inf), key=lambda e: (-by[e], e))[:n_top]
        chosen = sum(s[e] for e in order)
        for j, e in enumerate(order):
            ids[t, j] = e
            weights[t, j] = scale * (s[e] / chosen if renormalise and chosen > 0 else 0.0 if renormalise else s[e])
            rows_of[e].append((t, j))
    starts = np.concatenate([[0], np.cumsum([len(r) for r in rows_of])])
    row_token, token_rows = np.full(T * n_top, -1), np.full((T, n_top), -1)
    for r, (t, j) in enumerate(p for part in rows_of for p in part):
        row_token[r], token_rows[t, j] = t, r
    return ids, weights, starts, row_token, token_rows


def combine(rows, token_rows, weights, residual=None):
    out = np.zeros((len(token_rows), rows.shape[1])) if residual is None else np.array(residual, np.float64)
    for t, at in enumerate(token_rows):
        for j, r in enumerate(at):
            if 0 <= r < len(rows):
                out[t] += float(weights[t][j]) * rows[r]
    return out
