"""Oracle of what stands between the layer products of a token pass, in numpy and 64 bits: block tables, norm and rotation, the cache in
4 bits, attention over it, log probabilities.  Written from the definitions in include/dbf.h, by loops where those are plainer."""
import math

import numpy as np

BLOCK, GROUP, MOST = 32, 64, 57344.0


# ---- block tables ------------------------------------------------------------------------------------------


def block_tables(cached, new, page, free, table, max_tokens):
    """(table, q_start, kv_len, positions, slots, status) for lists of lengths; table: 2-d int array (copied)."""
    table = np.array(table, dtype=np.int64)
    stride = table.shape[1]
    start, kv, pos, slots, taken = [0], [], [], [], 0
    for i, (c, n) in enumerate(zip(cached, new)):
        c, n = max(int(c), 0), max(int(n), 0)
        have = -(-c // page)
        for r in range(have, -(-(c + n) // page)):
            if r < stride:
                table[i, r] = free[taken] if taken < len(free) else -1
            taken += 1
        for p in range(c, c + n):
            r = p // page
            pos.append(p)
            slots.append(int(table[i, r]) * page + p % page if r < stride and table[i, r] >= 0 else -1)
        start.append(start[-1] + n)
        kv.append(c + n)
    fill = max(0, max_tokens - len(pos))
    pos, slots = (pos + [0] * fill)[:max_tokens], (slots + [-1] * fill)[:max_tokens]
    return table, start, kv, pos, slots, [min(taken, len(free)), max(0, taken - len(free))]


# ---- heads -------------------------------------------------------------------------------------------------


def norm_rope(x, weight, eps, cos, sin, interleaved):
    """x [..., heads, D] with cos and sin [..., rot / 2] of each row's position (None: no rotation)."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    y = x.copy()
    if cos is not None:
        half = cos.shape[-1]
        for i in range(half):
            u, w = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            c, s = cos[..., None, i], sin[..., None, i]
            y[..., u] = x[..., u] * c - x[..., w] * s
            y[..., w] = x[..., w] * c + x[..., u] * s
    return y


# ---- the cache ---------------------------------------------------------------------------------------------


def group_of(d, D):
    return (d // 16) % (D // GROUP)


def scale_up(r):
    """r / 15 rounded up to 7 significant bits and to a multiple of 2^-24."""
    if r == 0:
        return 0.0
    m, e = math.frexp(r / 15)
    s = math.ldexp(math.ceil(math.ldexp(m, 7)), e - 7)
    return math.ceil(s * 2.0 ** 24) / 2.0 ** 24


def quantise(x):
    """(codes [D], s [D/64], z [D/64]) of a head's values."""
    x = np.clip(np.asarray(x, np.float64), -MOST, MOST)
    D = x.size
    codes, s, z = np.zeros(D, np.int64), np.zeros(D // GROUP), np.zeros(D // GROUP)
    for p in range(D // GROUP):
        dims = [d for d in range(D) if group_of(d, D) == p]
        lo, hi = min(0.0, x[dims].min()), max(0.0, x[dims].max())
        s[p] = scale_up(hi - lo)
        by = s[p] or 1.0
        z[p] = np.rint(-lo / by)
        codes[dims] = np.clip(np.rint(x[dims] / by) + z[p], 0, 15)
    return codes, s, z


def held(x):
    """The values that the cache holds of x [..., D]."""
    x = np.asarray(x, np.float64)
    out = np.zeros_like(x)
    for at in np.ndindex(x.shape[:-1]):
        c, s, z = quantise(x[at])
        p = [group_of(d, x.shape[-1]) for d in range(x.shape[-1])]
        out[at] = s[p] * (c - z[p])
    return out


def cache_bytes(pages, page, heads, D):
    return pages * (page // BLOCK) * heads * 36 * D


class Cache:
    """The bytes of a cache, written and read by the layout's description, token by token."""

    def __init__(self, pages, page, heads, D, fill=0):
        self.pages, self.page, self.heads, self.D, self.n = pages, page, heads, D, D // GROUP
        self.data = np.full(cache_bytes(pages, page, heads, D), fill, np.uint8)

    def record(self, slot, head):
        p, t = divmod(slot, self.page)
        at = ((p * self.heads + head) * (self.page // BLOCK) + t // BLOCK) * 36 * self.D
        return self.data[at: at + 36 * self.D], t % BLOCK

    def places(self, t):
        """[(key byte, key half, value byte, value half)] of a token's values."""
        h, g, i = t // 16, t // 4 % 4, t % 4
        for d in range(self.D):
            run, l = divmod(d, 16)
            p, r = run % self.n, run // self.n
            yield t * (self.D // 2) + d // 2, d % 2, 16 * self.D + 1024 * p + 16 * (16 * g + l) + 4 * (2 * (r // 2) + h) + i, r % 2

    def words(self, rec, t):
        w = rec[32 * self.D:].view(np.float16).reshape(2, self.n, BLOCK, 2)
        return w[0, :, t], w[1, :, t]

    def write(self, slot, head, k, v):
        rec, t = self.record(slot, head)
        fine = np.isfinite(k).all() and np.isfinite(v).all()
        (kc, ks, kz), (vc, vs, vz) = quantise(np.where(np.isfinite(k), k, 0)), quantise(np.where(np.isfinite(v), v, 0))
        for d, (kb, kh, vb, vh) in enumerate(self.places(t)):
            rec[kb] = rec[kb] & (0xF0 if kh == 0 else 0x0F) | int(kc[d]) << 4 * kh
            rec[vb] = rec[vb] & (0xF0 if vh == 0 else 0x0F) | int(vc[d]) << 4 * vh
        kw, vw = self.words(rec, t)
        kw[:, 0], kw[:, 1] = ks, (-ks * kz if fine else np.nan)
        vw[:, 0], vw[:, 1] = (vs, -vs * vz) if fine else (0, 0)

    def read(self, slot, head):
        rec, t = self.record(slot, head)
        kw, vw = (w.astype(np.float64) for w in self.words(rec, t))
        k, v = np.zeros(self.D), np.zeros(self.D)
        for d, (kb, kh, vb, vh) in enumerate(self.places(t)):
            p = group_of(d, self.D)
            k[d] = kw[p, 0] * (int(rec[kb]) >> 4 * kh & 15) + kw[p, 1]
            v[d] = vw[p, 0] * (int(rec[vb]) >> 4 * vh & 15) + vw[p, 1]
        return k, v


# ---- attention ---------------------------------------------------------------------------------------------


def attend(q, k, v, scale, causal):
    """q [rows, n_q, D], k and v [tokens, n_kv, D] of one request -> (out, sum of p |v|, largest sum of |q k| scale of a row): the last two
    for bounds of the error.  Keys that a row does not see count for nothing, whatever they hold."""
    rows, n_q, D = q.shape
    tokens, n_kv = k.shape[:2]
    out, weight, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros((rows, n_q))
    for t in range(rows):
        seen = max(0, min(tokens, tokens - rows + t + 1)) if causal else tokens
        if not seen:
            continue
        for h in range(n_q):
            g = h // (n_q // n_kv)
            K, V = k[:seen, g], v[:seen, g]
            with np.errstate(invalid="ignore"):
                x = (K @ q[t, h]) * scale
                p = np.exp(x - x.max())
                p /= p.sum()
                out[t, h], weight[t, h] = p @ V, p @ np.abs(V)
                size[t, h] = (np.abs(K) @ np.abs(q[t, h])).max() * abs(scale)
    return out, weight, size


# ---- log probabilities -------------------------------------------------------------------------------------


def token_logprobs(x, targets, top):
    """(logprob, entropy, ids, their log probabilities) of rows of logits."""
    x = np.asarray(x, np.float64)
    rows, vocab = x.shape
    lp, h, ids, tops = np.zeros(rows), np.zeros(rows), np.zeros((rows, top), np.int64), np.zeros((rows, top))
    for r in range(rows):
        y = x[r]
        # no numbers first, then by value, ties to the lowest index
        order = np.lexsort((np.arange(vocab), -np.where(np.isnan(y), np.inf, y), ~np.isnan(y)))[:top]
        ids[r] = order
        if np.isnan(y).any() or np.isposinf(y).any() or np.isneginf(y).all():
            lp[r] = h[r] = np.nan
            tops[r] = np.nan
        else:
            with np.errstate(divide="ignore", invalid="ignore"):
                l = (y - y.max()) - np.log(np.exp(y - y.max()).sum())
                lp[r] = l[targets[r]] if 0 <= targets[r] < vocab else np.nan
                h[r] = -np.where(np.isneginf(l), 0, np.exp(l) * np.where(np.isneginf(l), 0, l)).sum()
                tops[r] = l[order]
        if targets[r] < 0:
            lp[r] = 0.0
    return lp, h, ids, tops
