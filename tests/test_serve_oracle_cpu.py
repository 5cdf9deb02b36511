"""Pins of oracle/serve_oracle.py (what stands between the layer products): closed forms, brute force and invariances; and the refusals of the
library's entry points for them, which are made before any GPU call."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import serve_oracle as S
from paper_2505_11076_amd import binding as B


def test_block_tables_by_hand():
    table = np.array([[7, -1, -1], [3, 4, -1], [-1, -1, -1]])
    out = S.block_tables([30, 64, 0], [3, 0, 33], 32, [9, 8, 6], table, 40)
    assert out[0].tolist() == [[7, 9, -1], [3, 4, -1], [8, 6, -1]]
    assert out[1] == [0, 3, 3, 36] and out[2] == [33, 64, 33]
    assert out[3][:4] == [30, 31, 32, 0] and out[3][35:] == [32, 0, 0, 0, 0]
    assert out[4][:4] == [7 * 32 + 30, 7 * 32 + 31, 9 * 32, 8 * 32] and out[4][35:] == [6 * 32, -1, -1, -1, -1]
    assert out[5] == [3, 0]
    # a page short: the tokens on it have no slot, and it is counted
    out = S.block_tables([30, 64, 0], [3, 0, 33], 32, [9, 8], table, 36)
    assert out[5] == [2, 1] and out[4][35] == -1 and out[0][2].tolist() == [8, -1, -1]


def test_norm_and_rotation():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(5, 2, 8))
    a = rng.uniform(0, 6, (5, 3))
    for inter in (False, True):
        y = S.norm_rope(x, None, 0.0, np.cos(a), np.sin(a), inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))             # a rotation keeps lengths
        assert np.array_equal(y[..., 6:], x[..., 6:])
        back = S.norm_rope(y, None, 0.0, np.cos(a), -np.sin(a), inter)
        assert np.allclose(back, x)
    y = S.norm_rope(x, np.ones(8), 0.0, None, None, False)
    assert np.allclose((y ** 2).mean(-1), 1)
    quarter = S.norm_rope(np.array([[[1.0, 0, 0, 0]]]), None, 0, np.zeros((1, 2)), np.ones((1, 2)), False)
    assert np.allclose(quarter, [[[0, 0, 1, 0]]])


def test_quantisation():
    assert S.scale_up(15 * 0.5) == 0.5 and S.scale_up(15 * (1 + 1 / 64)) == 1 + 1 / 64 and S.scale_up(15 * (1 + 1 / 128)) == 1 + 1 / 64
    assert S.scale_up(15 * 2.0 ** -24) == 2.0 ** -24 and S.scale_up(2.0 ** -24) == 2.0 ** -24 and S.scale_up(0) == 0
    rng = np.random.default_rng(2)
    for D in (64, 128, 256):
        for x in (rng.normal(size=D), np.abs(rng.normal(size=D)), np.zeros(D), rng.normal(size=D) * 1e5, rng.normal(size=D) * 1e-7, np.full(D, 57344.0), np.full(D, -3.0)):
            c, s, z = S.quantise(x)
            p = [S.group_of(d, D) for d in range(D)]
            v = s[p] * (c - z[p])
            assert np.array_equal(v.astype(np.float16).astype(np.float64), v)    # exact in fp16
            assert c.min() >= 0 and c.max() <= 15 and z.min() >= 0 and z.max() <= 15
            # half a step inside the range; the range's ends, which the integer zero may shift, a whole one
            assert (np.abs(v - np.clip(x, -S.MOST, S.MOST)) <= s[p] + 1e-12).all()
            assert np.mean(np.abs(v - np.clip(x, -S.MOST, S.MOST)) <= 0.5 * s[p] * (1 + 1e-9) + 1e-12) > 0.9


@pytest.mark.parametrize("D,page", [(64, 32), (128, 64), (256, 128)])
def test_cache_layout(D, page):
    rng = np.random.default_rng(D)
    c = S.Cache(2, page, 2, D, fill=0xA5)
    places = [q for t in range(32) for kb, kh, vb, vh in c.places(t) for q in ((kb, kh), (vb, vh))]
    assert len(set(places)) == len(places) == 64 * D and max(places)[0] < 32 * D   # every half byte once
    slots = rng.permutation(2 * page)[:20]
    k, v = rng.normal(size=(2, 20, 2, D))
    for i, s in enumerate(slots):
        for h in range(2):
            c.write(s, h, k[i, h], v[i, h])
    for i, s in enumerate(slots):
        for h in range(2):
            a, b = c.read(s, h)
            assert np.array_equal(a, S.held(k[i, h])) and np.array_equal(b, S.held(v[i, h]))
    k[0, 0, 5] = np.inf
    c.write(slots[0], 0, k[0, 0], v[0, 0])
    a, b = c.read(slots[0], 0)
    assert np.isnan(a).all() and (b == 0).all()
    assert np.array_equal(c.read(slots[1], 0)[0], S.held(k[1, 0]))
    assert S.cache_bytes(2, page, 2, D) == B.dbf_cache_bytes(2, page, 2, D)


def test_attention():
    rng = np.random.default_rng(4)
    q, k, v = rng.normal(size=(3, 4, 8)), rng.normal(size=(5, 2, 8)), rng.normal(size=(5, 2, 8))
    out, _, _ = S.attend(q, k, v, 0.3, True)
    for t in range(3):
        for h in range(4):
            n = 5 - 3 + t + 1
            w = [math.exp(0.3 * math.fsum(q[t, h] * k[j, h // 2])) for j in range(n)]
            for d in range(8):
                assert abs(out[t, h, d] - math.fsum(w[j] * v[j, h // 2, d] for j in range(n)) / math.fsum(w)) < 1e-12
    assert np.array_equal(S.attend(q, k[:1], v[:1], 0.3, True)[0][:2], np.zeros((2, 4, 8)))    # rows that see nothing
    assert np.allclose(S.attend(q, np.zeros((5, 2, 8)), v, 1.0, False)[0][:, 0], v[:, 0].mean(0))
    k2 = k.copy()
    k2[4] = np.nan
    got, _, _ = S.attend(q, k2, v, 0.3, True)
    assert np.array_equal(got[:2], out[:2]) and np.isnan(got[2]).all()


def test_log_probabilities():
    x = np.log(np.array([[0.5, 0.25, 0.125, 0.125], [1, 1, 1, 1]])) + 3
    lp, h, ids, tops = S.token_logprobs(x, [1, 3], 3)
    assert np.allclose(lp, np.log([0.25, 0.25])) and np.allclose(h, [1.75 * math.log(2), math.log(4)])
    assert ids[0, :2].tolist() == [0, 1] and ids[1].tolist() == [0, 1, 2] and np.allclose(tops[0, :2], np.log([0.5, 0.25]))
    x = np.array([[-np.inf, 0, -np.inf], [-np.inf] * 3, [np.nan, 5, np.inf], [np.inf, 0, 0]])
    lp, h, ids, _ = S.token_logprobs(x, [1, -1, 2, 9], 2)
    assert lp[0] == 0 and h[0] == 0 and lp[1] == 0 and np.isnan(h[1:]).all() and np.isnan(lp[2:]).all()
    assert ids.tolist() == [[1, 0], [0, 1], [0, 2], [0, 1]]


# ---- refusals ----------------------------------------------------------------------------------------------

P = 1 << 20   # an aligned address that nothing reads: every call here is refused before the GPU


def _heads(**kw):
    return B.Heads(**{**dict(q=P, q_stride=512, k=P, k_stride=512, v=P, v_stride=512, q_out=P, q_out_stride=512, k_out=P, k_out_stride=512, dtype=B.F16, n_tokens=3,
                             n_q_heads=4, n_kv_heads=2, head_dim=64, q_weight=P, k_weight=P, eps=1e-6, rope=P, rope_len=10, rot_dim=64, positions=P), **kw})


def _cache(**kw):
    return B.Cache(**{**dict(data=P, n_pages=4, page_tokens=32, n_kv_heads=2, head_dim=64), **kw})


def _attend(**kw):
    return B.Attend(**{**dict(q=P, q_stride=256, out=P, out_stride=256, dtype=B.F16, n_tokens=3, n_seq=1, n_q_heads=4, max_q=3, max_kv=40, q_start=P, kv_len=P, block_table=P,
                              table_stride=2, scale=1.0, causal=1), **kw})


def _refused(code, call, *args):
    with pytest.raises(B.DbfError) as e:
        call(*args)
    assert e.value.code == code, (e.value, args)


def test_an_unknown_field_is_an_error():
    with pytest.raises(TypeError):
        B.Heads(queries=1)


@pytest.mark.parametrize("at,bad", [(0, 0), (1, 0), (2, 0), (2, -1), (2, (1 << 20) + 1), (3, 16), (3, 48), (3, 512), (4, 0), (5, -1), (6, 0), (7, 0), (8, -1), (9, 0), (10, 0),
                                    (11, 0), (12, 0), (13, 0)] + [(i, P + 2) for i in (0, 1, 4, 6, 9, 10, 11, 12, 13)])
def test_block_tables_refusals(at, bad):
    args = [P, P, 3, 32, P, 5, P, 4, 7, P, P, P, P, P, 0]
    args[at] = bad
    _refused(B.DBF_EINVAL, B.dbf_block_tables, *args)


@pytest.mark.parametrize("code,kw", [
    (B.DBF_EINVAL, dict(q=0, k=0)), (B.DBF_EINVAL, dict(q=P + 1)), (B.DBF_EINVAL, dict(q_out=0)), (B.DBF_EINVAL, dict(k_out=0)), (B.DBF_EINVAL, dict(dtype=B.F32)),
    (B.DBF_EINVAL, dict(dtype=7)), (B.DBF_EINVAL, dict(n_tokens=-1)), (B.DBF_EINVAL, dict(n_q_heads=0)), (B.DBF_EINVAL, dict(n_kv_heads=0)), (B.DBF_EINVAL, dict(q_stride=255)),
    (B.DBF_EINVAL, dict(k_stride=127)), (B.DBF_EINVAL, dict(q_out_stride=255)), (B.DBF_EINVAL, dict(k_out_stride=127)), (B.DBF_ESHAPE, dict(head_dim=63)),
    (B.DBF_ESHAPE, dict(head_dim=0)), (B.DBF_ESHAPE, dict(head_dim=1026)), (B.DBF_EINVAL, dict(rot_dim=66)), (B.DBF_EINVAL, dict(rot_dim=31)), (B.DBF_EINVAL, dict(rot_dim=0)),
    (B.DBF_EINVAL, dict(rope_len=0)), (B.DBF_EINVAL, dict(positions=0)), (B.DBF_EINVAL, dict(eps=-1.0)), (B.DBF_EINVAL, dict(eps=float("nan"))),
    (B.DBF_EINVAL, dict(rope=P + 2)), (B.DBF_EINVAL, dict(positions=P + 2)), (B.DBF_EINVAL, dict(q_weight=P + 1))])
def test_qk_norm_rope_refusals(code, kw):
    _refused(code, B.dbf_qk_norm_rope, _heads(**kw))
    if "k_out" not in kw and "k_out_stride" not in kw and kw != dict(q=0, k=0):
        _refused(code, B.dbf_cache_append, _heads(**kw), _cache(), P)


@pytest.mark.parametrize("code,heads,cache,slots", [
    (B.DBF_EINVAL, dict(k=0), {}, P), (B.DBF_EINVAL, dict(v=0), {}, P), (B.DBF_EINVAL, {}, {}, 0), (B.DBF_EINVAL, {}, {}, P + 2), (B.DBF_EINVAL, dict(v_stride=127), {}, P),
    (B.DBF_EINVAL, dict(v=P + 1), {}, P), (B.DBF_EINVAL, {}, dict(data=0), P), (B.DBF_EINVAL, {}, dict(data=P + 8), P), (B.DBF_EINVAL, {}, dict(n_pages=0), P),
    (B.DBF_EINVAL, {}, dict(page_tokens=40), P), (B.DBF_ESHAPE, {}, dict(n_kv_heads=1), P), (B.DBF_ESHAPE, {}, dict(head_dim=128), P),
    (B.DBF_ESHAPE, dict(head_dim=32, rot_dim=32), dict(head_dim=32), P), (B.DBF_EINVAL, {}, dict(n_pages=1 << 30), P)])
def test_cache_append_refusals(code, heads, cache, slots):
    _refused(code, B.dbf_cache_append, _heads(**heads), _cache(**cache), slots)


def test_cache_read_and_size_refusals():
    for args in ((0, 3, P, P, 0), (P, -1, P, P, 0), (P, 3, 0, P, 0), (P, 3, P, 0, 0), (P, 3, P, P, 3), (P + 2, 3, P, P, 0), (P, 3, P + 1, P, 0), (P, 3, P, P + 2, B.F32)):
        _refused(B.DBF_EINVAL, B.dbf_cache_read, _cache(), *args)
    _refused(B.DBF_EINVAL, B.dbf_cache_read, _cache(data=0), P, 3, P, P)
    for bad in ((0, 32, 2, 64), (4, 33, 2, 64), (4, 32, 0, 64), (4, 32, 2, 96), (-1, 32, 2, 64), (1 << 27, 64, 2, 64)):
        assert B.dbf_cache_bytes(*bad) == 0
    assert B.dbf_cache_bytes(1 << 20, 256, 16, 256) == (1 << 23) * 16 * 36 * 256   # past 32 bits


@pytest.mark.parametrize("code,kw", [
    (B.DBF_EINVAL, dict(q=0)), (B.DBF_EINVAL, dict(out=0)), (B.DBF_EINVAL, dict(kv_len=0)), (B.DBF_EINVAL, dict(block_table=0)), (B.DBF_EINVAL, dict(q=P + 1)),
    (B.DBF_EINVAL, dict(q_start=P + 2)), (B.DBF_EINVAL, dict(dtype=B.F32)), (B.DBF_EINVAL, dict(n_seq=0)), (B.DBF_EINVAL, dict(n_seq=65536)), (B.DBF_EINVAL, dict(n_tokens=-1)),
    (B.DBF_ESHAPE, dict(n_q_heads=3, q_stride=512, out_stride=512)), (B.DBF_EINVAL, dict(max_q=-1)), (B.DBF_EINVAL, dict(max_kv=-1)), (B.DBF_EINVAL, dict(table_stride=0)),
    (B.DBF_EINVAL, dict(q_stride=255)), (B.DBF_EINVAL, dict(out_stride=255)), (B.DBF_EINVAL, dict(scale=float("nan"))), (B.DBF_EINVAL, dict(scale=float("inf"))),
    (B.DBF_EINVAL, dict(n_q_heads=0))])
def test_cache_attend_refusals(code, kw):
    _refused(code, B.dbf_cache_attend, _attend(**kw), _cache(), P, 1 << 30)


def test_cache_attend_workspace():
    _refused(B.DBF_ESHAPE, B.dbf_cache_attend, _attend(), _cache(head_dim=96), P, 1 << 30)
    _refused(B.DBF_EINVAL, B.dbf_cache_attend, _attend(), _cache(data=0), P, 1 << 30)
    assert B.dbf_cache_attend_workspace_bytes(_attend(n_seq=0), _cache()) == 0
    long_one = dict(max_q=1, n_tokens=1, max_kv=100000, table_stride=4000)
    need = B.dbf_cache_attend_workspace_bytes(_attend(**long_one), _cache())
    if need:
        _refused(B.DBF_EWORKSPACE, B.dbf_cache_attend, _attend(**long_one), _cache(), P, need - 1)
        _refused(B.DBF_EWORKSPACE, B.dbf_cache_attend, _attend(**long_one), _cache(), P + 128, need)
        _refused(B.DBF_EWORKSPACE, B.dbf_cache_attend, _attend(**long_one), _cache(), 0, need)


def test_cache_attend_of_the_longest():
    """More than 2^30 tokens a request are refused, up to there offsets fit; where all requests together are more than the sums of shares hold, there are none."""
    longest = dict(max_q=1, n_tokens=1, max_kv=1 << 30, table_stride=1 << 25)
    _refused(B.DBF_EINVAL, B.dbf_cache_attend, _attend(**{**longest, "max_kv": (1 << 30) + 1}), _cache(), P, 1 << 30)
    assert B.dbf_cache_attend_workspace_bytes(_attend(**{**longest, "max_kv": (1 << 30) + 1}), _cache()) == 0
    assert B.dbf_cache_attend_workspace_bytes(_attend(**longest), _cache()) > 0
    assert B.dbf_cache_attend_workspace_bytes(_attend(**{**longest, "n_seq": 16, "n_tokens": 16}), _cache()) == 0


def test_token_logprobs_refusals():
    ok = [P, B.F16, 100, 4, 100, P, 5, P, P, P, P, P, 1 << 30]
    for code, at, bad in ((B.DBF_EINVAL, 0, 0), (B.DBF_EINVAL, 1, 3), (B.DBF_EINVAL, 2, 99), (B.DBF_EINVAL, 3, -1), (B.DBF_ESHAPE, 4, 0), (B.DBF_ESHAPE, 4, (1 << 24) + 1),
                          (B.DBF_EINVAL, 5, 0), (B.DBF_EINVAL, 6, -1), (B.DBF_EINVAL, 6, 65), (B.DBF_EINVAL, 7, 0), (B.DBF_EINVAL, 9, 0), (B.DBF_EINVAL, 10, 0),
                          (B.DBF_EINVAL, 0, P + 1), (B.DBF_EINVAL, 5, P + 2), (B.DBF_EINVAL, 8, P + 2)):
        args = list(ok)
        args[at] = bad
        _refused(code, B.dbf_token_logprobs, *args)
    _refused(B.DBF_EINVAL, B.dbf_token_logprobs, P, B.F16, 5, 4, 4, P, 5, P, P, P, P, P, 1 << 30)   # more alternatives than tokens
    assert B.dbf_token_logprobs_workspace_bytes(1, 0, 1) == 0
    need = B.dbf_token_logprobs_workspace_bytes(1, 128256, 20)
    if need:
        _refused(B.DBF_EWORKSPACE, B.dbf_token_logprobs, P, B.F16, 128256, 1, 128256, P, 20, P, P, P, P, P, need - 1)
        _refused(B.DBF_EWORKSPACE, B.dbf_token_logprobs, P, B.F16, 128256, 1, 128256, P, 20, P, P, P, P, P + 128, need)


def test_calls_with_nothing_to_do():
    """No token, no row: nothing is launched, so they succeed without a GPU."""
    B.dbf_qk_norm_rope(_heads(n_tokens=0))
    B.dbf_cache_append(_heads(n_tokens=0), _cache(), P)
    B.dbf_cache_read(_cache(), P, 0, P, P)
    B.dbf_cache_attend(_attend(n_tokens=0), _cache(), P, 1 << 30)
    B.dbf_cache_attend(_attend(max_q=0), _cache(), P, 1 << 30)
    B.dbf_token_logprobs(P, B.F16, 100, 0, 100, P, 5, P, P, P, P, P, 1 << 30)


def test_descriptors_match_the_header():
    """Sizes and offsets of the descriptors as a C compiler lays them out."""
    import os
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = []
    for cls, name in ((B.Cache, "dbf_cache"), (B.Heads, "dbf_heads"), (B.Attend, "dbf_attend")):
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f, _ in cls._fields_]
    with tempfile.TemporaryDirectory() as tmp:
        src = os.path.join(tmp, "layout.c")
        with open(src, "w") as fh:
            fh.write('#include <stdio.h>\n#include <stddef.h>\n#include "dbf.h"\nint main(void) {\n%s\nreturn 0;\n}\n' % "\n".join(lines))
        subprocess.run(["gcc", "-I", os.path.join(root, "include"), src, "-o", os.path.join(tmp, "layout")], check=True, capture_output=True)
        got = [int(v) for v in subprocess.run([os.path.join(tmp, "layout")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for cls in (B.Cache, B.Heads, B.Attend):
        want.append(C.sizeof(cls))
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want
