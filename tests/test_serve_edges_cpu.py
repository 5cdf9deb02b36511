"""Sizes and refusals of the calls between the layer products that need no GPU."""
import pytest

import test_serve_oracle_cpu as T
from paper_2505_11076_amd import binding as B


@pytest.mark.parametrize("kw", [dict(max_q=1, n_tokens=1, max_kv=131071, table_stride=4096), dict(max_q=40, n_tokens=40, max_kv=5000, table_stride=200), dict(max_q=1, n_tokens=1)])
def test_a_workspace_is_sized_before_there_is_a_cache(kw):
    """A program that makes its buffers first knows the cache's sizes and not yet where it lies (nor where q, out and the tables do)."""
    want = B.dbf_cache_attend_workspace_bytes(T._attend(**kw), T._cache())
    assert (want > 0) == (kw.get("max_kv", 0) > 4000)
    assert B.dbf_cache_attend_workspace_bytes(T._attend(**kw), T._cache(data=0)) == want
    assert B.dbf_cache_attend_workspace_bytes(T._attend(**{**kw, "q": 0, "out": 0, "q_start": 0, "kv_len": 0, "block_table": 0}), T._cache(data=0)) == want
    for bad in (dict(n_pages=0), dict(page_tokens=40), dict(n_kv_heads=0), dict(head_dim=96)):
        assert B.dbf_cache_attend_workspace_bytes(T._attend(**kw), T._cache(data=0, **bad)) == 0
    T._refused(B.DBF_EINVAL, B.dbf_cache_attend, T._attend(**kw), T._cache(data=0), T.P, 1 << 40)


def test_more_rows_of_a_request_than_a_launch_takes_are_refused():
    most = 65535 * 128
    for hq in (4, 256):
        rows = most // (hq // 2)
        kw = dict(n_q_heads=hq, q_stride=hq * 64, out_stride=hq * 64, n_tokens=0)
        B.dbf_cache_attend(T._attend(**kw, max_q=rows), T._cache(), T.P, 1 << 40)   # (no tokens: nothing to do)
        for n in (0, rows + 1):
            T._refused(B.DBF_EINVAL, B.dbf_cache_attend, T._attend(**{**kw, "n_tokens": n}, max_q=rows + 1), T._cache(), T.P, 1 << 40)
        assert B.dbf_cache_attend_workspace_bytes(T._attend(**kw, max_q=rows + 1, max_kv=100000, table_stride=4000), T._cache()) == 0
