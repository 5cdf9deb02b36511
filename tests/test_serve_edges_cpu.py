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
