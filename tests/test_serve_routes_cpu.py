"""Which kernels attention over the cache launches, and in what shape, on the two sides of each of its rules, without a GPU (tests/route_recorder.cpp)."""
import ctypes as C

import pytest

import test_serve_oracle_cpu as T
from paper_2505_11076_amd import binding as B
from test_routes_cpu import Recorder

WORKGROUPS = {64: 1024, 128: 768, 256: 512}   # that the chip holds at once, of few rows


@pytest.fixture(scope="module")
def rec():
    r = Recorder()
    r.lib.dbf_cache_attend_workspace_bytes.restype = C.c_size_t
    return r


def attend(rec, n_seq, hq, hk, D, max_q, max_kv, page=32):
    rec.launches()
    a = T._attend(n_seq=n_seq, n_tokens=n_seq * max_q, n_q_heads=hq, q_stride=hq * D, out_stride=hq * D, max_q=max_q, max_kv=max_kv, table_stride=-(-max_kv // page) + 1)
    c = T._cache(n_pages=1 << 20, page_tokens=page, n_kv_heads=hk, head_dim=D)
    n = rec.lib.dbf_cache_attend_workspace_bytes(C.byref(a), C.byref(c))
    assert rec.lib.dbf_cache_attend(C.byref(a), C.byref(c), C.c_void_p(T.P), C.c_size_t(n), None) == 0
    got = [(name, grid) for name, grid, _, _ in rec.launches()]
    assert all("dbf_attend" in name for name, _ in got)
    return [(name.replace("dbf_attend_", ""), grid) for name, grid in got], n


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n_seq,hk", [(1, 1), (1, 8), (13, 3), (64, 8), (300, 2), (600, 2)])
def test_items_are_shared_out_from_a_length_on_that_grows_with_their_number(rec, n_seq, hk, D):
    items = n_seq * hk
    most = 1200 + 11 * items
    got, n = attend(rec, n_seq, 2 * hk, hk, D, 1, most)
    assert got == [("items", (hk, n_seq, 1))] and n == 0
    got, n = attend(rec, n_seq, 2 * hk, hk, D, 3, most + 1)
    # a join's launch is by items where they are fewer than the shares, and else by shares
    assert got == [("shares", (WORKGROUPS[D], 1, 1)), ("join", (6, min(items, WORKGROUPS[D]), 1))] and n > 0


def test_few_rows_are_up_to_sixteen_of_a_request_and_key_head(rec):
    for hq, hk, rows in ((16, 1, 1), (8, 2, 4), (3, 1, 5), (7, 7, 16)):
        assert attend(rec, 2, hq, hk, 128, rows, 500)[0] == [("items", (hk, 2, 1))]
    for hq, hk, rows in ((17, 1, 1), (8, 2, 5), (3, 1, 6), (7, 7, 17)):
        got, _ = attend(rec, 2, hq, hk, 128, rows, 500)
        assert got == [("many", (hk, 2, 1))]


def test_the_long_axis_of_many_rows_goes_in_parts_where_workgroups_are_few(rec):
    # 512 workgroups and more: one part; fewer: as many parts as make them 512, of 512 tokens at least
    got, n = attend(rec, 4, 32, 32, 128, 512, 8192)
    assert got == [("many", (32, 4, 4))] and n == 0
    got, n = attend(rec, 1, 32, 8, 128, 512, 30000)    # 16 blocks of 8 heads
    assert got == [("many", (8 * 4, 1, 16)), ("parts", (2048 // 8, 8, 1))] and n == 8 * 4 * 2048 * (8 + 128 * 4)
    got, n = attend(rec, 1, 4, 4, 128, 130, 1100)
    assert got == [("many", (4 * 3, 1, 2)), ("parts", (17, 4, 1))] and n > 0
    assert attend(rec, 1, 4, 4, 128, 130, 512)[0] == [("many", (4, 1, 2))]
