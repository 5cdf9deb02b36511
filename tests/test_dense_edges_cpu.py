"""Launches of products with ordinary weights and of the router at the ends of their sizes, without a GPU (tests/route_recorder.cpp)."""
import ctypes as C

import pytest

import test_dense_oracle_cpu as T
from paper_2505_11076_amd import binding as B
from test_routes_cpu import Recorder


@pytest.fixture(scope="module")
def rec():
    r = Recorder()
    r.lib.dbf_route_workspace_bytes.restype = C.c_size_t
    return r


@pytest.mark.parametrize("tokens", [32, 33, 1 << 20, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, 3 << 24, 1 << 26, (1 << 27) - 32])
@pytest.mark.parametrize("experts", [8, 64, 128, 256, 257, 300, 1024])
def test_a_router_of_many_tokens_has_all_its_wavefronts(rec, tokens, experts):
    """32 tokens or more have 512 threads to a workgroup, whatever their number times the lanes of a token comes to."""
    rec.launches()
    r = T._router(n_tokens=tokens, n_experts=experts, row_stride=experts, n_top=4)
    assert rec.lib.dbf_route(C.byref(r), C.c_void_p(T.P), C.c_size_t(rec.lib.dbf_route_workspace_bytes(C.byref(r))), None) == B.DBF_OK
    (name, grid, threads, _), *_ = rec.launches()
    assert name == "dbf_route_choose" and grid == ((tokens + 31) // 32, 1, 1) and threads == 512


def test_a_router_of_few_tokens_has_no_wavefront_without_one(rec):
    for tokens, experts, threads in ((1, 64, 64), (4, 64, 64), (5, 64, 128), (31, 64, 512), (28, 64, 448), (1, 300, 64), (2, 300, 128), (7, 300, 448), (8, 300, 512), (31, 300, 512)):
        rec.launches()
        r = T._router(n_tokens=tokens, n_experts=experts, row_stride=experts, n_top=4)
        assert rec.lib.dbf_route(C.byref(r), None, C.c_size_t(0), None) == B.DBF_OK
        (_, grid, of, _), = rec.launches()
        assert grid == (1, 1, 1) and of == threads, (tokens, experts)
