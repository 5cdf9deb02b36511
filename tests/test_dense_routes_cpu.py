"""Which kernels products with ordinary weights launch, on the two sides of each rule, and in what shapes, without a GPU (tests/route_recorder.cpp)."""
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


def product(rec, rows, n_in, n_out, groups=0, **kw):
    rec.launches()
    kb = -(-n_in // 128)
    d = dict(n_rows=rows, n_x_rows=rows, n_in=n_in, n_out=n_out, x_stride=-(-n_in // 16) * 16, w_stride=-(-n_in // 16) * 16, x_scale_stride=-(-kb // 4) * 4, w_scale_stride=kb, y_stride=n_out)
    if groups:
        d |= dict(starts=T.P, n_groups=groups, w_group_stride=d["w_stride"] * n_out, w_scale_group_stride=kb * -(-n_out // 128))
    if kw.get("dtype", B.E4M3) != B.E4M3:
        d |= dict(x_scale=0, w_scale=0)
    f = rec.lib.dbf_grouped_gemm if groups else rec.lib.dbf_dense_gemm
    assert f(C.byref(T._dense(**{**d, **kw})), None, C.c_size_t(0), None) == 0
    (name, grid, threads, lds), = rec.launches()
    return name.replace("dbf_dense_", ""), grid, threads


def test_few_rows_stream_weights_that_no_cache_holds(rec):
    for rows in (1, 16):
        assert product(rec, rows, 4096, 16384)[0] == "stream"          # 64 MB
        assert product(rec, rows, 4096, 16383)[0] == "few"
        assert product(rec, rows, 4096, 8192, w_up=T.P, w_up_scale=T.P)[0] == "stream"
    assert product(rec, 17, 4096, 16384)[0] == "few" and product(rec, 33, 4096, 16384)[0] == "tiles"
    # rows of up to 8192 bytes, of whole pieces of 16
    assert product(rec, 4, 8192, 32000)[0] == "stream" and product(rec, 4, 8208, 32000)[0] == "few" and product(rec, 4, 8191, 32000)[0] == "few"
    assert product(rec, 4, 4096, 32000, dtype=B.F16)[0] == "stream" and product(rec, 4, 4104, 32000, dtype=B.F16)[0] == "few"
    # of groups: four rows on average, each with some
    assert product(rec, 256, 2048, 1024, 64)[0] == "stream" and product(rec, 257, 2048, 1024, 64)[0] == "tiles"
    assert product(rec, 8, 2048, 1024, 64)[0] == "few"                # (8 groups of 2 MB at most)


def test_few_rows_of_small_weights(rec):
    # a workgroup of four or of eight wavefronts, one set of 16 weights or two
    assert product(rec, 3, 4096, 4096) == ("few", (256, 1, 1), 512)
    assert product(rec, 3, 1024, 32768) == ("few", (1024, 1, 1), 256)
    assert product(rec, 3, 512, 32768, w_up=T.P, w_up_scale=T.P) == ("few", (2048, 1, 1), 256)
    assert product(rec, 17, 4096, 4096) == ("few", (256, 1, 1), 256) and product(rec, 32, 4096, 4096)[0] == "few"
    # more rows read the weights again for each 32, but tiles of few outputs are too few for a long axis
    assert product(rec, 33, 4096, 4096)[0] == "few" and product(rec, 96, 4096, 4096)[0] == "few" and product(rec, 97, 4096, 4096)[0] == "tiles"
    assert product(rec, 32, 4096, 8193)[0] == "few" and product(rec, 33, 4096, 8193)[0] == "tiles" and product(rec, 64, 11008, 4096)[0] == "few" and product(rec, 128, 11008, 4096)[0] == "tiles"
    assert product(rec, 32, 28672, 8192) == ("few", (512, 1, 1), 256) and product(rec, 96, 11008, 4096, dtype=B.BF16) == ("few", (256, 3, 1), 256)
    assert product(rec, 128, 128, 16)[0] == "few" and product(rec, 129, 128, 16)[0] == "tiles"
    assert product(rec, 64, 8192, 8192)[0] == "tiles" and product(rec, 64, 8192, 8192, out_dtype=B.F32)[0] == "few"
    assert product(rec, 300 * 8, 2048, 1024, 64, w_up=T.P, w_up_scale=T.P)[0] == "tiles" and product(rec, 32, 11008, 4096, 2)[0] == "few"
    # rows of groups: tiles of 16, one at least for each that may have some
    assert product(rec, 12, 256, 64, 5)[:2] == ("few", (4, 1 + 5, 1))
    assert product(rec, 3, 256, 64, 5)[:2] == ("few", (4, 1 + 3, 1))


def test_launches_stay_below_what_a_grid_may_hold(rec):
    # 2^32 threads: 65536 workgroups of outputs and as many rows of groups as there are
    for kw in (dict(rows=4096, n_in=24, n_out=1 << 20, groups=1024), dict(rows=1024, n_in=1 << 20, n_out=1 << 20, groups=1024, w_group_stride=0), dict(rows=1 << 22, n_in=1, n_out=16, groups=1024)):
        name, grid, threads = product(rec, **kw)
        assert grid[0] * grid[1] * grid[2] * threads < 1 << 32 and grid[1] >= 1, (name, kw)


def test_tiles_are_chosen_by_what_a_launch_costs(rec):
    def tiles(*a, **kw):
        name, grid, threads = product(rec, *a, **kw)
        assert name == "tiles"
        return grid[0], threads

    assert tiles(2048, 4096, 16384) == (8 * 64, 512)      # 256 x 256
    assert tiles(2048, 4096, 4096) == (16 * 32, 256)      # 128 x 128
    assert tiles(256, 4096, 16384)[0] in (2 * 128, 4 * 128)
    assert tiles(160, 4096, 4096) == (3 * 64, 128)        # 64 x 64
    assert tiles(2047, 4096, 11008, w_up=T.P, w_up_scale=T.P) == (8 * 86, 512)
    # fp32 outputs of 8 bits go through fp16, whose operands leave no registers for the largest
    assert tiles(2048, 4096, 16384, out_dtype=B.F32) == (16 * 128, 256)
    assert tiles(16384, 4096, 2048, 32, w_up=T.P, w_up_scale=T.P)[1] in (256, 512)


def test_a_router_takes_one_two_or_three_launches(rec):
    def launches(tokens, experts=64):
        rec.launches()
        r = T._router(n_tokens=tokens, n_experts=experts, row_stride=experts)
        assert rec.lib.dbf_route(C.byref(r), C.c_void_p(T.P), C.c_size_t(rec.lib.dbf_route_workspace_bytes(C.byref(r))), None) == 0
        return [(name.replace("dbf_route_", ""), grid[0], threads) for name, grid, threads, _ in rec.launches()]

    assert launches(0) == [("nothing", 1, 1024)]
    assert launches(1) == [("choose", 1, 64)] and launches(32) == [("choose", 1, 512)]
    assert launches(33) == [("choose", 2, 512), ("place", 2, 1024)]
    assert launches(8192, 256) == [("choose", 256, 512), ("place", 256, 1024)]
    assert launches(8193, 257) == [("choose", 257, 512), ("sums", 65, 1024), ("place", 257, 1024)]
