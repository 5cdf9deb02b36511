"""The oracle of products with ordinary weights against what it must be, and the refusals of their entry points, without a GPU."""
import math

import numpy as np
import pytest
import torch

from oracle import dense_oracle as O
from paper_2505_11076_amd import binding as B

P = 0x10000   # an address that is never looked at


def test_the_type_in_8_bits():
    assert O.E4M3[0x7E] == 448 and O.E4M3[0x01] == 2.0 ** -9 and O.E4M3[0x08] == 2.0 ** -6 and O.E4M3[0x38] == 1 and math.isnan(O.E4M3[0xFF]) and O.E4M3[0xB8] == -1
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.E4M3, want, equal_nan=True)
    v = np.concatenate([O.E4M3[:127], (O.E4M3[:126] + O.E4M3[1:127]) / 2, np.linspace(0, 448, 9001)])
    v = np.concatenate([v, -v])
    assert np.array_equal(O.encode(v), torch.from_numpy(v).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_scales_are_the_smallest_powers_of_two():
    assert O.scale_byte(448.0) == 127 and O.scale_byte(448.5) == 128 and O.scale_byte(224.0) == 126 and O.scale_byte(224.0 * (1 + 2.0 ** -23)) == 127
    assert O.scale_byte(0) == 127 and O.scale_byte(2.0 ** -149) == 0 and O.scale_byte(3.4e38) == 247
    x = np.random.default_rng(0).normal(size=(130, 300)) * np.exp(np.random.default_rng(1).normal(size=(130, 1)) * 5)
    for rows in (1, 128):
        codes, scales = O.quantize(x, rows)
        v = O.values(codes, scales, rows)
        assert np.max(np.abs(v - x) / np.maximum(np.abs(x), 2.0 ** -6 * np.repeat(np.repeat(O.scales_of(scales), rows, 0)[:130], 128, 1)[:, :300])) <= 2.0 ** -4
        assert np.max(np.abs(O.E4M3[codes])) > 224


def test_a_router_by_hand():
    ids, w, starts, row_token, token_rows = O.route(np.array([[0.0, 2.0, 1.0], [-math.inf, -math.inf, 5.0], [1.0, 1.0, 1.0], [-math.inf] * 3]), 2, False)
    assert ids.tolist() == [[1, 2], [2, -1], [0, 1], [-1, -1]] and starts.tolist() == [0, 1, 3, 5]
    assert row_token.tolist() == [2, 0, 2, 0, 1, -1, -1, -1] and token_rows.tolist() == [[1, 3], [4, -1], [0, 2], [-1, -1]]
    assert np.allclose(w, [[math.e / (1 + math.e), 1 / (1 + math.e)], [1, 0], [0.5, 0.5], [0, 0]])
    ids, w, *_ = O.route(np.array([[0.0, 0.1, 0.2]]), 1, True, bias=np.array([0.5, 0.0, 0.0]), renormalise=False, scale=2.0)
    assert ids.tolist() == [[0]] and np.allclose(w, [[1.0]])


def _refused(code, f, *args):
    with pytest.raises(B.DbfError) as e:
        f(*args)
    assert e.value.code == code


def _dense(**kw):
    base = dict(x=P, x_scale=P, w=P, w_scale=P, y=P, x_stride=256, x_scale_stride=4, w_stride=256, w_scale_stride=2, y_stride=64, dtype=B.E4M3, out_dtype=B.F16, w_scale_type=B.E8M0,
                n_rows=5, n_x_rows=5, n_in=200, n_out=64)
    return B.Dense(**{**base, **kw})


def _grouped(**kw):
    return _dense(**{**dict(starts=P, n_groups=3, w_group_stride=256 * 64, w_scale_group_stride=2), **kw})


@pytest.mark.parametrize("kw", [dict(x=0), dict(w=0), dict(y=0), dict(x=P + 8), dict(w=P + 4), dict(w_up=P + 8, w_up_scale=P), dict(y=P + 1), dict(dtype=B.F32), dict(dtype=7),
                                dict(out_dtype=B.E4M3), dict(w_scale_type=B.F16), dict(x_scale=0), dict(w_scale=0), dict(w_up=P), dict(w_up_scale=P), dict(x_scale=P + 2),
                                dict(x_scale_stride=6), dict(x_scale_stride=0), dict(w_scale_stride=1), dict(w_scale_type=B.F32, w_scale=P + 2), dict(x_stride=192), dict(x_stride=264),
                                dict(w_stride=192), dict(w_stride=260), dict(y_stride=63), dict(n_rows=-1), dict(n_x_rows=4), dict(n_x_rows=-1, x_rows=P), dict(n_x_rows=0, x_rows=P),
                                dict(x_rows=P + 2), dict(x_stride=1 << 23), dict(w_stride=1 << 23), dict(x_rows=P, n_x_rows=1 << 21, x_stride=4096),
                                dict(dtype=B.F16), dict(dtype=B.BF16, x_scale=0), dict(dtype=B.F16, x_scale=0, w_scale=0, x_stride=204)])
def test_products_refuse(kw):
    for f, make in ((B.dbf_dense_gemm, _dense), (B.dbf_grouped_gemm, _grouped)):
        _refused(B.DBF_EINVAL, f, make(**kw))


@pytest.mark.parametrize("kw", [dict(n_in=0), dict(n_in=(1 << 20) + 1), dict(n_out=0), dict(n_out=(1 << 20) + 1)])
def test_products_refuse_shapes(kw):
    _refused(B.DBF_ESHAPE, B.dbf_dense_gemm, _dense(**kw))
    _refused(B.DBF_ESHAPE, B.dbf_grouped_gemm, _grouped(**kw))


def test_products_refuse_rows_further_apart_than_offsets_reach():
    # 2^22 values; a gathered x, whose rows may be any, has 2^32 bytes in all, its scales as many
    far = 1 << 22
    for f, make in ((B.dbf_dense_gemm, _dense), (B.dbf_grouped_gemm, _grouped)):
        for kw in (dict(x_stride=far + 16), dict(w_stride=far + 16), dict(x_scale_stride=far + 4), dict(x_scale_stride=1 << 62), dict(y_stride=(1 << 32) + 1)):
            _refused(B.DBF_EINVAL, f, make(**kw))
            _refused(B.DBF_EINVAL, f, make(n_x_rows=1 << 20, x_rows=P, **kw))
            _refused(B.DBF_EINVAL, f, make(n_rows=0, **kw))
        _refused(B.DBF_EINVAL, f, make(x_rows=P, n_x_rows=1025, x_stride=far))
        _refused(B.DBF_EINVAL, f, make(x_rows=P, n_x_rows=1025, x_scale_stride=far))
        f(make(n_rows=0, x_rows=P, n_x_rows=1024, x_stride=far, x_scale_stride=far, w_stride=far, y_stride=1 << 32))


def test_groups_are_refused_where_they_do_not_belong():
    for kw in (dict(starts=0), dict(starts=P + 2), dict(n_groups=0), dict(n_groups=B.MAX_GROUPS + 1), dict(w_group_stride=-16), dict(w_group_stride=8), dict(w_scale_group_stride=-1)):
        _refused(B.DBF_EINVAL, B.dbf_grouped_gemm, _grouped(**kw))
    _refused(B.DBF_EINVAL, B.dbf_dense_gemm, _dense(starts=P))
    _refused(B.DBF_EINVAL, B.dbf_dense_gemm, _dense(n_groups=2))
    with pytest.raises(B.DbfError):
        B.dbf_dense_gemm(None)
    # (nothing to do)
    B.dbf_dense_gemm(_dense(n_rows=0))
    B.dbf_grouped_gemm(_grouped(n_rows=0, n_x_rows=0))
    assert B.dbf_dense_gemm_workspace_bytes(_dense()) == 0 and B.dbf_grouped_gemm_workspace_bytes(_grouped()) == 0


@pytest.mark.parametrize("code,args", [
    (B.DBF_EINVAL, dict(x=0)), (B.DBF_EINVAL, dict(codes=0)), (B.DBF_EINVAL, dict(scales=0)), (B.DBF_EINVAL, dict(dtype=B.E4M3)), (B.DBF_EINVAL, dict(x=P + 1)), (B.DBF_EINVAL, dict(x_stride=199)),
    (B.DBF_EINVAL, dict(rows=-1)), (B.DBF_EINVAL, dict(block=64)), (B.DBF_EINVAL, dict(codes=P + 8)), (B.DBF_EINVAL, dict(codes_stride=216)), (B.DBF_EINVAL, dict(codes_stride=192)),
    (B.DBF_EINVAL, dict(scales_stride=1)), (B.DBF_ESHAPE, dict(cols=0)), (B.DBF_ESHAPE, dict(cols=(1 << 20) + 1)), (B.DBF_EINVAL, dict(dtype=B.F32, x=P + 2))])
def test_rounding_refuses(code, args):
    a = {**dict(x=P, dtype=B.F16, x_stride=200, rows=3, cols=200, block=1, codes=P, codes_stride=208, scales=P, scales_stride=2), **args}
    _refused(code, B.dbf_quantize, a["x"], a["dtype"], a["x_stride"], a["rows"], a["cols"], a["block"], a["codes"], a["codes_stride"], a["scales"], a["scales_stride"])


def _router(**kw):
    return B.Router(**{**dict(logits=P, row_stride=64, expert_ids=P, weights=P, starts=P, row_token=P, token_rows=P, dtype=B.F32, n_tokens=5, n_experts=64, n_top=6, scale=1.0), **kw})


def test_a_router_refuses():
    for kw in (dict(logits=0), dict(expert_ids=0), dict(weights=0), dict(starts=0), dict(row_token=0), dict(token_rows=0), dict(dtype=B.E4M3), dict(logits=P + 2), dict(bias=P + 2),
               dict(starts=P + 1), dict(n_tokens=-1), dict(n_top=0), dict(n_top=33), dict(n_top=7, n_experts=6), dict(row_stride=63), dict(score=2), dict(n_tokens=(1 << 31) // 6 + 1)):
        _refused(B.DBF_EINVAL, B.dbf_route, _router(**kw))
    for n in (0, B.MAX_GROUPS + 1):
        _refused(B.DBF_ESHAPE, B.dbf_route, _router(n_experts=n, row_stride=2000, n_top=1))
    assert B.dbf_route_workspace_bytes(_router(n_tokens=32)) == 0
    for n in (33, 9000):
        size = B.dbf_route_workspace_bytes(_router(n_tokens=n))
        assert size >= -(-n // 32) * 64
        for args in ((0, size), (P, size - 1), (P + 128, size)):
            _refused(B.DBF_EWORKSPACE, B.dbf_route, _router(n_tokens=n), *args)
    assert B.dbf_route_workspace_bytes(_router(n_top=0)) == 0


def test_a_router_refuses_more_tokens_than_a_launch_has_workgroups_for():
    # 32 tokens to a workgroup of 1024 threads, of which a launch has less than 2^32
    most = (1 << 27) - 32
    assert B.dbf_route_workspace_bytes(_router(n_tokens=most, n_top=1)) >= most // 32 * 64
    for n in (most + 1, 1 << 30):
        assert B.dbf_route_workspace_bytes(_router(n_tokens=n, n_top=1)) == 0
        _refused(B.DBF_EINVAL, B.dbf_route, _router(n_tokens=n, n_top=1), P, 1 << 60)


def test_a_sum_of_rows_refuses():
    def sums(**kw):
        return B.Combine(**{**dict(rows=P, token_rows=P, weights=P, residual=P, out=P, row_stride=10, residual_stride=10, out_stride=10, dtype=B.F16, n_rows=4, n_tokens=3, n_top=2, n_cols=10), **kw})

    for kw in (dict(rows=0), dict(token_rows=0), dict(weights=0), dict(out=0), dict(dtype=B.E4M3), dict(rows=P + 1), dict(out=P + 1), dict(residual=P + 1), dict(weights=P + 2),
               dict(token_rows=P + 2), dict(n_rows=-1), dict(n_tokens=-1), dict(n_top=0), dict(n_top=33), dict(row_stride=9), dict(out_stride=9), dict(residual_stride=9)):
        _refused(B.DBF_EINVAL, B.dbf_combine, sums(**kw))
    for n in (0, (1 << 20) + 1):
        _refused(B.DBF_ESHAPE, B.dbf_combine, sums(n_cols=n, row_stride=1 << 21, out_stride=1 << 21, residual_stride=1 << 21))
    B.dbf_combine(sums(n_tokens=0))
