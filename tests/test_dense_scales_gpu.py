"""Scales of products with ordinary weights at their edges: what lies behind a row's last block, and the ends of their range.  Bounds are those of
tests/test_dense_gpu.py; fp32 outputs have nothing of the 8-bit instructions' beside theirs, whatever the scales are."""
import numpy as np
import pytest
import torch

import gpu_util as G
import test_dense_gpu as D
from oracle import dense_oracle as O
from paper_2505_11076_amd import binding as B

pytestmark = pytest.mark.gpu


def kb_of(n_in):
    return -(-n_in // 128)


def spoil(o, n_in):
    """No numbers in every scale behind the last block of a row."""
    assert o.scale.shape[-1] > kb_of(n_in) or kb_of(n_in) % 4 == 0
    o.scale[..., kb_of(n_in):] = 255 if o.scale.dtype == torch.uint8 else float("nan")


def small(w, scale_type):
    w.values *= 2.0 ** -8
    w.scale = w.scale - 8 if scale_type == B.E8M0 else w.scale * 2.0 ** -8


# rows, n_in, n_out: weights that stream (64 MB and more), few rows, tiles; 9, 10, 11, 18, 23, 42 and 45 blocks, the last of them whole or not
SIZES = [(1, 1152, 58300), (13, 1280, 52500), (16, 1408, 47700), (3, 2304, 29200), (2, 2880, 23400), (7, 5376, 12500), (4, 1040, 64600), (5, 5648, 11900),
         (1, 1152, 40), (24, 1280, 40), (16, 1408, 300), (130, 1152, 70), (200, 1280, 130), (300, 2880, 300)]


@pytest.mark.parametrize("scale_type,out", [(B.E8M0, B.F16), (B.E8M0, B.F32), (B.F32, B.BF16), (B.F32, B.F32)], ids=lambda t: str(t))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "%dx%dx%d" % s)
def test_scales_behind_the_last_block_are_not_looked_at(size, gated, scale_type, out):
    rows, n_in, n_out = size
    if gated and n_out > 1000:
        n_out = n_out // 2 + 1
    g = D.gen(rows + n_in)
    x = D.Operand(rows, n_in, B.E4M3, g, extra=1)
    w = [D.Operand(n_out, n_in, B.E4M3, g, 128, scale_type, extra=1) for _ in range(1 + gated)]
    for o in w:
        small(o, scale_type)
    for o in [x] + w:
        spoil(o, n_in)
    what = "%d x %d -> %d, scales %d, out %d%s" % (rows, n_in, n_out, scale_type, out, ", gated" if gated else "")
    G.say(what)
    y = D.run_dense(x, w[0], w[1] if gated else None, n_in, n_out, out, rows, scale_type=scale_type)
    torch.cuda.synchronize()
    want, off = D.expected(x.values[0], w[0].values[0], w[1].values[0] if gated else None, out == B.F32, out)
    assert torch.isfinite(y[want.abs() < 60000]).all(), what
    keep = want.abs() < 60000
    D.near(torch.where(keep, y.double(), 0), torch.where(keep, want, 0), off, what)


@pytest.mark.parametrize("out", [B.F16, B.F32])
@pytest.mark.parametrize("n_in", [1152, 1280, 1408])
def test_scales_behind_the_last_block_of_experts_rows(n_in, out):
    """The way down of a decode batch's experts: 40 rows of 64 groups, weights that stream (40 groups of 4.7 MB at most)."""
    groups, rows, n_out = 64, 40, 4100
    g = D.gen(n_in)
    x, w = D.Operand(rows, n_in, B.E4M3, g, extra=1), D.Operand(n_out, n_in, B.E4M3, g, 128, groups=groups)
    small(w, B.E8M0)
    spoil(x, n_in)
    each = D.split(rows, groups, g)
    starts = torch.tensor([sum(each[:i]) for i in range(groups + 1)], dtype=torch.int32, device="cuda")
    y = D.run_dense(x, w, None, n_in, n_out, out, rows, starts=starts)
    torch.cuda.synchronize()
    for i, m in enumerate(each):
        at = slice(int(starts[i]), int(starts[i]) + m)
        want, off = D.expected(x.values[0][at], w.values[i], None, out == B.F32, out)
        keep = want.abs() < 60000
        D.near(torch.where(keep, y[at].double(), 0), torch.where(keep, want, 0), off, "group %d" % i)


@pytest.mark.parametrize("rows,n_out", [(3, 60000), (3, 50), (140, 70)])
def test_rounded_rows_in_a_buffer_of_no_numbers(rows, n_out):
    """dbf_quantize into scales whose room held 255 everywhere, then the product: what rounding leaves as it was counts for nothing."""
    n_in = 1152
    g = D.gen(rows)
    t = torch.randn(rows, n_in, generator=g, device="cuda").half()
    codes, scales = torch.full((rows, n_in), 0x7F, dtype=torch.uint8, device="cuda"), torch.full((rows, 12), 255, dtype=torch.uint8, device="cuda")
    B.dbf_quantize(t.data_ptr(), B.F16, n_in, rows, n_in, 1, codes.data_ptr(), n_in, scales.data_ptr(), 12, G.stream_handle())
    w = D.Operand(n_out, n_in, B.E4M3, g, 128)
    small(w, B.E8M0)
    y = torch.empty(rows, n_out, device="cuda")
    B.dbf_dense_gemm(B.Dense(x=codes.data_ptr(), x_scale=scales.data_ptr(), x_stride=n_in, x_scale_stride=12, n_x_rows=rows, w=w.data.data_ptr(), w_scale=w.scale_ptr(), w_stride=w.stride,
                             w_scale_stride=w.scale_stride, y=y.data_ptr(), y_stride=n_out, dtype=B.E4M3, out_dtype=B.F32, w_scale_type=B.E8M0, n_rows=rows, n_in=n_in, n_out=n_out), 0, 0,
                     G.stream_handle())
    torch.cuda.synchronize()
    xv = torch.from_numpy(O.values(*O.quantize(t.double().cpu().numpy(), 1), 1)).cuda()
    want, off = D.expected(xv, w.values[0], None, True, B.F32)
    D.near(y, want, off, "%d rows" % rows)


# Scales of rows (bytes) and of weights that meet within fp32: numbers near 2^-126 and below it, whose sums with the smallest codes leave fp32's normal range on the way
ENDS = [(240, 1.7 * 2.0 ** -126), (247, 1.3 * 2.0 ** -100), (254, -1.9 * 2.0 ** -120), (253, 1.625 * 2.0 ** -140), (254, 3 * 2.0 ** -149), (200, 1.1 * 2.0 ** -126), (0, 1.3 * 2.0 ** 112),
        (1, -1.7 * 2.0 ** 120), (0, 1.9 * 2.0 ** 127), (127, 1.0), (100, 3.1e7), (140, 0.0)]


@pytest.mark.parametrize("rows,n_in,n_out", [(3, 128, 20), (3, 640, 20), (70, 640, 20), (200, 384, 130), (2, 1024, 66000)])
@pytest.mark.parametrize("codes", ["smallest", "all"])
def test_fp32_scales_at_the_ends_of_their_range_cost_no_precision(rows, n_in, n_out, codes):
    g = D.gen(rows + n_in)
    x, w = D.Operand(rows, n_in, B.E4M3, g), D.Operand(n_out, n_in, B.E4M3, g, 128, B.F32)
    if codes == "smallest":   # (subnormal codes, of either sign: products of 2^-18 and some of them)
        for o in (x, w):
            o.data &= 0x83
    xv, wv = D.table()[x.data[0, :, :n_in].int()], D.table()[w.data[0, :, :n_in].int()]
    v, size = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    for a, b in ENDS:
        x.scale[:], w.scale[:] = a, b
        b = float(np.float32(b))
        y = D.run_dense(x, w, None, n_in, n_out, B.F32, rows, scale_type=B.F32)
        torch.cuda.synchronize()
        s = 2.0 ** (a - 127) * b
        want = v * s
        # (a sum in chains of K + 3 additions, the scale, the output; what is subnormal as a result is off by half of 2^-149 for each block)
        off = (n_in + 4) * D.U * size * abs(s) + D.U * want.abs() + 2.0 ** -150 * (kb_of(n_in) + 1)
        keep = size * abs(s) < 3e38
        far = torch.where(keep, (y.double() - want).abs() / off, 0).max().item()
        G.say("%d x %d -> %d, scales 2^%d and %g: %.3g of the bound" % (rows, n_in, n_out, a - 127, b, far))
        assert torch.isfinite(y[keep]).all() and far <= 1, (a, b)


@pytest.mark.parametrize("rows,n_in,n_out", [(3, 640, 20), (70, 640, 20), (200, 384, 130), (2, 1024, 66000)])
def test_powers_of_two_at_the_ends_of_their_range_cost_no_precision(rows, n_in, n_out):
    g = D.gen(rows + n_in)
    x, w = D.Operand(rows, n_in, B.E4M3, g), D.Operand(n_out, n_in, B.E4M3, g, 128)
    for o in (x, w):
        o.data &= 0x83
    xv, wv = D.table()[x.data[0, :, :n_in].int()], D.table()[w.data[0, :, :n_in].int()]
    v, size = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    for a, b in ((0, 240), (240, 0), (1, 253), (0, 0), (100, 140), (254, 120)):
        x.scale[:], w.scale[:] = a, b
        y = D.run_dense(x, w, None, n_in, n_out, B.F32, rows)
        torch.cuda.synchronize()
        s = 2.0 ** (a + b - 254)
        off = (n_in + 4) * D.U * size * s + D.U * (v * s).abs() + 2.0 ** -150 * (kb_of(n_in) + 1)
        assert torch.isfinite(y).all() and ((y.double() - v * s).abs() <= off).all(), (a, b)
