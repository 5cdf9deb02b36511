"""Products with ordinary weights, rounding to 8 bits, routing and the way back, against their definitions in 64 bits.

Tolerances (u = 2^-24, half a step of fp32 relative to the value):
  codes, scales, ids, rows: equal.
  a product of K values in fp32, of exact products of 16-bit operands (or of codes made fp16): a chain of K + 3 additions at most, scales among them: (K + 4) u sum |x w|.
  from the 8-bit instructions: what they cut off of each product is below 2^-13 of the largest of its sixteen neighbours, so 16 * 2^-13 of that for each sixteen, beside the above.
  gated, y = silu(g) v with errors dg and dv: |silu'| < 1.1, so 1.1 dg (|v| + dv) + |silu(g)| dv; exponential, quotient and products a few u: 8 u |y|.
  the output's rounding: half a step of its type, 2^-25 absolutely for fp16's subnormals.
  weights of a router: scores and quotients in 64 bits, one rounding: 2 u.
  sums of rows: (n_top + 2) u sum |terms|, and the rounding."""
import math

import numpy as np
import pytest
import torch

import gpu_util as G
from oracle import dense_oracle as O
from paper_2505_11076_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = {B.F16: torch.float16, B.BF16: torch.bfloat16, B.F32: torch.float32}
HALF = {B.F16: 2.0 ** -11, B.BF16: 2.0 ** -8, B.F32: 2.0 ** -24}
U = 2.0 ** -24
TABLE = None


def table():
    global TABLE
    if TABLE is None:
        TABLE = torch.from_numpy(O.E4M3).cuda()
    return TABLE


def up(n, to):
    return -(-n // to) * to


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Operand:
    """Rows in 8 or 16 bits at a stride with no numbers behind them, scales of all sizes, and what they stand for in 64 bits."""

    def __init__(self, rows, cols, dtype, g, block_rows=1, scale_type=B.E8M0, extra=0, groups=1):
        self.dtype, per = dtype, 16 if dtype == B.E4M3 else 8
        self.stride = up(cols, per) + extra * per
        shape = (groups, rows, cols)
        if dtype == B.E4M3:
            self.data = torch.full((groups, rows, self.stride), 0x7F, dtype=torch.uint8, device="cuda")
            codes = torch.randint(0, 256, shape, generator=g, device="cuda", dtype=torch.uint8)
            codes[(codes & 127) == 127] = 0x28
            self.data[..., :cols] = codes
            kb, nb = -(-cols // 128), -(-rows // block_rows)
            self.scale_stride = up(kb, 4) + 4 * extra if block_rows == 1 else kb + extra
            if scale_type == B.E8M0:
                self.scale = torch.randint(116, 130, (groups, nb, self.scale_stride), generator=g, device="cuda", dtype=torch.uint8)
                s = torch.exp2(self.scale.double() - 127).float().double()
            else:
                self.scale = torch.rand(groups, nb, self.scale_stride, generator=g, device="cuda") * 0.01 + 1e-4
                s = self.scale.double()
            s = s[..., :kb].repeat_interleave(block_rows, 1)[:, :rows].repeat_interleave(128, 2)[..., :cols]
            self.values = table()[codes.int()] * s
        else:
            self.data = torch.full((groups, rows, self.stride), float("nan"), dtype=TYPES[dtype], device="cuda")
            self.data[..., :cols] = torch.randn(shape, generator=g, device="cuda").to(TYPES[dtype])
            self.scale, self.scale_stride, self.values = None, 0, self.data[..., :cols].double()

    def scale_ptr(self):
        return 0 if self.scale is None else self.scale.data_ptr()


def product_and_bound(x, w, exact):
    """x w^T in 64 bits, and how far fp32 may be off; rows of x one by one."""
    K = x.shape[1]
    y, off = torch.matmul(x, w.t().contiguous()), torch.empty(x.shape[0], w.shape[0], dtype=torch.float64, device="cuda")
    pad = torch.nn.functional.pad
    w_abs = pad(w.abs().float(), (0, up(K, 16) - K))
    for i in range(x.shape[0]):
        p = pad(x[i].abs().float(), (0, up(K, 16) - K)) * w_abs
        off[i] = (K + 4) * U * p.sum(1).double()
        if not exact:
            off[i] += 16 * 2.0 ** -13 * p.view(w.shape[0], -1, 16).amax(2).sum(1).double()
    return y, off * (1 + 1e-5)


def expected(x, w, w_up, exact, out):
    y, off = product_and_bound(x, w, exact)
    if w_up is not None:
        v, off_v = product_and_bound(x, w_up, exact)
        s = y * torch.sigmoid(y)
        off = 1.1 * off * (v.abs() + off_v) + s.abs() * off_v + 8 * U * (s * v).abs()
        y = s * v
    off = off + HALF[out] * (y.abs() + off) + (2.0 ** -25 if out == B.F16 else 0)
    return y, off


def near(got, want, off, what):
    got = got.double()
    assert torch.isfinite(got).all(), what + ": not finite"
    far = ((got - want).abs() / off.clamp(min=1e-300)).max().item() if got.numel() else 0.0
    G.say("%s: %.3g of the bound" % (what, far))
    assert far <= 1, what


def run_dense(x, w, w_up, n_in, n_out, out, n_rows, x_rows=None, starts=None, scale_type=B.E8M0, y_extra=0, stream=None):
    y = torch.full((n_rows, n_out + y_extra), -77.0, dtype=TYPES[out], device="cuda")
    d = B.Dense(x=x.data.data_ptr(), x_scale=x.scale_ptr(), x_stride=x.stride, x_scale_stride=x.scale_stride, n_x_rows=x.data.shape[1], x_rows=0 if x_rows is None else x_rows.data_ptr(),
                w=w.data.data_ptr(), w_scale=w.scale_ptr(), w_stride=w.stride, w_scale_stride=w.scale_stride, w_group_stride=w.data.stride(0),
                w_scale_group_stride=0 if w.scale is None else w.scale.stride(0), w_scale_type=scale_type, w_up=0 if w_up is None else w_up.data.data_ptr(),
                w_up_scale=0 if w_up is None else w_up.scale_ptr(), y=y.data_ptr(), y_stride=n_out + y_extra, dtype=x.dtype, out_dtype=out, n_rows=n_rows, n_in=n_in, n_out=n_out,
                starts=0 if starts is None else starts.data_ptr(), n_groups=0 if starts is None else w.data.shape[0])
    f = B.dbf_dense_gemm if starts is None else B.dbf_grouped_gemm
    f(d, 0, 0, G.stream_handle() if stream is None else stream)
    return y


# rows, n_in, n_out: on the sides of the rules that choose a kernel, lengths that end inside a step, a piece, a byte behind one
SIZES = [(1, 1, 1), (1, 16, 16), (1, 128, 5), (3, 127, 33), (16, 129, 64), (2, 1000, 100), (16, 4096, 256), (17, 520, 70), (32, 1040, 130), (33, 300, 200), (64, 2048, 64), (65, 143, 129),
         (100, 640, 257), (129, 256, 300), (200, 1999, 100), (257, 384, 513), (300, 1, 40), (520, 900, 1100), (1030, 272, 520),
         (129, 16, 16), (130, 128, 5), (131, 143, 129), (150, 127, 33), (140, 1040, 130), (160, 300, 200), (192, 2048, 64)]
KINDS = [(B.E4M3, B.E8M0, B.F16), (B.E4M3, B.F32, B.BF16), (B.E4M3, B.E8M0, B.F32), (B.E4M3, B.F32, B.F32), (B.F16, B.E8M0, B.F16), (B.BF16, B.E8M0, B.F32)]


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "%d-%d-%d" % k)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "%dx%dx%d" % s)
def test_a_product(size, gated, kind):
    (rows, n_in, n_out), (dtype, scale_type, out) = size, kind
    g = gen(rows + 7 * n_in + 3 * n_out)
    x = Operand(rows, n_in, dtype, g, extra=rows % 2)
    w = [Operand(n_out, n_in, dtype, g, 128, scale_type, extra=n_out % 3) for _ in range(1 + gated)]
    if dtype == B.E4M3:
        for o in w:   # (gates of a size at which they are not all 0 or 1, outputs that fp16 holds)
            o.values *= 2.0 ** -8
            o.scale = o.scale - 8 if scale_type == B.E8M0 else o.scale * 2.0 ** -8
    what = "%d x %d -> %d, types %s%s" % (rows, n_in, n_out, kind, ", gated" if gated else "")
    G.say(what)
    y = run_dense(x, w[0], w[1] if gated else None, n_in, n_out, out, rows, scale_type=scale_type, y_extra=n_out % 2 * 3)
    torch.cuda.synchronize()
    want, off = expected(x.values[0], w[0].values[0], w[1].values[0] if gated else None, dtype != B.E4M3 or out == B.F32, out)
    keep = want.abs() < 60000   # (beyond fp16)
    near(torch.where(keep, y[:, :n_out].double(), 0), torch.where(keep, want, 0), off, what)
    assert (y[:, n_out:] == -77).all(), what


# few rows past 64 MB of weights and more: all lengths of a wavefront's part, the last of which ends inside a step
@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "%d-%d-%d" % k)
@pytest.mark.parametrize("rows,bytes_in,n_out,gated", [(1, 1024, 66000, False), (16, 1040, 65000, False), (5, 2048, 32801, False), (7, 2064, 16500, True), (3, 4096, 16389, False),
                                                       (2, 4080, 8240, True), (16, 8192, 8215, False), (9, 6544, 10300, False), (4, 8176, 4111, True), (1, 992, 33900, True)])
def test_weights_that_stream(rows, bytes_in, n_out, gated, kind):
    dtype, scale_type, out = kind
    n_in = bytes_in if dtype == B.E4M3 else bytes_in // 2
    g = gen(rows + bytes_in)
    x = Operand(rows, n_in, dtype, g)
    w = [Operand(n_out, n_in, dtype, g, 128, scale_type) for _ in range(1 + gated)]
    if dtype == B.E4M3:
        for o in w:
            o.values *= 2.0 ** -8
            o.scale = o.scale - 8 if scale_type == B.E8M0 else o.scale * 2.0 ** -8
    what = "%d rows past %d x %d, types %s%s" % (rows, n_out, n_in, kind, ", gated" if gated else "")
    G.say(what)
    y = run_dense(x, w[0], w[1] if gated else None, n_in, n_out, out, rows, scale_type=scale_type)
    torch.cuda.synchronize()
    want, off = expected(x.values[0], w[0].values[0], w[1].values[0] if gated else None, dtype != B.E4M3 or out == B.F32, out)
    keep = want.abs() < 60000
    near(torch.where(keep, y.double(), 0), torch.where(keep, want, 0), off, what)


def split(rows, groups, g):
    """Rows of each group: some empty, one with many."""
    if groups == 1:
        return [rows]
    share = torch.rand(groups, generator=g, device="cuda") ** 4
    share[torch.rand(groups, generator=g, device="cuda") < 0.3] = 0
    share[groups // 2] += 0.5
    cut = torch.round(share.cumsum(0) / share.sum() * rows).long().tolist()
    return [b - a for a, b in zip([0] + cut, cut)]


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: "%d-%d-%d" % k)
@pytest.mark.parametrize("rows,groups,n_in,n_out,gated,gathered", [(1, 1, 64, 17, False, False), (8, 64, 512, 96, True, True), (50, 16, 333, 129, True, True), (200, 5, 1000, 65, False, False),
                                                                   (700, 60, 272, 300, False, True), (700, 3, 700, 130, True, False), (1500, 4, 512, 520, True, True), (40, 1000, 144, 40, False, True),
                                                                   (64, 70, 2048, 512, True, True), (600, 4, 333, 129, True, True), (900, 6, 1000, 65, False, False), (1100, 8, 144, 40, False, True),
                                                                   (270, 2, 64, 17, False, False), (2000, 12, 272, 300, True, True)])
def test_a_product_by_groups(rows, groups, n_in, n_out, gated, gathered, kind):
    dtype, scale_type, out = kind
    g = gen(rows + groups)
    n_x = 37 if gathered else rows + 9
    x = Operand(n_x, n_in, dtype, g)
    w = [Operand(n_out, n_in, dtype, g, 128, scale_type, groups=groups) for _ in range(1 + gated)]
    if dtype == B.E4M3:
        for o in w:
            o.values *= 2.0 ** -8
            o.scale = o.scale - 8 if scale_type == B.E8M0 else o.scale * 2.0 ** -8
    before, behind = 2, 5   # rows of no group
    each = split(rows, groups, g)
    starts = torch.tensor([before] + [before + sum(each[: i + 1]) for i in range(groups)], dtype=torch.int32, device="cuda")
    n_rows = before + rows + behind
    x_rows = None
    if gathered:
        x_rows = torch.randint(0, n_x, (n_rows,), generator=g, device="cuda", dtype=torch.int32)
        x_rows[before + rows // 2] = -1 if rows > 1 else 0
        x_rows[n_rows - 1] = 1 << 30
        if rows > 9:
            x_rows[before + 3] = n_x
    else:
        n_rows = min(n_rows, n_x)
    what = "%d rows of %d groups, %d -> %d, types %s" % (rows, groups, n_in, n_out, kind)
    G.say(what)
    y = run_dense(x, w[0], w[1] if gated else None, n_in, n_out, out, n_rows, x_rows, starts, scale_type, y_extra=1)
    torch.cuda.synchronize()
    assert (y[:before] == -77).all() and (y[before + rows:] == -77).all() and (y[:, n_out:] == -77).all(), what
    at = before
    for i, m in enumerate(each):
        if not m:
            continue
        take = x_rows[at: at + m].long() if gathered else torch.arange(at, at + m, device="cuda")
        none = (take < 0) | (take >= n_x)
        xs = x.values[0][take.clamp(0, n_x - 1)]
        xs = torch.where(none[:, None], torch.zeros_like(xs), xs)
        want, off = expected(xs, w[0].values[i], w[1].values[i] if gated else None, dtype != B.E4M3 or out == B.F32, out)
        keep = want.abs() < 60000
        near(torch.where(keep, y[at: at + m, :n_out].double(), 0), torch.where(keep, want, 0), off, "%s, group %d" % (what, i))
        assert (y[at: at + m, :n_out][none] == 0).all()
        at += m


@pytest.mark.parametrize("rows,n_out", [(4, 33), (40, 33), (300, 130), (2, 66000)])
@pytest.mark.parametrize("kind", [KINDS[0], KINDS[3], KINDS[4]], ids=lambda k: "%d-%d-%d" % k)
def test_no_numbers_stay_where_they_are(rows, n_out, kind):
    dtype, scale_type, out = kind
    n_in = 1024 if n_out > 1000 else 300
    g = gen(rows)
    x, w = Operand(rows, n_in, dtype, g), Operand(n_out, n_in, dtype, g, 128, scale_type)
    bad = 0x7F if dtype == B.E4M3 else float("nan")
    x.data[0, rows // 2, n_in - 1] = bad
    w.data[0, 17, 0] = bad
    y = run_dense(x, w, None, n_in, n_out, B.F32, rows, scale_type=scale_type)
    torch.cuda.synchronize()
    want = torch.zeros(rows, n_out, dtype=torch.bool, device="cuda")
    want[rows // 2], want[:, 17] = True, True
    assert torch.equal(torch.isnan(y), want)
    if dtype == B.E4M3 and scale_type == B.E8M0:   # a scale that is no number
        x, w = Operand(rows, n_in, dtype, g), Operand(n_out, n_in, dtype, g, 128, scale_type)
        x.scale[0, 1, 1] = 255
        w.scale[0, 0, 2] = 255
        for out in (B.F16, B.F32):
            y = run_dense(x, w, None, n_in, n_out, out, rows, scale_type=scale_type)
            torch.cuda.synchronize()
            want = torch.zeros(rows, n_out, dtype=torch.bool, device="cuda")
            want[1], want[:, :128] = True, True
            assert torch.equal(torch.isnan(y), want)


def test_the_smallest_and_largest_scales():
    for out in (B.F32, B.F16):
        for rows in (3, 70):
            g = gen(rows)
            x, w = Operand(rows, 128, B.E4M3, g), Operand(20, 128, B.E4M3, g, 128)
            v = table()[x.data[0, :, :128].int()] @ table()[w.data[0, :, :128].int()].t().contiguous()
            for a, b in ((0, 240), (240, 0), (1, 253), (100, 140)):
                x.scale[:], w.scale[:] = a, b
                y = run_dense(x, w, None, 128, 20, out, rows)
                torch.cuda.synchronize()
                want = v * 2.0 ** (a + b - 254)
                off = 16 * 2.0 ** -13 * 8 * 448 * 448 * 2.0 ** (a + b - 254) + HALF[out] * want.abs() + (2.0 ** -25 if out == B.F16 else 2.0 ** -149)
                keep = want.abs() < (60000 if out == B.F16 else 3e38)   # (65520 and more round to infinity in fp16)
                assert torch.isfinite(y[keep]).all() and (((y.double() - want).abs() <= off) | ~keep).all(), (out, rows, a, b)


def test_the_smallest_and_largest_scales_of_32_bits():
    """Scales of rows and of weights that meet within fp32, though a sum with one of them does not; a scale of 0."""
    for out in (B.F32, B.F16):
        for rows, n_out in ((3, 20), (70, 20), (2, 66000)):
            n_in = 1024 if n_out > 20 else 128
            g = gen(rows)
            x, w = Operand(rows, n_in, B.E4M3, g), Operand(n_out, n_in, B.E4M3, g, 128, B.F32)
            v = table()[x.data[0, :, :n_in].int()] @ table()[w.data[0, :, :n_in].int()].t().contiguous()
            for a, b in ((0, 1.3 * 2.0 ** 112), (240, 1.7 * 2.0 ** -126), (127, 0.0), (247, 1e-36), (100, 3.1e7)):
                x.scale[:], w.scale[:] = a, b
                y = run_dense(x, w, None, n_in, n_out, out, rows, scale_type=B.F32)
                torch.cuda.synchronize()
                s = 2.0 ** (a - 127) * float(np.float32(b))
                want = v * s
                off = 16 * 2.0 ** -13 * (n_in / 16) * 448 * 448 * s + HALF[out] * want.abs() + (2.0 ** -25 if out == B.F16 else 2.0 ** -149)
                keep = want.abs() < (60000 if out == B.F16 else 3e38)
                assert torch.isfinite(y[keep]).all() and (((y.double() - want).abs() <= off) | ~keep).all(), (out, rows, a, b)


def test_groups_whose_rows_are_not_there():
    """Starts that fall, that lie outside, that are all the same: rows are held to those of y, what is no group's is left alone."""
    g = gen(5)
    x, w = Operand(60, 144, B.E4M3, g), Operand(48, 144, B.E4M3, g, 128, groups=4)
    for starts, rows in (([-9, 10, 5, 30, 1 << 30], {0: (0, 10), 2: (5, 30), 3: (30, 60)}), ([60, 0, 0, 0, 0], {}), ([7, 7, 7, 7, 7], {}), ([-(1 << 31), -5, 0, 100, 90], {2: (0, 60)})):
        y = run_dense(x, w, None, 144, 48, B.F32, 60, starts=torch.tensor(starts, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        members = torch.zeros(60, dtype=torch.int32, device="cuda")
        for a, b in rows.values():
            members[a:b] += 1
        for i, (a, b) in rows.items():
            once = members[a:b] == 1   # (what a row of two groups holds is not said)
            want, off = expected(x.values[0][a:b], w.values[i], None, True, B.F32)
            near(y[a:b][once], want[once], off[once], "%s, group %d" % (starts, i))
        assert (y[members == 0] == -77).all()


def test_rows_and_groups_beyond_4_gib():
    g = gen(1)
    # weights of the second group 5 GB behind the first
    gap = 5 << 30
    x = Operand(40, 256, B.E4M3, g)
    w = Operand(64, 256, B.E4M3, g, 128, groups=2)
    far = torch.empty(gap + 64 * 256, dtype=torch.uint8, device="cuda")
    for i in range(2):
        far[i * gap: i * gap + 64 * 256] = w.data[i].flatten()
    starts = torch.tensor([0, 15, 40], dtype=torch.int32, device="cuda")
    real, w.data = w.data, far.view(1, -1).expand(2, -1)
    y = torch.empty(40, 64, dtype=torch.float32, device="cuda")
    d = dict(x=x.data.data_ptr(), x_scale=x.scale_ptr(), x_stride=256, x_scale_stride=4, n_x_rows=40, w=far.data_ptr(), w_scale=w.scale_ptr(), w_stride=256, w_scale_stride=2, w_group_stride=gap,
             w_scale_group_stride=2, y=y.data_ptr(), y_stride=64, dtype=B.E4M3, out_dtype=B.F32, w_scale_type=B.E8M0, n_rows=40, n_in=256, n_out=64, n_groups=2, starts=starts.data_ptr())
    B.dbf_grouped_gemm(B.Dense(**d), 0, 0, G.stream_handle())
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(((0, 15), (15, 40))):
        want, off = expected(x.values[0][a:b], w.values[i], None, True, B.F32)
        near(y[a:b], want, off, "group %d" % i)
    # rows of x and of y further apart than 32 bits count: tiles behind the first 4 GiB
    del far
    stride, n = 1 << 22, 1100
    wide = torch.zeros(n * stride, dtype=torch.uint8, device="cuda").view(n, stride)
    x = Operand(n, 256, B.E4M3, g)
    wide[:, :256] = x.data[0, :, :256]
    y = torch.empty(n, 64, dtype=torch.float32, device="cuda")
    d |= dict(x=wide.data_ptr(), x_stride=stride, x_scale=x.scale_ptr(), n_x_rows=n, n_rows=n, w=real.data_ptr(), y=y.data_ptr(), n_groups=0, starts=0)
    B.dbf_dense_gemm(B.Dense(**d), 0, 0, G.stream_handle())
    torch.cuda.synchronize()
    want, off = expected(x.values[0], w.values[0], None, True, B.F32)
    near(y, want, off, "rows 4 MiB apart")


# ---- rounding to 8 bits ---------------------------------------------------------------------------------------


def test_more_small_tiles_than_a_launch_has_workgroups_for():
    """1024 rows of as many groups through 2^20 outputs: 32768 workgroups of outputs, of which a launch has 256 times as many at most; group g's weights begin 8 g rows in."""
    g, groups, n_out, n_in = gen(53), 1024, 1 << 20, 12
    x = Operand(groups, n_in, B.F16, g)
    w = Operand(n_out + 8 * (groups - 1), n_in, B.F16, g)
    starts = torch.arange(groups + 1, dtype=torch.int32, device="cuda")
    y = torch.full((groups, n_out), float("nan"), dtype=torch.float16, device="cuda")
    d = B.Dense(x=x.data.data_ptr(), x_stride=x.stride, n_x_rows=groups, w=w.data.data_ptr(), w_stride=w.stride, w_group_stride=8 * w.stride, y=y.data_ptr(), y_stride=n_out, dtype=B.F16,
                out_dtype=B.F16, n_rows=groups, n_in=n_in, n_out=n_out, starts=starts.data_ptr(), n_groups=groups)
    B.dbf_grouped_gemm(d, 0, 0, G.stream_handle())
    torch.cuda.synchronize()
    for part in y.split(64):
        assert torch.isfinite(part).all()
    cols = torch.cat([torch.randint(0, n_out, (200,), generator=g, device="cuda"), torch.tensor([0, 15, 16, n_out - 17, n_out - 1], device="cuda")])
    for r in range(groups):
        want, off = expected(x.values[0, r : r + 1], w.values[0, 8 * r + cols], None, True, B.F16)
        far = ((y[r, cols].double() - want[0]).abs() / off[0]).max().item()
        assert far <= 1, (r, far)


@pytest.mark.parametrize("dtype", [B.F16, B.BF16, B.F32])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,extra", [(1, 1, 0), (1, 128, 3), (7, 130, 0), (33, 1000, 1), (129, 257, 7), (300, 640, 0), (128, 16, 0), (2, 5000, 13)])
def test_rounding_to_8_bits(rows, cols, extra, block_rows, dtype):
    rng = np.random.default_rng(rows * cols)
    x = rng.normal(size=(rows, cols)) * np.exp(3 * rng.normal(size=(rows, 1))) * np.exp(rng.normal(size=cols))
    x[0, 0] = 0
    if rows > 3:
        x[1] = 0
        x[2] = rng.choice([448.0, -448.0, 224.0, 0.4375, 2.0 ** -9, 3 * 2.0 ** -10, 2.0 ** -10, 1e-7], cols)   # borders of scales and of codes
        x[3] = 448.0 * 1.002 * rng.choice([1, -1, 0.001], cols)
    if rows > 40 and dtype != B.F16:
        x[40] *= 1e-39 if dtype == B.F32 else 1e-36
        x[30] *= 1e34
    if rows > 128:
        x[-1, cols // 2], x[17, -1] = np.inf, np.nan
    t = torch.full((rows, cols + extra), 3.0, dtype=TYPES[dtype], device="cuda")
    t[:, :cols] = torch.from_numpy(x).cuda().to(TYPES[dtype])
    codes = torch.full((rows, up(cols, 16) + 16), 0x55, dtype=torch.uint8, device="cuda")
    kb = -(-cols // 128)
    scales = torch.full((-(-rows // block_rows), kb + 2), 0x66, dtype=torch.uint8, device="cuda")
    B.dbf_quantize(t.data_ptr(), dtype, cols + extra, rows, cols, block_rows, codes.data_ptr(), codes.shape[1], scales.data_ptr(), scales.shape[1], G.stream_handle())
    torch.cuda.synchronize()
    want, want_scales = O.quantize(t[:, :cols].double().cpu().numpy(), block_rows)
    got = codes.cpu().numpy()
    assert np.array_equal(scales.cpu().numpy()[:, :kb], want_scales) and (scales[:, kb:] == 0x66).all()
    a, b = got[:, :cols], want
    same = (a == b) | ((a & 127 == 0) & (b & 127 == 0))   # (a zero of either sign)
    assert same.all(), np.argwhere(~same)[:5]
    assert (got[:, cols: up(cols, 16)] == 0).all() and (got[:, up(cols, 16):] == 0x55).all()


# ---- routing ----------------------------------------------------------------------------------------------------


def run_route(x, n_top, sigmoid, bias, renormalise, scale, ws=None):
    T, E = x.shape
    ints = lambda *s: torch.full(s, -99, dtype=torch.int32, device="cuda")  # noqa: E731
    out = [ints(T, n_top), torch.full((T, n_top), -9.0, device="cuda"), ints(E + 1), ints(T * n_top), ints(T, n_top)]
    r = B.Router(logits=x.data_ptr(), row_stride=x.stride(0), bias=0 if bias is None else bias.data_ptr(), expert_ids=out[0].data_ptr(), weights=out[1].data_ptr(), starts=out[2].data_ptr(),
                 row_token=out[3].data_ptr(), token_rows=out[4].data_ptr(), dtype={v: k for k, v in TYPES.items()}[x.dtype], n_tokens=T, n_experts=E, n_top=n_top,
                 score=B.SCORE_SIGMOID if sigmoid else B.SCORE_SOFTMAX, renormalise=int(renormalise), scale=scale)
    size = B.dbf_route_workspace_bytes(r)
    ws = torch.full((max(size, 256),), 0xA5, dtype=torch.uint8, device="cuda")
    B.dbf_route(r, ws.data_ptr(), size, G.stream_handle())
    return out


@pytest.mark.parametrize("T,E,n_top,dtype,sigmoid,biased,renormalise", [
    (1, 1, 1, B.F32, False, False, True), (1, 64, 6, B.BF16, False, False, False), (2, 64, 32, B.F32, True, False, True), (31, 5, 2, B.F16, False, True, True), (32, 65, 8, B.BF16, True, True, False),
    (33, 128, 17, B.F32, False, False, True), (70, 129, 4, B.F16, True, False, False), (200, 256, 8, B.F32, True, True, True), (65, 257, 3, B.F32, False, True, False), (40, 1000, 32, B.BF16, False, False, True),
    (3, 1024, 20, B.F32, True, True, True), (700, 33, 1, B.F16, False, False, False)])
def test_a_router(T, E, n_top, dtype, sigmoid, biased, renormalise):
    g = gen(T + E)
    x = (2 * torch.randn(T, E + 3, generator=g, device="cuda")).to(TYPES[dtype])
    v = x[:, :E]
    v[torch.rand(T, E, generator=g, device="cuda") < 0.05] = float("-inf")
    v[torch.rand(T, E, generator=g, device="cuda") < 0.02] = float("nan")
    if T > 1:
        v[-1] = float("-inf")
    if T > 30:
        v[3] = 1.0                                     # ties
        v[4] = float("-inf")
        v[4, E // 2] = -5.0                            # one left
        v[5, : E // 2 + 1] = float("inf")
        v[6] = -60000.0
        v[7] = torch.where(torch.arange(E, device="cuda") % 2 == 0, 0.0, -0.0).to(v.dtype)
    bias = None
    if biased:
        bias = 0.3 * torch.randn(E, generator=g, device="cuda")
        bias[E - 1], bias[0] = float("-inf"), float("nan")
    scale = 1.0 if renormalise else 2.5
    G.say("%d tokens, %d of %d experts" % (T, n_top, E))
    got = run_route(x[:, :E], n_top, sigmoid, bias, renormalise, scale)
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        want = O.route(np.where(np.isnan(v.double().cpu().numpy()), -np.inf, v.double().cpu().numpy()), n_top, sigmoid, None if bias is None else np.where(np.isnan(bias.cpu().numpy()), -np.inf, bias.cpu().numpy()), renormalise, scale)
    for k in (0, 2, 3, 4):
        assert np.array_equal(got[k].cpu().numpy(), want[k]), "output %d" % k
    assert np.all(np.abs(got[1].cpu().numpy() - want[1]) <= 2 * U * np.abs(want[1]) + 2.0 ** -149)


@pytest.mark.parametrize("T", [64, 8192, 8193, 20011])
def test_many_tokens_are_put_in_order(T):
    """The order alone, against a stable sort: counts added up in one launch or in two."""
    g = gen(T)
    x = torch.randn(T, 48, generator=g, device="cuda")
    x[torch.rand(T, generator=g, device="cuda") < 0.1] = float("-inf")
    ids, weights, starts, row_token, token_rows = run_route(x, 4, False, None, True, 1.0)
    torch.cuda.synchronize()
    top = torch.topk(x, 4, 1)
    assert torch.equal(ids.long(), torch.where(top.values > float("-inf"), top.indices, -1))
    flat = torch.where(ids >= 0, ids, 48).flatten().long()
    key, order = torch.sort(flat, stable=True)
    n = int((flat < 48).sum())
    assert torch.equal(starts.long(), torch.searchsorted(key, torch.arange(49, device="cuda")))
    assert torch.equal(row_token[:n].long(), order[:n] // 4) and (row_token[n:] == -1).all()
    rows = torch.full_like(flat, -1)
    rows[order[:n]] = torch.arange(n, device="cuda")
    assert torch.equal(token_rows.flatten().long(), rows)


def test_a_router_without_tokens_has_no_rows():
    starts = torch.full((66,), 7, dtype=torch.int32, device="cuda")
    B.dbf_route(B.Router(logits=starts.data_ptr(), row_stride=64, expert_ids=starts.data_ptr(), weights=starts.data_ptr(), starts=starts.data_ptr(), row_token=starts.data_ptr(),
                         token_rows=starts.data_ptr(), dtype=B.F32, n_tokens=0, n_experts=64, n_top=2, scale=1.0), 0, 0, G.stream_handle())
    torch.cuda.synchronize()
    assert starts.tolist() == [0] * 65 + [7]


# ---- rows back to their tokens ------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [B.F16, B.BF16, B.F32])
@pytest.mark.parametrize("T,n_top,cols,extra,residual", [(1, 1, 1, 0, False), (5, 3, 64, 0, True), (9, 8, 1000, 0, False), (33, 2, 77, 2, True), (200, 6, 512, 8, True), (3, 32, 24, 4, False)])
def test_a_sum_of_rows(T, n_top, cols, extra, residual, dtype):
    g = gen(T * cols)
    n = T * n_top
    make = lambda r: torch.randn(r, cols + extra, generator=g, device="cuda").to(TYPES[dtype])  # noqa: E731
    rows, res = make(n), make(T) if residual else None
    at = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(T, n_top)
    weights = torch.rand(T, n_top, generator=g, device="cuda")
    if T > 2:
        at[0, 0], at[1, 0], at[2] = -1, n, -5
        weights[2] = float("nan")          # (of no row)
    out = res.clone() if residual else torch.full((T, cols + extra), 5.0, dtype=TYPES[dtype], device="cuda")
    B.dbf_combine(B.Combine(rows=rows.data_ptr(), token_rows=at.data_ptr(), weights=weights.data_ptr(), residual=out.data_ptr() if residual else 0, out=out.data_ptr(), row_stride=cols + extra,
                            residual_stride=cols + extra, out_stride=cols + extra, dtype=dtype, n_rows=n, n_tokens=T, n_top=n_top, n_cols=cols), G.stream_handle())
    torch.cuda.synchronize()
    r, w = rows[:, :cols].double().cpu().numpy(), weights.cpu().numpy()
    base = None if res is None else res[:, :cols].double().cpu().numpy()
    want = O.combine(r, at.tolist(), w, base)
    size = O.combine(np.abs(r), at.tolist(), w, None if base is None else np.abs(base))
    off = (n_top + 2) * U * size + HALF[dtype] * np.abs(want) * (1 + 1e-5) + (2.0 ** -25 if dtype == B.F16 else 0)
    assert np.all(np.abs(out[:, :cols].double().cpu().numpy() - want) <= off)
    if extra:
        assert torch.equal(out[:, cols:], res[:, cols:]) if residual else (out[:, cols:] == 5).all()


# ---- together, on other streams, captured ---------------------------------------------------------------------------


class Experts:
    """A layer of experts as a program runs it: choice, rounding, both products, sum; fixed buffers."""

    def __init__(self, T, hidden, inner, E, n_top, seed):
        g = gen(seed)
        self.T, self.hidden, self.inner, self.E, self.n_top = T, hidden, inner, E, n_top
        e = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.x, self.logits = e(T, hidden, dtype=torch.bfloat16), e(T, E, dtype=torch.float32)
        self.w = [Operand(n, k, B.E4M3, g, 128, B.E8M0, groups=E) for n, k in ((inner, hidden), (inner, hidden), (hidden, inner))]
        for o in self.w:
            o.values *= 2.0 ** -9
            o.scale -= 9
        R = T * n_top
        self.ids, self.weights, self.starts, self.row_token, self.token_rows = e(T, n_top), e(T, n_top, dtype=torch.float32), e(E + 1), e(R), e(T, n_top)
        u8 = torch.uint8
        self.xq, self.xs = e(T, up(hidden, 16), dtype=u8), e(T, up(-(-hidden // 128), 4), dtype=u8)
        self.h, self.hq, self.hs = e(R, inner, dtype=torch.bfloat16), e(R, up(inner, 16), dtype=u8), e(R, up(-(-inner // 128), 4), dtype=u8)
        self.rows, self.out = e(R, hidden, dtype=torch.bfloat16), e(T, hidden, dtype=torch.bfloat16)
        self.router = B.Router(logits=self.logits.data_ptr(), row_stride=E, expert_ids=self.ids.data_ptr(), weights=self.weights.data_ptr(), starts=self.starts.data_ptr(),
                               row_token=self.row_token.data_ptr(), token_rows=self.token_rows.data_ptr(), dtype=B.F32, n_tokens=T, n_experts=E, n_top=n_top, renormalise=1, scale=1.0)
        self.ws = torch.empty(max(256, B.dbf_route_workspace_bytes(self.router)), dtype=u8, device="cuda")
        self.up_gate = self.product(self.w[0], self.w[1], self.xq, self.xs, T, self.row_token, self.h, hidden, inner)
        self.down = self.product(self.w[2], None, self.hq, self.hs, R, None, self.rows, inner, hidden)
        self.sum = B.Combine(rows=self.rows.data_ptr(), token_rows=self.token_rows.data_ptr(), weights=self.weights.data_ptr(), residual=self.x.data_ptr(), out=self.out.data_ptr(),
                             row_stride=hidden, residual_stride=hidden, out_stride=hidden, dtype=B.BF16, n_rows=R, n_tokens=T, n_top=n_top, n_cols=hidden)

    def product(self, w, w_up, x, xs, n_x, x_rows, y, n_in, n_out):
        return B.Dense(x=x.data_ptr(), x_scale=xs.data_ptr(), x_stride=x.shape[1], x_scale_stride=xs.shape[1], n_x_rows=n_x, x_rows=0 if x_rows is None else x_rows.data_ptr(), w=w.data.data_ptr(),
                       w_scale=w.scale.data_ptr(), w_up=0 if w_up is None else w_up.data.data_ptr(), w_up_scale=0 if w_up is None else w_up.scale.data_ptr(), w_stride=w.stride,
                       w_group_stride=w.data.stride(0), w_scale_stride=w.scale_stride, w_scale_group_stride=w.scale.stride(0), y=y.data_ptr(), y_stride=n_out, dtype=B.E4M3, out_dtype=B.BF16,
                       w_scale_type=B.E8M0, n_rows=self.T * self.n_top, n_in=n_in, n_out=n_out, n_groups=self.E, starts=self.starts.data_ptr())

    def run(self):
        s, R = torch.cuda.current_stream().cuda_stream, self.T * self.n_top
        B.dbf_route(self.router, self.ws.data_ptr(), self.ws.numel(), s)
        B.dbf_quantize(self.x.data_ptr(), B.BF16, self.hidden, self.T, self.hidden, 1, self.xq.data_ptr(), self.xq.shape[1], self.xs.data_ptr(), self.xs.shape[1], s)
        B.dbf_grouped_gemm(self.up_gate, 0, 0, s)
        B.dbf_quantize(self.h.data_ptr(), B.BF16, self.inner, R, self.inner, 1, self.hq.data_ptr(), self.hq.shape[1], self.hs.data_ptr(), self.hs.shape[1], s)
        B.dbf_grouped_gemm(self.down, 0, 0, s)
        B.dbf_combine(self.sum, s)
        return self.out

    def new_inputs(self, seed, padded=0):
        g = gen(seed)
        self.x.copy_(torch.randn(self.T, self.hidden, generator=g, device="cuda"))
        self.logits.copy_(torch.randn(self.T, self.E, generator=g, device="cuda"))
        if padded:
            self.logits[-padded:] = float("-inf")

    def expected(self):
        """In 64 bits, roundings to 8 bits among them: of x; of what the first product made, as it lies there (a value next to a border may fall to either side)."""
        x = self.x.double().cpu().numpy()
        xv = O.values(*O.quantize(x, 1), 1)
        ids, weights, starts, row_token, token_rows = O.route(self.logits.double().cpu().numpy(), self.n_top, False)
        h = self.h.double().cpu().numpy()
        rows, first = np.zeros((len(row_token), self.hidden)), np.zeros((len(row_token), self.inner))
        hv = O.values(*O.quantize(h, 1), 1)
        for e in range(self.E):
            at = np.s_[starts[e]: starts[e + 1]]
            w = [o.values[e].cpu().numpy() for o in self.w]
            xe = xv[row_token[at]]
            first[at] = O.silu(xe @ w[0].T) * (xe @ w[1].T)
            rows[at] = hv[at] @ w[2].T
        return first, O.combine(rows, token_rows, weights, x), starts[-1]


@pytest.mark.parametrize("T,padded", [(1, 0), (7, 2), (45, 0), (300, 60)])
def test_a_layer_of_experts(T, padded):
    layer = Experts(T, 256, 160, 12, 3, T)
    layer.new_inputs(T, padded)
    out = layer.run()
    torch.cuda.synchronize()
    first, want, n = layer.expected()
    # relative to the size of all (errors of a product are, not of each value): bf16's half step, the instructions' 2^-13 of the largest, and the second rounding
    size = lambda a: np.linalg.norm(a) / math.sqrt(max(a.size, 1))  # noqa: E731
    h = layer.h.double().cpu().numpy()[:n]
    assert np.linalg.norm(h - first[:n]) <= 2.0 ** -8 * np.linalg.norm(first[:n])
    assert np.linalg.norm(out.double().cpu().numpy() - want) <= 2.0 ** -7 * np.linalg.norm(want)
    if padded:
        assert torch.equal(out[-padded:], layer.x[-padded:]), "tokens without experts keep what they had"
    assert size(want) > 0


def test_captured_and_replayed_over_other_inputs():
    """Two graphs of the same buffers, replayed in turn with eager work between, against eager results."""
    layer = Experts(40, 256, 160, 12, 3, 3)
    side = torch.cuda.Stream()
    layer.new_inputs(0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.run()
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            layer.run()
    for i in range(6):
        layer.new_inputs(100 + i, padded=i * 5)
        layer.run()
        torch.cuda.synchronize()
        want = [layer.out.clone(), layer.starts.clone(), layer.ids.clone()]
        for t in (layer.out, layer.starts, layer.h, layer.row_token, layer.ids):
            t.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [layer.out, layer.starts, layer.ids])), i


def test_two_streams_at_once_and_the_same_bits_each_time():
    layers = [Experts(90, 256, 160, 12, 3, s) for s in (1, 2)]
    want = []
    for i, layer in enumerate(layers):
        layer.new_inputs(i)
        layer.run()
        torch.cuda.synchronize()
        want.append(layer.out.clone())
    streams = [torch.cuda.Stream() for _ in layers]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for layer, s in zip(layers, streams):
            with torch.cuda.stream(s):
                layer.out.zero_()
                layer.run()
    torch.cuda.synchronize()
    assert all(torch.equal(layer.out, w) for layer, w in zip(layers, want))


def test_a_head_in_8_bits_before_log_probabilities():
    """Rows rounded, the head's product, log probabilities of given tokens: the last steps of a pass."""
    g = gen(9)
    rows, hidden, vocab = 5, 256, 1003
    x = torch.randn(rows, hidden, generator=g, device="cuda").half()
    w = torch.randn(vocab, hidden, generator=g, device="cuda") / 16
    codes, scales = torch.empty(vocab, hidden, dtype=torch.uint8, device="cuda"), torch.empty(8, 2, dtype=torch.uint8, device="cuda")
    xq, xs = torch.empty(rows, hidden, dtype=torch.uint8, device="cuda"), torch.empty(rows, 4, dtype=torch.uint8, device="cuda")
    s = G.stream_handle()
    B.dbf_quantize(w.data_ptr(), B.F32, hidden, vocab, hidden, 128, codes.data_ptr(), hidden, scales.data_ptr(), 2, s)
    B.dbf_quantize(x.data_ptr(), B.F16, hidden, rows, hidden, 1, xq.data_ptr(), hidden, xs.data_ptr(), 4, s)
    logits = torch.empty(rows, vocab, device="cuda")
    B.dbf_dense_gemm(B.Dense(x=xq.data_ptr(), x_scale=xs.data_ptr(), x_stride=hidden, x_scale_stride=4, n_x_rows=rows, w=codes.data_ptr(), w_scale=scales.data_ptr(), w_stride=hidden, w_scale_stride=2,
                             y=logits.data_ptr(), y_stride=vocab, dtype=B.E4M3, out_dtype=B.F32, w_scale_type=B.E8M0, n_rows=rows, n_in=hidden, n_out=vocab), 0, 0, s)
    targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    lp = torch.empty(rows, device="cuda")
    ws = torch.empty(max(256, B.dbf_token_logprobs_workspace_bytes(rows, vocab, 0)), dtype=torch.uint8, device="cuda")
    B.dbf_token_logprobs(logits.data_ptr(), B.F32, vocab, rows, vocab, targets.data_ptr(), 0, lp.data_ptr(), 0, 0, 0, ws.data_ptr(), ws.numel(), s)
    torch.cuda.synchronize()
    xv = O.values(*O.quantize(x.double().cpu().numpy(), 1), 1)
    wv = O.values(*O.quantize(w.double().cpu().numpy(), 128), 128)
    y = xv @ wv.T
    want = y[np.arange(rows), targets.cpu().numpy()] - np.log(np.exp(y - y.max(1, keepdims=True)).sum(1)) - y.max(1)
    # logits within (K + 4) u sum |x w|, log probabilities of numbers of some ten within 2^-18 of them
    off = 2 * (hidden + 4) * U * (np.abs(xv) @ np.abs(wv).T).max() + 2.0 ** -18 * np.abs(want)
    assert np.all(np.abs(lp.double().cpu().numpy() - want) <= off)
