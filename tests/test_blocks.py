"""Rows in 8-bit floating point with a scale for each block of 128, and their products, against plain 64-bit implementations.

Rows in 8 bits have to be exact.  Products: u = 2^-24 is half a step of float32, T(t) half a step of the output's type.  The tensor cores add up a block's products with an error below
2^-20 of the sum of their sizes (measured 2^-21.8 at most over random bits, normal and positive values); scaling a block is two roundings, adding kb of
them at most kb + 16 more (the blocks of one sum may be dealt to as many as 16 partial sums), bias one.
"""
import ctypes as C
import os
import subprocess
import sys

import pytest
import torch

from paper_1712_01670_b200 import binding as B

U = 2.0 ** -24
BLOCK = 128
E4M3 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
gpu = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def up(n, to=BLOCK):
    return -(-n // to)


def bytes_like(rows, k, extra=0):
    """Rows of 8-bit values, all bits of the rest set to a NaN's."""
    return torch.full((rows, up(k, 16) * 16 + extra), 0x7F, dtype=torch.uint8, device="cuda").view(E4M3)[:, :k]


def bits(t):
    return t.contiguous().view(torch.uint8)


def e4m3(v):
    """The value of the type next to v (64 bits, |v| <= 448), halves to even."""
    _, e = torch.frexp(v)
    step = torch.exp2(torch.clamp(e.double() - 4, min=-9))
    return torch.round(v / step) * step


def quantize64(x, block_rows):
    """(q, scale) of x; NaN and infinity: scale NaN, zeros"""
    rows, k = x.shape
    rb, kb = up(rows, block_rows), up(k)
    p = torch.zeros(rb * block_rows, kb * BLOCK, dtype=torch.float64, device="cuda")
    p[:rows, :k] = x.double()
    t = p.view(rb, block_rows, kb, BLOCK)
    most = t.abs().amax((1, 3))
    bad = ~torch.isfinite(t).all(3).all(1)
    m, e = torch.frexp(torch.where(bad, torch.ones_like(most), most))
    scale = torch.exp2(torch.clamp(e.double() - 9 + (m > 0.875), min=-126.0))
    q = e4m3(t / scale[:, None, :, None])
    q = torch.where(bad[:, None, :, None], torch.zeros_like(q), q)
    scale = torch.where(most == 0, torch.zeros_like(scale), scale)
    scale[bad] = float("nan")
    return q.view(rb * block_rows, kb * BLOCK)[:rows, :k], scale


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double(), nan=-1e30), torch.nan_to_num(b.double(), nan=-1e30))


def make(rows, k, dtype, seed):
    g = gen(seed)
    x = torch.randn(rows, k, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda")) * torch.exp(torch.randn(k, generator=g, device="cuda"))
    return x.to(dtype)


def check_quantize(x, block_rows=1, q=None, q_t=None):
    rows, k = x.shape
    q = bytes_like(rows, k) if q is None else q
    q_t = bytes_like(k, rows) if q_t is None else q_t
    s, s_t = torch.empty(up(rows, block_rows), up(k), device="cuda"), torch.empty(up(k, block_rows), up(rows), device="cuda")
    B.dc_quantize_blocks(x, q, s, q_t, s_t, block_rows)
    wq, ws = quantize64(x, block_rows)
    tq, ts = quantize64(x.t(), block_rows)
    assert same(s, ws) and same(s_t, ts)
    assert torch.equal(q.double(), wq) and torch.equal(q_t.double(), tq)
    # either alone: the same bits, and nothing else
    a, b = bytes_like(rows, k), bytes_like(k, rows)
    sa, sb = torch.empty_like(s), torch.empty_like(s_t)
    B.dc_quantize_blocks(x, a, sa, block_rows=block_rows)
    B.dc_quantize_blocks(x, None, None, b, sb, block_rows)
    assert torch.equal(bits(a), bits(q)) and torch.equal(bits(b), bits(q_t)) and same(sa, s) and same(sb, s_t)
    return q, s, q_t, s_t


SHAPES = [(1, 1), (1, 16), (1, 1000), (3, 127), (7, 128), (8, 129), (128, 128), (129, 130), (100, 300), (1000, 333), (300, 17), (2, 9216), (513, 1024), (4000, 70)]


@gpu
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k", SHAPES)
def test_quantize(rows, k, dtype, block_rows):
    check_quantize(make(rows, k, TYPES[dtype], rows + k), block_rows)


@gpu
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_of_halves_and_borders(dtype, block_rows):
    """Every e4m3 value and the middle between it and the next one; a largest value on either side of 448 times a power of two."""
    v = torch.arange(0, 0x7F, dtype=torch.uint8, device="cuda").view(E4M3).double()
    mid = (v[1:] + v[:-1]) / 2
    x = torch.zeros(40, 256, device="cuda", dtype=torch.float64)
    x[:, :127], x[:, 128:254] = v, mid
    x[:, 254] = 448
    x[::2] *= -1
    x *= torch.exp2(torch.arange(-20, 20, device="cuda").double())[:, None]
    x[3, 5] = 449 * 2.0 ** -17
    x[4, 7] = 450 * 2.0 ** -16 if dtype == "bf16" else 448.00003 * 2.0 ** -16
    check_quantize(x.to(TYPES[dtype]), block_rows)


@gpu
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_of_zeros_of_the_smallest_and_the_largest(dtype, block_rows):
    x = make(300, 300, torch.float32, 1)
    x[5], x[:, 140:] = 0.0, 0.0
    x[128:256] *= 2.0 ** -126                                 # denormal numbers among them
    x[256:] *= 1e37 / x[256:].abs().max()
    check_quantize(x.to(TYPES[dtype]), block_rows)
    check_quantize(torch.full((2, 130), 2.0 ** -133, device="cuda").to(TYPES[dtype]), block_rows)
    check_quantize(torch.full((2, 130), torch.finfo(TYPES[dtype]).max, device="cuda", dtype=TYPES[dtype]), block_rows)


@gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_nan_stays_in_its_block(dtype, block_rows, bad):
    x = make(200, 300, TYPES[dtype], 2)
    x[150, 140] = bad
    _, s, _, s_t = check_quantize(x, block_rows)
    assert torch.isnan(s).sum() == 1 and torch.isnan(s_t).sum() == 1


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pitch,offset,extra", [(300, 0, 0), (301, 0, 16), (304, 1, 0), (304, 8, 32)])
def test_quantize_strided_rows(pitch, offset, extra, dtype):
    x = make(140, 290, TYPES[dtype], 3)
    buf = torch.zeros(140 * pitch + offset + 16, dtype=x.dtype, device="cuda")
    view = buf[offset:offset + 140 * pitch].view(140, pitch)[:, :290]
    view.copy_(x)
    q, q_t = bytes_like(140, 290, extra), bytes_like(290, 140, extra)
    check_quantize(view, 1, q, q_t)
    for t, k in ((q, 290), (q_t, 140)):                       # what lies behind the rows' ends
        pitch = t.stride(0)
        whole = torch.as_strided(t.view(torch.uint8), (t.shape[0], pitch), (pitch, 1))
        assert (whole[:, k:] == 0x7F).all()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k", [(6000, 1000), (47000, 128), (400, 17000), (130, 40000), (100000, 8), (6001, 1003)])
def test_quantize_of_many_tiles(rows, k, dtype):
    check_quantize(make(rows, k, TYPES[dtype], 5))


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def random_rows(rows, k, seed, extra=0):
    """Any bits but NaN."""
    g = gen(seed)
    t = bytes_like(rows, k, extra)
    v = torch.randint(0, 256, (rows, k), generator=g, device="cuda").to(torch.uint8)
    v[(v & 0x7F) == 0x7F] ^= 0x15
    t.view(torch.uint8).copy_(v)
    return t


def random_scales(rows, kb, seed):
    g = gen(seed)
    return torch.exp(2.0 * torch.randn(rows, kb, generator=g, device="cuda")) * (0.01 + torch.rand(rows, kb, generator=g, device="cuda"))


def product64(a, sa, b, sb, bias, relu):
    """(out, bound before the last rounding)"""
    m, k = a.shape
    n, kb = b.shape[0], up(k)
    rows = torch.arange(n, device="cuda") // (BLOCK if sb.shape[0] == up(n) else 1)
    out, size = torch.zeros(m, n, dtype=torch.float64, device="cuda"), torch.zeros(m, n, dtype=torch.float64, device="cuda")
    for i in range(kb):
        p, w = a[:, i * BLOCK:(i + 1) * BLOCK].double(), b[:, i * BLOCK:(i + 1) * BLOCK].double()
        s = sa[:, i:i + 1].double() * sb[rows, i].double()
        out += s * (p @ w.t())
        size += s.abs() * (p.abs() @ w.abs().t())
    bound = size * (2.0 ** -20 + (kb + 20) * U)
    if bias is not None:
        out = out + bias.double()
        bound = bound + 2 * U * (size + bias.double().abs())
    return (out.clamp(min=0) if relu else out), bound


def check_product(a, sa, b, sb, bias, relu, dtype, out=None):
    m, n = a.shape[0], b.shape[0]
    out = torch.full((m, n), 77.0, dtype=TYPES[dtype], device="cuda") if out is None else out
    B.dc_matmul_blocks(a, sa, b, sb, bias, out, relu)
    want, bound = product64(a, sa, b, sb, bias, relu)
    T = torch.finfo(TYPES[dtype]).eps / 2
    over = (out.double() - want).abs() - (bound * (1 + T) + T * want.abs() + 1e-37)
    assert over.max() <= 0, f"off by {over.max():.3e} more than the bound"
    return out


PRODUCTS = [(1, 1, 1), (1, 8, 16), (1, 1000, 128), (1, 300, 4096), (2, 129, 129), (3, 64, 333), (7, 4096, 127), (8, 200, 1024), (16, 256, 512), (17, 1000, 1000), (32, 520, 4100), (33, 128, 31),
            (64, 130, 640), (100, 1000, 256), (127, 127, 127), (128, 128, 128), (129, 257, 257), (200, 512, 384), (256, 256, 2048), (300, 333, 77), (513, 1024, 200), (1000, 777, 333),
            (777, 333, 1000), (2500, 256, 64), (4000, 50, 40), (1500, 1500, 1500), (5000, 640, 300), (40, 40, 40000), (20000, 64, 640), (3000, 3000, 130), (300, 5000, 1280)]


@gpu
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, dtype, each):
    a, b = random_rows(m, k, m + k, 16 * (m % 3)), random_rows(n, k, n + k + 1, 16 * (n % 2))
    sa, sb = random_scales(m, up(k), 1), random_scales(n if each else up(n), up(k), 2)
    bias = 100 * torch.randn(n, generator=gen(3), device="cuda") if (m + n) % 2 else None
    check_product(a, sa, b, sb, bias, bool((m + k) % 2), dtype)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m", [1, 5, 40, 300])
@pytest.mark.parametrize("pitch,offset", [(200, 0), (203, 0), (208, 1), (208, 8)])
def test_product_into_strided_rows(m, pitch, offset, dtype):
    n, k = 199, 260
    a, b = random_rows(m, k, 1), random_rows(n, k, 2)
    sa, sb = random_scales(m, 3, 3), random_scales(2, 3, 4)
    buf = torch.full((m * pitch + offset + 64,), 77.0, dtype=TYPES[dtype], device="cuda")
    out = buf[offset:offset + m * pitch].view(m, pitch)[:, :n]
    check_product(a, sa, b, sb, torch.randn(n + 1, generator=gen(5), device="cuda")[1:], True, dtype, out)
    out.fill_(77.0)
    assert (buf == 77.0).all(), "something beside the rows was written"


@gpu
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,pitch,offset", [(600, 1008, 0), (40, 1003, 0), (600, 1000, 1), (129, 1008, 8)])
def test_product_of_wide_tiles_into_strided_rows(k, pitch, offset, dtype, each):
    m, n = 4600, 1000
    a, b = random_rows(m, k, 1), random_rows(n, k, 2)
    sa, sb = random_scales(m, up(k), 3), random_scales(n if each else up(n), up(k), 4)
    buf = torch.full((m * pitch + offset + 64,), 77.0, dtype=TYPES[dtype], device="cuda")
    out = buf[offset:offset + m * pitch].view(m, pitch)[:, :n]
    check_product(a, sa, b, sb, torch.randn(n + 1, generator=gen(5), device="cuda")[1:] if offset != 8 else None, offset != 0, dtype, out)
    out.fill_(77.0)
    assert (buf == 77.0).all(), "something beside the rows was written"


def far(rows, columns, pitch, dtype):
    """Rows `pitch` elements apart, the last ones behind 2^32 bytes and (of 8-bit values) elements."""
    t = torch.empty(rows * pitch, dtype=dtype, device="cuda").view(rows, pitch)[:, :columns]
    assert (rows - 1) * pitch * t.element_size() > 1 << 32
    return t


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_behind_four_gigabytes(dtype):
    rows, k, t = 1300, 264, TYPES[dtype]
    near = make(rows, k, t, 3)
    x, q, qt = far(rows, k, 1 << 21, t), far(rows, k, 1 << 22, torch.uint8), far(k, rows, 1 << 24, torch.uint8)
    x.copy_(near)
    for block in (1, 128):
        want = [bytes_like(rows, k), bytes_like(k, rows)]
        got = [torch.empty(up(rows, block), up(k), device="cuda"), torch.empty(up(k, block), up(rows), device="cuda")]
        scales = [torch.empty_like(v) for v in got]
        B.dc_quantize_blocks(near, want[0], scales[0], want[1], scales[1], block)
        B.dc_quantize_blocks(x, q, got[0], qt, got[1], block)
        assert torch.equal(q, bits(want[0])) and torch.equal(qt, bits(want[1])) and torch.equal(got[0], scales[0]) and torch.equal(got[1], scales[1])
    del qt


@gpu
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(1300, 1030), (20, 1030)])
def test_products_of_rows_behind_four_gigabytes(m, n, dtype, each):
    k, t = 300, TYPES[dtype]
    a, b = random_rows(m, k, 1), random_rows(n, k, 2)
    sa, sb = random_scales(m, up(k), 3), random_scales(n if each else up(n), up(k), 4)
    want = torch.empty(m, n, dtype=t, device="cuda")
    B.dc_matmul_blocks(a, sa, b, sb, None, want)
    far_a, far_b, out = far(m, k, 1 << 28 if m < 100 else 1 << 22, torch.uint8), far(n, k, 1 << 23, torch.uint8), far(m, n, 1 << 27 if m < 100 else 1 << 21, t)
    far_a.copy_(a.view(torch.uint8)), far_b.copy_(b.view(torch.uint8))
    B.dc_matmul_blocks(far_a, sa, far_b, sb, None, out)
    assert torch.equal(out, want)


@gpu
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("m,n,k", [(1, 200, 300), (20, 200, 300), (300, 600, 300)])
def test_nan_values_and_scales_reach_their_rows_alone(m, n, k, each):
    a, b = random_rows(m, k, 1), random_rows(n, k, 2)
    sa, sb = random_scales(m, 3, 3), random_scales(n if each else up(n), 3, 4)
    clean = torch.empty(m, n, device="cuda")
    B.dc_matmul_blocks(a, sa, b, sb, None, clean)
    a.view(torch.uint8)[m // 2, 299] = 0x7F
    b.view(torch.uint8)[150, 5] = 0xFF
    sb[-1, 1] = float("nan")
    out = torch.empty(m, n, device="cuda")
    B.dc_matmul_blocks(a, sa, b, sb, None, out, True)
    hit = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    hit[m // 2], hit[:, 150] = True, True
    hit[:, n - 1 if each else (n - 1) // BLOCK * BLOCK:] = True
    assert torch.isnan(out[hit]).all() and torch.equal(out[~hit], clean[~hit].clamp(min=0))


@gpu
@pytest.mark.parametrize("m", [1, 20, 300])
def test_scales_of_any_size(m):
    """Scales that are no powers of two, very small and very large ones whose product is not."""
    a, b = random_rows(m, 400, 1), random_rows(140, 400, 2)
    sa, sb = random_scales(m, 4, 3) * 1e-30, random_scales(2, 4, 4) * 1e28
    check_product(a, sa, b, sb, None, False, "f32")
    out = torch.full((m, 140), 77.0, device="cuda")
    B.dc_matmul_blocks(a, torch.zeros_like(sa), b, sb, None, out)
    assert (out == 0).all()


@gpu
def test_products_beside_each_other_and_other_kernels():
    """Large and split products, layers and integer products on four streams at once: each takes tensor memory, and none changes another's bits."""
    calls = []
    for i, (m, n, k) in enumerate([(2000, 1500, 900), (40, 3000, 4096), (100, 2000, 3000), (1, 4000, 2048)]):
        a, b = random_rows(m, k, i), random_rows(n, k, i + 9)
        sa, sb = random_scales(m, up(k), i), random_scales(up(n), up(k), i)
        calls.append(lambda out, a=a, b=b, sa=sa, sb=sb: B.dc_matmul_blocks(a, sa, b, sb, None, out))
        calls[-1].shape = (m, n)
    g = gen(3)
    a8, b8 = (torch.randint(-127, 128, (r, 2048), generator=g, device="cuda", dtype=torch.int8) for r in (64, 3000))
    s64, s3k = torch.rand(64, generator=g, device="cuda"), torch.rand(3000, generator=g, device="cuda")
    calls.append(lambda out: B.dc_matmul_quantized(a8, s64, b8, s3k, None, out))
    calls[-1].shape = (64, 3000)
    want = [torch.empty(c.shape, device="cuda") for c in calls]
    for c, o in zip(calls, want):
        c(o)
    torch.cuda.synchronize()
    got, streams = [torch.full_like(o, 7.0) for o in want], [torch.cuda.Stream() for _ in range(4)]
    for _ in range(12):
        for i, (c, o) in enumerate(zip(calls, got)):
            with torch.cuda.stream(streams[i % 4]):
                c(o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@gpu
def test_nothing_to_do():
    B.dc_matmul_blocks(bytes_like(0, 100), torch.empty(0, 1, device="cuda"), random_rows(8, 100, 1), random_scales(1, 1, 1), None, torch.empty(0, 8, device="cuda"))
    B.dc_quantize_blocks(torch.empty(0, 100, device="cuda"), bytes_like(0, 100), torch.empty(0, 1, device="cuda"))
    x = torch.ones(3, 100, device="cuda")
    B.dc_quantize_blocks(x)


# ---------------------------------------------------------------------------
# whole layers, and the operators together
# ---------------------------------------------------------------------------
def scratch(n):
    return torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda")


def weights(n, k, seed, each=False):
    w = torch.randn(n, k, generator=gen(seed), device="cuda")
    q, s = bytes_like(n, k), torch.empty(n if each else up(n), up(k), device="cuda")
    B.dc_quantize_blocks(w, q, s, block_rows=1 if each else BLOCK)
    return q, s


LAYERS = [(1, 1, 1), (1, 128, 100), (1, 1000, 4096), (1, 4096, 9216), (2, 512, 2048), (3, 10, 7), (4, 256, 1024), (8, 333, 500), (9, 256, 256), (20, 1000, 3000), (150, 384, 384), (700, 200, 129)]


@gpu
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", LAYERS)
def test_layer(m, n, k, dtype, each):
    """A layer is the product of its rows in 8 bits."""
    x = make(m, k, TYPES[dtype], m + n)
    w, s = weights(n, k, 2, each)
    bias = torch.randn(n, generator=gen(3), device="cuda")
    out = torch.full((m, n), 77.0, dtype=x.dtype, device="cuda")
    B.dc_linear_blocks(x, w, s, bias, out, True, scratch(B.dc_linear_blocks_workspace(m, k)))
    q, sx = quantize64(x, 1)
    want, bound = product64(q, sx, w, s, bias, True)
    T = torch.finfo(x.dtype).eps / 2
    assert ((out.double() - want).abs() <= bound * (1 + T) + T * want.abs() + 1e-37).all()


@gpu
@pytest.mark.parametrize("m", [1, 2, 8, 50])
@pytest.mark.parametrize("offset,pitch", [(0, 600), (1, 601), (8, 608)])
def test_layer_of_strided_rows_and_over_its_input(m, offset, pitch):
    n = k = 600
    buf = torch.zeros(m * pitch + offset + 64, dtype=torch.bfloat16, device="cuda")
    x = buf[offset:offset + m * pitch].view(m, pitch)[:, :k]
    x.copy_(make(m, k, torch.bfloat16, 1))
    w, s = weights(n, k, 2)
    work = scratch(B.dc_linear_blocks_workspace(m, k))
    q, sx = quantize64(x, 1)
    want, bound = product64(q, sx, w, s, None, False)
    T = 2.0 ** -8
    dense = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    B.dc_linear_blocks(x, w, s, None, dense, False, work)
    B.dc_linear_blocks(x, w, s, None, x, False, work[1:] if work.numel() > B.dc_linear_blocks_workspace(m, k) else work)
    for got in (dense, x):
        assert ((got.double() - want).abs() <= bound * (1 + T) + T * want.abs() + 1e-37).all()


@gpu
@pytest.mark.parametrize("m", [1, 3])
def test_layer_over_other_rows_of_its_input(m):
    """Output rows that lie over other input rows, or over parts of their own: all of the input is read first."""
    n, k = 256, 1024
    buf = torch.zeros(m * k + 4 * n, dtype=torch.bfloat16, device="cuda")
    x = buf[:m * k].view(m, k)
    x.copy_(make(m, k, torch.bfloat16, 4))
    w, s = weights(n, k, 5)
    apart = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    work = scratch(B.dc_linear_blocks_workspace(m, k))
    B.dc_linear_blocks(x.clone(), w, s, None, apart, False, work)
    q, sx = quantize64(x, 1)
    want, bound = product64(q, sx, w, s, None, False)
    out = buf[64:64 + m * n].view(m, n)
    B.dc_linear_blocks(x, w, s, None, out, False, work)
    for got in (apart, out):
        assert ((got.double() - want).abs() <= bound * 1.01 + 2.0 ** -8 * want.abs() + 1e-37).all()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_block_of_layers_forward_and_backward(dtype):
    """Normalisation with SiLU, a layer in 8 bits and both's gradients, as one step uses them: against the same step in 64 bits from the same 8-bit values."""
    maps, pixels, c, n, groups = 3, 77, 160, 200, 8
    m, T = maps * pixels, torch.finfo(TYPES[dtype]).eps / 2
    g = gen(9)
    x = torch.randn(maps, pixels, c, generator=g, device="cuda").to(TYPES[dtype])
    gamma, beta = 1 + 0.2 * torch.randn(c, generator=g, device="cuda"), 0.1 * torch.randn(c, generator=g, device="cuda")
    w32 = torch.randn(n, c, generator=g, device="cuda") / c ** 0.5
    w, ws, w_t, ws_t = bytes_like(n, c), torch.empty(up(n), up(c), device="cuda"), bytes_like(c, n), torch.empty(up(c), up(n), device="cuda")
    B.dc_quantize_blocks(w32, w, ws, w_t, ws_t, BLOCK)
    assert torch.equal(bits(w_t), bits(w.t())) and torch.equal(ws_t, ws.t())
    work = scratch(max(B.dc_group_norm_workspace(maps, pixels, c, groups), B.dc_linear_blocks_workspace(m, c)))
    y, mean, rstd = torch.empty_like(x), torch.empty(maps, groups, device="cuda"), torch.empty(maps, groups, device="cuda")
    out = torch.empty(m, n, dtype=x.dtype, device="cuda")
    B.dc_group_norm(x, groups, gamma, beta, y, mean, rstd, B.DC_ACT_SILU, 1e-5, work)
    B.dc_linear_blocks(y.view(m, c), w, ws, None, out, False, work)
    dout = torch.randn(m, n, generator=g, device="cuda").to(x.dtype)
    q, s, q_t, s_t = bytes_like(m, n), torch.empty(m, up(n), device="cuda"), bytes_like(n, m), torch.empty(n, up(m), device="cuda")
    B.dc_quantize_blocks(dout, q, s, q_t, s_t)
    y_t, ys_t = bytes_like(c, m), torch.empty(c, up(m), device="cuda")
    B.dc_quantize_blocks(y.view(m, c), None, None, y_t, ys_t)
    dy, dw, dx = torch.empty_like(x), torch.empty(n, c, device="cuda"), torch.empty_like(x)
    B.dc_matmul_blocks(q, s, w_t, ws_t, None, dy.view(m, c))
    B.dc_matmul_blocks(q_t, s_t, y_t, ys_t, None, dw)
    dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    B.dc_group_norm_backward(dy, x, groups, gamma, beta, mean, rstd, dx, dg, db, B.DC_ACT_SILU, work)
    # 64 bits, step by step from what each call was given
    want, bound = product64(*quantize64(y.view(m, c), 1), w, ws, None, False)
    assert ((out.double() - want).abs() <= bound * (1 + T) + T * want.abs()).all()
    want, bound = product64(*quantize64(dout, 1), *quantize64(w32.t(), BLOCK), None, False)
    assert ((dy.view(m, c).double() - want).abs() <= bound * (1 + T) + T * want.abs()).all()
    want, bound = product64(*quantize64(dout.t(), 1), *quantize64(y.view(m, c).t(), 1), None, False)
    assert ((dw.double() - want).abs() <= bound + U * want.abs()).all()
    v = x.double().view(maps, pixels, groups, -1).requires_grad_()
    gd, bd = gamma.double().requires_grad_(), beta.double().requires_grad_()
    d = v - v.mean((1, 3), keepdim=True)
    z = (d * (d.square().mean((1, 3), keepdim=True) + 1e-5).rsqrt()).reshape(maps, pixels, c) * gd + bd
    (z * torch.sigmoid(z) * dy.double()).sum().backward()
    # (the bounds of test_group_norm.py in one: sums of at most 77 * 20 terms, everything of order one)
    size = dy.double().abs().amax() * rstd.double().amax() * 2
    assert ((dx.double() - v.grad.reshape(maps, pixels, c)).abs() <= T * v.grad.reshape(maps, pixels, c).abs() + 2000 * U * size).all()
    assert ((dg.double() - gd.grad).abs() <= 2000 * U * size * m).all() and ((db.double() - bd.grad).abs() <= 2000 * U * size * m).all()


@gpu
def test_equal_calls_give_equal_bits_on_streams_and_in_graphs():
    for m, n, k in ((1, 600, 2048), (5, 300, 700), (40, 600, 2048), (600, 700, 900)):
        w, s = weights(n, k, 2)
        xs = [make(m, k, torch.bfloat16, i) for i in (1, 2)]
        outs = lambda: (torch.empty(m, n, dtype=torch.bfloat16, device="cuda"), scratch(B.dc_linear_blocks_workspace(m, k)))
        want = [outs() for _ in xs]
        for x, (o, t) in zip(xs, want):
            B.dc_linear_blocks(x, w, s, None, o, False, t)
        torch.cuda.synchronize()
        got, streams = [outs() for _ in xs], [torch.cuda.Stream() for _ in xs]
        for _ in range(4):
            for x, (o, t), stream in zip(xs, got, streams):
                with torch.cuda.stream(stream):
                    B.dc_linear_blocks(x, w, s, None, o, False, t)
        torch.cuda.synchronize()
        assert all(torch.equal(a[0], b[0]) for a, b in zip(want, got))
        x, (o, t) = xs[0].clone(), outs()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.dc_linear_blocks(x, w, s, None, o, False, t)
        x.copy_(xs[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[1][0])


# ---------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------
def test_refusals_of_the_c_abi():
    lib = B.load()
    buf = (C.c_char * 4096)()
    at = (C.addressof(buf) + 255) & ~255
    n = C.c_size_t()
    assert lib.dc_linear_blocks_workspace(1, 1, None) == B.DC_ERR_ARG and lib.dc_linear_blocks_workspace(-1, 1, C.byref(n)) == B.DC_ERR_ARG
    assert lib.dc_linear_blocks_workspace(2, (1 << 28) + 1, C.byref(n)) == B.DC_ERR_LIMIT and lib.dc_linear_blocks_workspace(1 << 31, 8, C.byref(n)) == B.DC_ERR_LIMIT
    assert lib.dc_linear_blocks_workspace(2, 0, C.byref(n)) == B.DC_ERR_ARG and lib.dc_linear_blocks_workspace(2, 32, C.byref(n)) == B.DC_OK
    room = n.value

    def quantize(x=at, x_pitch=128, rows=2, c=32, dtype=B.DC_FP32, block=1, q=at, q_pitch=32, s=at, qt=None, qt_pitch=0, st=None):
        return lib.dc_quantize_blocks(x, x_pitch, rows, c, dtype, block, q, q_pitch, s, qt, qt_pitch, st, None)

    assert quantize(dtype=3) == B.DC_ERR_CONFIG and quantize(block=2) == B.DC_ERR_CONFIG and quantize(block=0) == B.DC_ERR_CONFIG
    assert quantize(rows=-1) == B.DC_ERR_ARG and quantize(c=0) == B.DC_ERR_ARG and quantize(s=None) == B.DC_ERR_ARG and quantize(qt=at) == B.DC_ERR_ARG and quantize(st=at) == B.DC_ERR_ARG
    assert quantize(x=None) == B.DC_ERR_ARG and quantize(x=at + 2) == B.DC_ERR_ARG and quantize(x_pitch=124) == B.DC_ERR_ARG and quantize(x_pitch=130) == B.DC_ERR_ARG
    assert quantize(q=at + 8) == B.DC_ERR_ARG and quantize(q_pitch=40) == B.DC_ERR_ARG and quantize(q_pitch=16) == B.DC_ERR_ARG and quantize(s=at + 2) == B.DC_ERR_ARG
    assert quantize(qt=at + 4, qt_pitch=16, st=at) == B.DC_ERR_ARG and quantize(qt=at, qt_pitch=8, st=at) == B.DC_ERR_ARG
    assert quantize(rows=1 << 31) == B.DC_ERR_LIMIT and quantize(x_pitch=1 << 32) == B.DC_ERR_LIMIT and quantize(q_pitch=1 << 40) == B.DC_ERR_LIMIT
    assert quantize(c=(1 << 28) + 1, rows=1) == B.DC_ERR_LIMIT
    assert quantize(q=None, s=None) == B.DC_OK and quantize(rows=0) == B.DC_OK

    def product(a=at, a_pitch=32, sa=at, b=at, b_pitch=32, sb=at, block=128, bias=None, m=2, n=4, k=32, dtype=B.DC_FP32, out=at, out_pitch=16):
        return lib.dc_matmul_blocks(a, a_pitch, sa, b, b_pitch, sb, block, bias, m, n, k, 0, dtype, out, out_pitch, None)

    def layer(x=at, x_pitch=128, b=at, b_pitch=32, sb=at, block=128, bias=None, m=2, n=4, k=32, dtype=B.DC_FP32, out=at, out_pitch=16, work=at, bytes_=room):
        return lib.dc_linear_blocks(x, x_pitch, b, b_pitch, sb, block, bias, m, n, k, 0, dtype, out, out_pitch, work, bytes_, None)

    for call in (product, layer):
        assert call(dtype=2) == B.DC_ERR_CONFIG and call(block=64) == B.DC_ERR_CONFIG
        assert call(m=-1) == B.DC_ERR_ARG and call(n=0) == B.DC_ERR_ARG and call(k=0) == B.DC_ERR_ARG and call(m=0) == B.DC_OK
        assert call(k=(1 << 28) + 1) == B.DC_ERR_LIMIT
        assert call(n=(1 << 28) + 1) == B.DC_ERR_LIMIT and call(m=1 << 31) == B.DC_ERR_LIMIT and call(b_pitch=1 << 40) == B.DC_ERR_LIMIT
        assert call(b=None) == B.DC_ERR_ARG and call(b=at + 8) == B.DC_ERR_ARG and call(b_pitch=24) == B.DC_ERR_ARG and call(b_pitch=16) == B.DC_ERR_ARG
        assert call(sb=None) == B.DC_ERR_ARG and call(sb=at + 2) == B.DC_ERR_ARG and call(bias=at + 1) == B.DC_ERR_ARG
        assert call(out=None) == B.DC_ERR_ARG and call(out=at + 2) == B.DC_ERR_ARG and call(out_pitch=12) == B.DC_ERR_ARG and call(out_pitch=18) == B.DC_ERR_ARG
    assert product(a=None) == B.DC_ERR_ARG and product(a=at + 1) == B.DC_ERR_ARG and product(a_pitch=16) == B.DC_ERR_ARG and product(sa=None) == B.DC_ERR_ARG and product(a_pitch=1 << 40) == B.DC_ERR_LIMIT
    assert layer(x=None) == B.DC_ERR_ARG and layer(x=at + 2) == B.DC_ERR_ARG and layer(x_pitch=100) == B.DC_ERR_ARG and layer(x_pitch=1 << 32) == B.DC_ERR_LIMIT
    assert layer(work=None) == B.DC_ERR_ARG and layer(bytes_=room - 1) == B.DC_ERR_ARG


@gpu
def test_refusals_of_tensors():
    a, b = random_rows(4, 200, 1), random_rows(6, 200, 2)
    sa, sb = random_scales(4, 2, 3), random_scales(1, 2, 4)
    out = torch.empty(4, 6, device="cuda")
    for bad in (dict(a=a.float()), dict(a=a[:, ::2]), dict(a=a.t()), dict(sa=sa[:, :1]), dict(sa=sa.double()), dict(sb=random_scales(2, 2, 1)), dict(b=random_rows(6, 201, 2)), dict(out=out.half()),
                dict(out=out.t()), dict(sa=sa.cpu()), dict(sb=None), dict(bias=torch.zeros(5, device="cuda"))):
        v = dict(a=a, sa=sa, b=b, sb=sb, out=out, bias=None)
        v.update(bad)
        with pytest.raises((TypeError, ValueError)):
            B.dc_matmul_blocks(v["a"], v["sa"], v["b"], v["sb"], v["bias"], v["out"])
    x = torch.zeros(4, 200, device="cuda")
    with pytest.raises(B.DeepCacheError):
        B.dc_linear_blocks(x, b, sb, None, out, False, None)
    with pytest.raises(B.DeepCacheError):
        B.dc_quantize_blocks(x, a, sa, block_rows=64)
    with pytest.raises(B.DeepCacheError):                      # rows in 8 bits that are not 16 bytes apart
        B.dc_matmul_blocks(torch.zeros(4, 200, dtype=torch.uint8, device="cuda").view(E4M3), sa, b, sb, None, out)
    with pytest.raises((TypeError, ValueError)):
        B.dc_quantize_blocks(x, a, sa, random_rows(4, 200, 1), sa)


# ---------------------------------------------------------------------------
# a process's first call, workspaces anywhere
# ---------------------------------------------------------------------------
FIRST = """
import torch
from paper_1712_01670_b200 import binding as B
m, n, k = 20, 512, 4096
a, b = (torch.randint(0, 0x7F, (r, k), dtype=torch.uint8, device="cuda") for r in (m, n))
sa, sb = torch.rand(m, k // 128, device="cuda"), torch.rand(n // 128, k // 128, device="cuda")
out, want = torch.zeros(m, n, device="cuda"), torch.zeros(m, n, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    B.dc_matmul_blocks(a, sa, b, sb, None, out)
graph.replay()
B.dc_matmul_blocks(a, sa, b, sb, None, want)
torch.cuda.synchronize()
assert want.abs().min() > 0 and torch.equal(out, want)
"""


@gpu
def test_a_first_call_that_is_captured():
    """What a call asks of the device once (how many clusters it holds), it may ask while a stream is captured; a query that fails is the call's error, never a guess that would sum up in another order."""
    done = subprocess.run([sys.executable, "-c", FIRST], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


@gpu
@pytest.mark.parametrize("shift", [0, 1, 100, 255])
@pytest.mark.parametrize("m,n,k", [(1, 300, 4100), (20, 130, 1000), (700, 300, 333)])
def test_layer_with_a_workspace_of_any_alignment(m, n, k, shift):
    """As many bytes as asked for, from any one on: the same bits, and nothing beside them is written."""
    x = make(m, k, torch.bfloat16, 7)
    w, s = weights(n, k, 2)
    need = B.dc_linear_blocks_workspace(m, k)
    want, out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda"), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    B.dc_linear_blocks(x, w, s, None, want, False, scratch(need))
    room = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    at = -room.data_ptr() % 256 + shift
    B.dc_linear_blocks(x, w, s, None, out, False, room[at:at + need])
    assert torch.equal(out, want)
    assert (room[:at] == 0x5A).all() and (room[at + need:] == 0x5A).all()


# ---------------------------------------------------------------------------
# waits that run out
# ---------------------------------------------------------------------------
def stall_next(ms, blocks):
    f = B.load().dc_debug_stall_next_blocks
    f.restype, f.argtypes = C.c_int, [C.c_int, C.c_int]
    return f(ms, blocks)


@gpu
@pytest.mark.parametrize("blocks", [0, 1, 5, 9, 10])
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(6000, 4000, 600), (2500, 1900, 600), (1200, 1000, 1200), (5000, 60, 600)])
def test_waits_that_run_out_leave_nan_and_nothing_wrong(m, n, k, dtype, each, blocks):
    """Operands stop coming behind so many blocks of each CTA, without a fault: its waits run out after some milliseconds, the kernel returns, and every value is either right or NaN.
    The next call is an ordinary one."""
    a, b = random_rows(m, k, 1), random_rows(n, k, 2)
    sa, sb = random_scales(m, up(k), 3), random_scales(n if each else up(n), up(k), 4)
    want, out = (torch.full((m, n), 77.0, dtype=TYPES[dtype], device="cuda") for _ in range(2))
    B.dc_matmul_blocks(a, sa, b, sb, None, want)
    assert not torch.isnan(want).any()
    assert stall_next(5, blocks) == B.DC_OK
    B.dc_matmul_blocks(a, sa, b, sb, None, out)
    lost = torch.isnan(out)
    assert torch.equal(out[~lost], want[~lost])
    if blocks < 2:
        assert lost.all()                                     # not one sum is whole (of clusters that share one the first CTA alone gets too few: two blocks of ten or of five at least)
    if m == 6000 and blocks >= up(k):                         # several tiles to a CTA, and the operands of one or two
        assert lost.any() and not lost.all()
    again = torch.empty_like(out)
    B.dc_matmul_blocks(a, sa, b, sb, None, again)
    assert torch.equal(again, want)


@gpu
@pytest.mark.parametrize("blocks", [0, 1])
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("m", [1, 20, 60, 100])
def test_a_cluster_whose_first_cta_gets_no_operands_stores_nan(m, each, blocks):
    n, k = 512, 9216
    a, b = random_rows(m, k, 1), random_rows(n, k, 2)
    sa, sb = random_scales(m, up(k), 3), random_scales(n if each else up(n), up(k), 4)
    want, out = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    B.dc_matmul_blocks(a, sa, b, sb, None, want)
    assert stall_next(5, blocks) == B.DC_OK
    B.dc_matmul_blocks(a, sa, b, sb, None, out)
    assert not torch.isnan(want).any() and torch.isnan(out).all()
    B.dc_matmul_blocks(a, sa, b, sb, None, out)
    assert torch.equal(out, want)


def test_refusals_of_stalls():
    assert stall_next(0, 1) == B.DC_ERR_ARG and stall_next(1001, 1) == B.DC_ERR_ARG and stall_next(5, -1) == B.DC_ERR_ARG
