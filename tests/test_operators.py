"""Layer normalisation, its gradients, 8-bit rows and their products, against plain 64-bit implementations.

Tolerances: u = 2^-24 is half a step of float32, T(t) half a step of the map's type (2^-24, bfloat16 2^-8), relative to the value.
A sum of n float32 terms made in a tree of depth d is off by at most d u sum|terms|; no lane adds more than 64 terms one behind another,
and at most 16 joins (lanes, warps) follow, so d = 80 is used throughout.
"""
import ctypes as C

import pytest
import torch

from paper_1712_01670_b200 import binding as B

U = 2.0 ** -24
DEPTH = 80
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
gpu = pytest.mark.gpu


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make_map(rows, c, dtype, seed, shift=0.7):
    g = gen(seed)
    x = torch.randn(rows, c, generator=g, device="cuda") * torch.exp(torch.randn(c, generator=g, device="cuda")) + shift
    return x.to(dtype)


def spread(x, pitch, offset=0):
    """The same rows `pitch` elements apart, `offset` elements behind the start of an allocation."""
    rows, c = x.shape
    buf = torch.full((rows * pitch + offset + 64,), 77, dtype=x.dtype, device=x.device)
    view = buf[offset:offset + rows * pitch].view(rows, pitch)[:, :c]
    view.copy_(x)
    return view, buf


def q_like(rows, k):
    return torch.full((rows, (k + 15) // 16 * 16), 55, dtype=torch.int8, device="cuda")[:, :k]


def scratch(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def norm64(x, gamma, beta, eps):
    """(y, mean, rstd, bound of y's error before it is rounded to the map's type)"""
    x = x.double()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    g = torch.ones(x.shape[1], device=x.device, dtype=torch.float64) if gamma is None else gamma.double()
    b = torch.zeros_like(g) if beta is None else beta.double()
    y = d * rstd * g + b
    # the mean is off by DEPTH u mean|x|, each difference by half a step more, the sum of squares by DEPTH u and by the square of the mean's
    # error, the root, division, two products and the sum by half a step each
    dm = (DEPTH + 2) * U * x.abs().mean(1, keepdim=True)
    bound = g.abs() * rstd * (dm * (1 + (d * rstd).abs() * dm * rstd) + d.abs() * (DEPTH / 2 + 8) * U) + 2 * U * (y.abs() + b.abs())
    return y, mean[:, 0], rstd[:, 0], bound


def check_norm(x, gamma, beta, eps=1e-5, y=None):
    rows, c = x.shape
    y = torch.empty(rows, c, dtype=x.dtype, device="cuda") if y is None else y
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    want, wmean, wrstd, bound = norm64(x, gamma, beta, eps)
    B.dc_layer_norm(x, gamma, beta, y, mean, rstd, eps)
    T = half_step(x.dtype)
    over = (y.double() - want).abs() - (bound * (1 + T) + T * want.abs() + 1e-38)
    assert over.max() <= 0, f"y off by {over.max():.3e} more than the bound"
    xd = x.double()
    assert ((mean.double() - wmean).abs() <= (DEPTH + 2) * U * xd.abs().mean(1)).all()
    assert ((rstd.double() - wrstd).abs() <= wrstd * ((DEPTH / 2 + 8) * U + ((DEPTH + 2) * U * xd.abs().mean(1) * wrstd) ** 2)).all()
    return y


NORM_SHAPES = [(1, 1), (1, 7), (3, 8), (5, 16), (33, 24), (130, 48), (257, 96), (64, 100), (1000, 256), (31, 257), (77, 512), (19, 513), (9, 1000), (50, 1024),
               (49, 2048), (6, 2049), (5, 4096), (3, 4100), (3, 8192), (2, 8193), (2, 16384), (700, 64), (40000, 32), (70001, 1), (50000, 3), (30000, 17)]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", NORM_SHAPES)
def test_norm(rows, c, dtype):
    g = gen(rows + c)
    gamma, beta = torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")
    check_norm(make_map(rows, c, TYPES[dtype], rows * 7 + c), gamma, beta)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gamma,beta", [(True, False), (False, True), (False, False)])
def test_norm_without_weights(gamma, beta, dtype):
    w = torch.randn(96, generator=gen(1), device="cuda")
    check_norm(make_map(70, 96, TYPES[dtype], 2), w if gamma else None, w if beta else None)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c,pitch,offset", [(20, 64, 64, 1), (20, 64, 80, 0), (20, 64, 72, 3), (20, 64, 65, 0), (11, 256, 264, 8), (9, 1024, 1032, 4), (3, 4096, 4097, 2)])
def test_norm_of_strided_and_shifted_rows(rows, c, pitch, offset, dtype):
    g = gen(5)
    x, _ = spread(make_map(rows, c, TYPES[dtype], 9), pitch, offset)
    y, buf = spread(torch.zeros(rows, c, dtype=TYPES[dtype], device="cuda"), pitch, offset)
    gamma = torch.randn(c + 1, generator=g, device="cuda")[1:]        # not 16-byte aligned either
    check_norm(x, gamma, None, y=y)
    rest = buf.clone()
    rest[offset:offset + rows * pitch].view(rows, pitch)[:, :c] = 77
    assert (rest == 77).all(), "something beside the rows was written"


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_between_maps_of_different_strides_and_a_part_of_the_statistics(dtype):
    rows, c = 90, 128
    x = make_map(rows, c, TYPES[dtype], 1)
    want, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.dc_layer_norm(x, None, None, want, mean, rstd)
    for pitch, offset in ((136, 0), (129, 0), (128, 3)):
        y, _ = spread(torch.zeros_like(x), pitch, offset)
        m, r = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        check_norm(x, None, None, y=y)
        B.dc_layer_norm(x, None, None, y, m)
        B.dc_layer_norm(x, None, None, y, None, r)
        xs, _ = spread(x, pitch, offset)
        z = torch.empty_like(x)
        check_norm(xs, None, None, y=z)
        if pitch % 8 == 0 and offset == 0:
            assert torch.equal(y, want) and torch.equal(z, want) and torch.equal(m, mean) and torch.equal(r, rstd)


@gpu
def test_norm_in_place_equals_out_of_place():
    x = make_map(333, 192, torch.bfloat16, 3)
    y = torch.empty_like(x)
    B.dc_layer_norm(x, None, None, y)
    B.dc_layer_norm(x, None, None, x)
    assert torch.equal(x, y)


@gpu
def test_norm_of_rows_with_large_means_and_constant_rows():
    g = gen(8)
    x = torch.randn(64, 384, generator=g, device="cuda") + 1000.0     # the squares' difference would have nothing left here
    x[5] = 3.25
    x[6] = 0.0
    check_norm(x, torch.randn(384, generator=g, device="cuda"), None)


@gpu
@pytest.mark.parametrize("c", [64, 257, 2048, 5000])
def test_norm_keeps_what_is_not_finite_to_its_row(c):
    x = make_map(12, c, torch.float32, 4)
    clean = torch.empty_like(x)
    B.dc_layer_norm(x, None, None, clean)
    x[3, c // 2], x[7, 0], x[8, c - 1] = float("nan"), float("inf"), float("-inf")
    y = torch.empty_like(x)
    B.dc_layer_norm(x, None, None, y)
    bad = torch.zeros(12, dtype=torch.bool, device="cuda")
    bad[[3, 7, 8]] = True
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[~bad])


@gpu
def test_norm_of_rows_far_apart():
    """Rows 2^31 bytes apart and more: offsets that 32 bits do not hold."""
    c, pitch, rows = 64, (1 << 29) + 4, 4
    buf = torch.empty(pitch * (rows - 1) + c, device="cuda")
    x = buf.as_strided((rows, c), (pitch, 1))
    x.copy_(make_map(rows, c, torch.float32, 6))
    check_norm(x, None, None)


@gpu
def test_norm_of_a_map_of_more_than_two_billion_elements():
    rows, c = (1 << 23) + 5, 256
    x = torch.zeros(rows, c, dtype=torch.bfloat16, device="cuda")
    tail = make_map(64, c, torch.bfloat16, 11)
    x[-64:] = tail
    q, scale = torch.zeros(rows, c, dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")
    B.dc_layer_norm_quantize(x, None, None, q, scale, x)
    y, q2, s2 = torch.empty_like(tail), q_like(64, c), torch.empty(64, device="cuda")
    B.dc_layer_norm_quantize(tail, None, None, q2, s2, y)
    assert torch.equal(x[-64:], y) and torch.equal(q[-64:], q2) and torch.equal(scale[-64:], s2)
    assert int(x[:-64].float().abs().max()) == 0


# ---------------------------------------------------------------------------
# gradients
# ---------------------------------------------------------------------------
def backward64(dy, x, gamma, mean, rstd):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    g = torch.ones(x.shape[1], device=x.device, dtype=torch.float64) if gamma is None else gamma.double()
    xh, gy = (x - mean) * rstd, dy * g
    m1, m2 = gy.mean(1, keepdim=True), (gy * xh).mean(1, keepdim=True)
    dx = rstd * (gy - m1 - xh * m2)
    # xh is off by 3 u of itself, the means by DEPTH u and their terms' own 4 u
    bound = U * rstd * (8 * gy.abs() + (DEPTH + 8) * gy.abs().mean(1, keepdim=True) + (DEPTH + 16) * xh.abs() * (gy * xh).abs().mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), bound, (dy * xh).abs().sum(0), dy.abs().sum(0)


def run_backward(dy, x, gamma, mean, rstd, dx=None):
    c = x.shape[1]
    dx = torch.empty(x.shape, dtype=x.dtype, device="cuda") if dx is None else dx
    dg, db = torch.full((c,), 9.0, device="cuda"), torch.full((c,), 9.0, device="cuda")
    work = scratch(B.dc_layer_norm_workspace(c))
    work.fill_(0x7f)                                                   # large floats: what is not written is not read
    B.dc_layer_norm_backward(dy, x, gamma, mean, rstd, dx, dg, db, work)
    return dx, dg, db


def check_backward(dy, x, gamma, dx=None):
    _, mean, rstd, _ = norm64(x, None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    want, wg, wb, bound, sg, sb = backward64(dy, x, gamma, mean, rstd)
    dx, dg, db = run_backward(dy, x, gamma, mean, rstd, dx)
    T = half_step(x.dtype)
    assert ((dx.double() - want).abs() <= bound * (1 + T) + T * want.abs() + 1e-38).all()
    # rows that one lane adds one behind another, and the joins of warps and CTAs
    depth = DEPTH + 4 + x.shape[0] / 64
    assert ((dg.double() - wg).abs() <= depth * U * sg).all()
    assert ((db.double() - wb).abs() <= depth * U * sb).all()
    return mean, rstd, dx, dg, db


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", NORM_SHAPES)
def test_backward(rows, c, dtype):
    g = gen(3 * rows + c)
    x = make_map(rows, c, TYPES[dtype], rows + 5 * c)
    dy = torch.randn(rows, c, generator=g, device="cuda").to(TYPES[dtype])
    check_backward(dy, x, torch.randn(c, generator=g, device="cuda"))


@gpu
@pytest.mark.parametrize("rows", [2000, 12345])
@pytest.mark.parametrize("c", [20, 256, 640])
def test_backward_of_many_rows_is_the_same_every_time(rows, c):
    g = gen(rows)
    x, dy = make_map(rows, c, torch.bfloat16, 1), torch.randn(rows, c, generator=g, device="cuda").to(torch.bfloat16)
    mean, rstd, *first = check_backward(dy, x, None)
    for _ in range(3):
        again = run_backward(dy, x, None, mean, rstd)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


# three vectors per lane (whole and with places to spare), two or three per thread of longer rows, small and large maps
@gpu
@pytest.mark.parametrize("dtype,rows,c", [("bf16", 1001, 24), ("bf16", 1500, 136), ("bf16", 3000, 192), ("bf16", 1111, 384), ("bf16", 2000, 552), ("bf16", 2751, 768),
                                          ("bf16", 2101, 1000), ("bf16", 2055, 1024), ("bf16", 1400, 1536), ("bf16", 1499, 1480), ("bf16", 400, 8192), ("bf16", 300, 8184),
                                          ("f32", 1001, 12), ("f32", 3000, 96), ("f32", 1300, 92), ("f32", 1999, 384), ("f32", 2800, 768), ("f32", 2999, 760),
                                          ("f32", 2222, 1024), ("f32", 600, 6144), ("f32", 400, 6136)])
def test_backward_of_large_maps(dtype, rows, c):
    g = gen(5 * rows + c)
    x, dy = make_map(rows, c, TYPES[dtype], rows + c), torch.randn(rows, c, generator=g, device="cuda").to(TYPES[dtype])
    gamma = torch.randn(c, generator=g, device="cuda")
    mean, rstd, *first = check_backward(dy, x, gamma)
    again = run_backward(dy, x, gamma, mean, rstd)
    assert all(torch.equal(p, q) for p, q in zip(first, again))


@gpu
@pytest.mark.parametrize("rows,c", [(1207, 24), (1207, 48), (1207, 136), (1207, 192), (1207, 384), (1207, 520), (1207, 640), (1207, 768), (9601, 1024), (6001, 1024), (9601, 1000)])
def test_norm_and_quantise_of_three_and_four_vectors_per_lane(rows, c):
    g = gen(c)
    x = make_map(rows, c, torch.bfloat16, c)
    gamma, beta = torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")
    y = check_norm(x, gamma, beta)
    q, scale, q2, scale2 = q_like(rows, c), torch.empty(rows, device="cuda"), q_like(rows, c), torch.empty(rows, device="cuda")
    B.dc_layer_norm_quantize(x, gamma, beta, q, scale)
    B.dc_quantize_rows(y, q2, scale2)
    assert torch.equal(q, q2) and torch.equal(scale, scale2)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_of_strided_rows_and_of_a_part_of_the_gradients(dtype):
    g = gen(2)
    rows, c = 37, 120
    x, _ = spread(make_map(rows, c, TYPES[dtype], 9), 131, 1)
    dy, _ = spread(torch.randn(rows, c, generator=g, device="cuda").to(TYPES[dtype]), 125, 0)
    gamma = torch.randn(c, generator=g, device="cuda")
    out, buf = spread(torch.zeros(rows, c, dtype=TYPES[dtype], device="cuda"), 129, 2)
    mean, rstd, dx, dg, db = check_backward(dy, x, gamma, dx=out)
    rest = buf.clone()
    rest[2:2 + rows * 129].view(rows, 129)[:, :c] = 77
    assert (rest == 77).all()
    work = scratch(B.dc_layer_norm_workspace(c))
    only = torch.empty(rows, c, dtype=TYPES[dtype], device="cuda")
    B.dc_layer_norm_backward(dy, x, gamma, mean, rstd, dx=only)       # no workspace needed
    assert torch.equal(only, dx)
    g2, b2 = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    B.dc_layer_norm_backward(dy, x, gamma, mean, rstd, dgamma=g2, workspace=work)
    B.dc_layer_norm_backward(dy, x, gamma, mean, rstd, dbeta=b2, workspace=work)
    assert torch.equal(g2, dg) and torch.equal(b2, db)
    for k in (0, 1):                                                   # in place: the bits of the same call with an output of its own
        inplace = [dy.clone(), x.clone()]
        B.dc_layer_norm_backward(inplace[0], inplace[1], gamma, mean, rstd, dx=only)
        B.dc_layer_norm_backward(inplace[0], inplace[1], gamma, mean, rstd, dx=inplace[k])
        assert torch.equal(inplace[k], only) and torch.equal(inplace[1 - k], (x, dy)[k])


@gpu
def test_backward_against_differences():
    """Central differences of sum(dy * y) of the 64-bit forward formula, of step h: their own error is h^2 / 6 of a third derivative of
    order one here, and 2^-52 / h of the sum's size."""
    rows, c, h = 3, 10, 1e-4
    g = gen(7)
    x = torch.randn(rows, c, generator=g, device="cuda")
    gamma, beta = torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")
    dy = torch.randn(rows, c, generator=g, device="cuda")

    def value(x, gamma, beta):
        d = x - x.mean(1, keepdim=True)
        return float((dy.double() * (d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * gamma + beta)).sum())

    _, mean, rstd, _ = norm64(x, gamma, beta, 1e-5)
    got = run_backward(dy, x, gamma, mean.float(), rstd.float())
    args = [x.double(), gamma.double(), beta.double()]
    for k, grad in enumerate(got):
        want = torch.empty_like(args[k])
        for i in range(want.numel()):
            moved = []
            for s in (h, -h):
                a = [t.clone() for t in args]
                a[k].view(-1)[i] += s
                moved.append(value(*a))
            want.view(-1)[i] = (moved[0] - moved[1]) / (2 * h)
        assert (grad.double() - want).abs().max() < 5e-6


@gpu
def test_backward_of_no_rows():
    c = 40
    x = torch.empty(0, c, device="cuda")
    dg, db = torch.full((c,), 5.0, device="cuda"), torch.full((c,), 5.0, device="cuda")
    B.dc_layer_norm_backward(x, x, None, torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), x, dg, db, scratch(B.dc_layer_norm_workspace(c)))
    assert (dg == 0).all() and (db == 0).all()


# ---------------------------------------------------------------------------
# rows in 8 bits
# ---------------------------------------------------------------------------
def quantise64(x):
    """127 x / max|x| to the nearest integer: 127 x is exact in 64 bits, and a quotient of two numbers of at most 31 and 24 bits that is not a
    half lies further from it than 64 bits round."""
    x = x.double()
    most = x.abs().amax(1, keepdim=True)
    q = torch.round(127.0 * x / torch.where(most > 0, most, torch.ones_like(most)))
    scale = (most[:, 0] / 127.0).float()
    bad = ~torch.isfinite(x).all(1)
    q[bad], scale[bad] = 0.0, float("nan")
    return q.to(torch.int8), scale


def check_quantise(x, q=None):
    rows, k = x.shape
    q = q_like(rows, k) if q is None else q
    scale = torch.full((rows,), 9.0, device="cuda")
    wq, ws = quantise64(x)
    B.dc_quantize_rows(x, q, scale)
    assert torch.equal(q, wq)
    assert torch.equal(torch.nan_to_num(scale, nan=-1.0), torch.nan_to_num(ws, nan=-1.0))


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k", NORM_SHAPES + [(3, 25088), (2, 30011), (2, 40000), (1, 131071)])
def test_quantise(rows, k, dtype):
    x = make_map(rows, k, TYPES[dtype], rows + k)
    x[rows // 2] = 0
    check_quantise(x)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantise_halves_and_their_neighbours(dtype):
    """Every half between two steps, for many largest values, and the numbers next to it."""
    t = TYPES[dtype]
    g = gen(12)
    most = torch.cat([torch.tensor([127.0, 254.0, 1.0, 3.0, 2.0 ** -100, 2.0 ** -130, 2.0 ** -149, 2.0 ** 127], device="cuda"),
                      torch.exp(4 * torch.randn(300, generator=g, device="cuda"))]).to(t).float()
    half = torch.arange(-126, 127, device="cuda").double() + 0.5
    x = (most.double()[:, None] * half / 127.0).to(t)
    x = torch.cat([most.to(t)[:, None], x], 1)
    step = torch.finfo(t).eps
    for f in (1.0, 1.0 + step, 1.0 - step):
        y = (x.double() * f).to(t)
        y[:, 0] = most.to(t)
        check_quantise(y)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [9, 64, 2048, 5000, 40000])
def test_quantise_smallest_largest_and_not_finite(k, dtype):
    t = TYPES[dtype]
    x = make_map(10, k, t, 21)
    x[1] = (x[1].float() * 2.0 ** -140).to(t)                          # numbers below the normal range
    x[2] = (x[2].float() * 1e34).to(t)
    x[3, 0] = torch.finfo(t).max
    x[4, k // 2] = float("nan")
    x[5, k - 1] = float("inf")
    x[6, 0], x[6, 1] = float("-inf"), float("nan")
    x[7] = 0
    x[7, 3] = -torch.finfo(t).tiny
    check_quantise(x)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantise_strided_rows_and_what_lies_behind_them(dtype):
    x, _ = spread(make_map(21, 70, TYPES[dtype], 3), 83, 5)
    full = torch.full((21, 96), 55, dtype=torch.int8, device="cuda")
    check_quantise(x, full[:, :70])
    assert (full[:, 70:] == 55).all()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(1, 5), (40, 64), (33, 257), (50, 1024), (7, 4096), (3, 9000), (2, 16384)])
def test_norm_and_quantise_in_one_pass_has_the_bits_of_two(rows, c, dtype):
    g = gen(rows)
    x = make_map(rows, c, TYPES[dtype], c)
    if rows > 2:
        x[2, 0] = float("nan")
    gamma, beta = torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")
    y, q, scale = torch.empty_like(x), q_like(rows, c), torch.empty(rows, device="cuda")
    B.dc_layer_norm(x, gamma, beta, y)
    B.dc_quantize_rows(y, q, scale)
    y1, q1, s1 = torch.empty_like(x), q_like(rows, c), torch.empty(rows, device="cuda")
    B.dc_layer_norm_quantize(x, gamma, beta, q1, s1, y1)
    q2, s2 = q_like(rows, c), torch.empty(rows, device="cuda")
    B.dc_layer_norm_quantize(x, gamma, beta, q2, s2)

    def bits(t):
        return t.view(torch.int16 if t.element_size() == 2 else torch.int32) & (0x7fff if t.element_size() == 2 else 0x7fffffff)

    assert torch.equal(torch.nan_to_num(y.float(), nan=3.0), torch.nan_to_num(y1.float(), nan=3.0))
    assert torch.equal(q, q1) and torch.equal(q, q2) and torch.equal(bits(scale), bits(s1)) and torch.equal(bits(scale), bits(s2))


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(900, 64), (400, 512), (50, 2048), (700, 1000)])
def test_norm_and_quantise_with_an_output_that_is_not_aligned(rows, c, dtype):
    """The bits of the two calls where the map between them is aligned in both or in neither; else each within its bound, and its steps exact."""
    t, g = TYPES[dtype], gen(c)
    x = make_map(rows, c, t, rows)
    gamma, beta = torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")
    outs = [spread(torch.zeros_like(x), pitch, offset)[0] for pitch, offset in ((c, 0), (c + 1, 0), (c, 1), (c + 8, 3))]
    done = []
    for y in outs:
        check_norm(x, gamma, beta, y=y)
        q, s, q1, s1, y1 = q_like(rows, c), torch.empty(rows, device="cuda"), q_like(rows, c), torch.empty(rows, device="cuda"), spread(torch.zeros_like(x), y.stride(0), y.storage_offset())[0]
        B.dc_quantize_rows(y, q, s)
        B.dc_layer_norm_quantize(x, gamma, beta, q1, s1, y1)
        wq, ws = quantise64(y)
        assert torch.equal(y, y1) and torch.equal(q, q1) and torch.equal(s, s1) and torch.equal(q, wq) and torch.equal(s, ws)
        done.append((q, s))
    q, s = q_like(rows, c), torch.empty(rows, device="cuda")
    B.dc_layer_norm_quantize(x, gamma, beta, q, s)
    assert torch.equal(q, done[0][0]) and torch.equal(s, done[0][1])


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(400, 17), (300, 64), (200, 250), (200, 511), (100, 1001), (100, 2048), (60, 5001), (60, 7001), (30, 9001), (20, 16383)])
def test_norm_and_quantise_has_the_bits_of_two_with_any_weights(rows, c, dtype):
    """Rows of every kind of kernel, whole vectors and single elements, with either weight or none."""
    t, g = TYPES[dtype], gen(c)
    x, _ = spread(make_map(rows, c, t, 5), c + (3 if c % 2 else 8), c % 2)
    for gamma in (None, torch.randn(c, generator=g, device="cuda")):
        for beta in (None, torch.randn(c, generator=g, device="cuda")):
            y, y1, q, q1, q2 = torch.empty(rows, c, dtype=t, device="cuda"), torch.empty(rows, c, dtype=t, device="cuda"), q_like(rows, c), q_like(rows, c), q_like(rows, c)
            s, s1, s2 = (torch.empty(rows, device="cuda") for _ in range(3))
            check_norm(x, gamma, beta, y=y)
            B.dc_quantize_rows(y, q, s)
            B.dc_layer_norm_quantize(x, gamma, beta, q1, s1, y1)
            wq, ws = quantise64(y1)
            assert torch.equal(y, y1) and torch.equal(q, q1) and torch.equal(s, s1) and torch.equal(q1, wq) and torch.equal(s1, ws)
            B.dc_layer_norm_quantize(x, gamma, beta, q2, s2)
            if c % 8 == 0 or c * y.element_size() % 16:                # (the map is aligned alike: rows of whole 16 bytes, or single elements either way)
                assert torch.equal(q, q2) and torch.equal(s, s2)


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def random_q(rows, k, seed, pitch=None):
    g = gen(seed)
    q = torch.full((rows, pitch or (k + 15) // 16 * 16), 101, dtype=torch.int8, device="cuda")
    q[:, :k] = torch.randint(-128, 128, (rows, k), generator=g, device="cuda").to(torch.int8)
    return q[:, :k], torch.rand(rows, generator=g, device="cuda") * 0.01


def product64(a, sa, b, sb, bias, relu):
    """(out, bound of its error before it is rounded to the map's type): the sum to float32, two products and a sum, half a step each"""
    acc = (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()
    out = acc + (0.0 if bias is None else bias.double())
    bound = 4 * U * acc.abs() + U * out.abs()
    return (torch.where(out < 0, torch.zeros_like(out), out) if relu else out), bound


def check_product(a, sa, b, sb, bias, relu, dtype, out=None):
    out = torch.empty(a.shape[0], b.shape[0], dtype=dtype, device="cuda") if out is None else out
    B.dc_matmul_quantized(a, sa, b, sb, bias, out, relu)
    want, bound = product64(a, sa, b, sb, bias, relu)
    T = half_step(dtype)
    assert ((out.double() - want).abs() <= bound * (1 + T) + T * want.abs() + 1e-38).all()
    return out


PRODUCTS = [(1, 1, 1), (1, 16, 8), (1, 300, 77), (1, 4096, 1000), (2, 64, 64), (3, 1000, 130), (7, 128, 256), (8, 2048, 513), (9, 96, 40), (16, 512, 1024), (31, 4096, 200),
            (33, 160, 96), (64, 9216, 512), (100, 31, 33), (127, 129, 127), (128, 128, 128), (129, 257, 65), (200, 384, 1536), (256, 64, 1000), (300, 700, 17), (1000, 256, 64),
            (5000, 48, 24), (1, 64, 100000), (5, 48, 65537), (100352, 16, 8), (17, 131, 4097), (4096, 512, 2048), (4100, 520, 2050), (21952, 64, 256), (40000, 16, 8)]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", PRODUCTS)
def test_product(m, k, n, dtype):
    a, sa = random_q(m, k, m + k)
    b, sb = random_q(n, k, n + k + 1)
    g = gen(n)
    relu = (m + n) % 2 == 0
    check_product(a, sa, b, sb, torch.randn(n, generator=g, device="cuda") if k % 3 else None, relu, TYPES[dtype])


@gpu
@pytest.mark.parametrize("m", [1, 5, 40, 300])
def test_product_of_the_longest_rows_and_the_largest_values(m):
    k, n = 131071, 40
    a = torch.full((m, 131072), -128, dtype=torch.int8, device="cuda")[:, :k]
    b = torch.full((n, 131072), -128, dtype=torch.int8, device="cuda")[:, :k]
    b[1::2] = 127
    one = torch.ones(max(m, n), device="cuda")
    out = check_product(a, one[:m], b, one[:n], None, False, torch.float32)
    assert float(out[0, 0]) == 131071.0 * 16384.0


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n,pitch,offset", [(20, 100, 40, 48, 0), (150, 256, 250, 256, 0), (150, 64, 33, 40, 0), (300, 512, 1001, 1008, 0), (20, 100, 40, 41, 3), (150, 256, 250, 250, 1), (150, 256, 250, 301, 0), (1, 200, 33, 33, 1), (6, 200, 300, 333, 0)])
def test_product_into_strided_and_shifted_rows(m, k, n, pitch, offset, dtype):
    a, sa = random_q(m, k, 1, pitch=(k + 15) // 16 * 16 + 32)
    b, sb = random_q(n, k, 2, pitch=(k + 15) // 16 * 16 + 16)
    out, buf = spread(torch.zeros(m, n, dtype=TYPES[dtype], device="cuda"), pitch, offset)
    check_product(a, sa, b, sb, None, False, TYPES[dtype], out=out)
    rest = buf.clone()
    rest[offset:offset + m * pitch].view(m, pitch)[:, :n] = 77
    assert (rest == 77).all(), "something beside the rows was written"


@gpu
@pytest.mark.parametrize("pitch", [0, 16, 1 << 32, 1 << 41, (1 << 63) - 16])
def test_a_single_row_has_any_pitch(pitch):
    L, st = B.load(), torch.cuda.current_stream().cuda_stream
    for m, k, n in ((1, 300, 5), (1, 300, 1), (200, 300, 1), (1, 4096, 40000)):
        (a, sa), (b, sb) = random_q(m, k, 1), random_q(n, k, 2)
        want, got = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
        B.dc_matmul_quantized(a, sa, b, sb, None, want)
        assert L.dc_matmul_quantized(a.data_ptr(), pitch if m == 1 else a.stride(0), sa.data_ptr(), b.data_ptr(), pitch if n == 1 else b.stride(0), sb.data_ptr(), None,
                                     m, n, k, 0, B.DC_FP32, got.data_ptr(), pitch if m == 1 else 4 * n, st) == B.DC_OK
        assert torch.equal(got, want)
    x, y, want, q, wq, s, ws = *(torch.empty(1, 300, device="cuda") for _ in range(3)), q_like(1, 300), q_like(1, 300), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    x.copy_(make_map(1, 300, torch.float32, 4))
    B.dc_layer_norm(x, None, None, want)
    B.dc_quantize_rows(x, wq, ws)
    assert L.dc_layer_norm(x.data_ptr(), pitch, None, None, 1, 300, 1e-5, B.DC_FP32, y.data_ptr(), pitch, None, None, st) == B.DC_OK
    assert L.dc_quantize_rows(x.data_ptr(), pitch, 1, 300, B.DC_FP32, q.data_ptr(), pitch, s.data_ptr(), st) == B.DC_OK
    assert torch.equal(y, want) and torch.equal(q, wq) and torch.equal(s, ws)


@gpu
def test_product_of_rows_far_apart():
    """Rows of either side and of the output more than 4 GB apart."""
    k, pitch = 96, (1 << 32) + 16
    buf = torch.empty(2 * pitch + 4 * k, dtype=torch.int8, device="cuda")
    far = buf.as_strided((3, k), (pitch, 1))
    near, sn = random_q(3, k, 1)
    far.copy_(near)
    for rows in (40, 300):
        other, so = random_q(rows, k, 2)
        for a, sa, b, sb, c in ((far, sn, other, so, near), (other, so, far, sn, other)):
            assert torch.equal(check_product(a, sa, b, sb, None, False, torch.float32), check_product(c, sa, near if b is far else b, sb, None, False, torch.float32))
    out = torch.empty(2 * (pitch // 4) + 64, device="cuda").as_strided((3, 64), (pitch // 4, 1))
    b, sb = random_q(64, k, 3)
    check_product(near, sn, b, sb, None, True, torch.float32, out=out)


@gpu
@pytest.mark.parametrize("m", [1, 6, 64, 700])
@pytest.mark.parametrize("relu", [False, True])
def test_linear_has_the_bits_of_its_two_steps_and_keeps_what_is_not_finite_to_its_row(m, relu):
    k, n = 384, 200
    for dtype in TYPES.values():
        x = make_map(m, k, dtype, m)
        if m > 5:
            x[2, 7], x[4, 0], x[5] = float("nan"), float("inf"), 0.0
        w = torch.randn(n, k, generator=gen(3), device="cuda")
        wq, ws = q_like(n, k), torch.empty(n, device="cuda")
        B.dc_quantize_rows(w, wq, ws)
        bias = torch.randn(n, generator=gen(4), device="cuda")
        q, s, out = q_like(m, k), torch.empty(m, device="cuda"), torch.empty(m, n, dtype=dtype, device="cuda")
        B.dc_quantize_rows(x, q, s)
        B.dc_matmul_quantized(q, s, wq, ws, bias, out, relu)
        got = torch.empty_like(out)
        work = scratch(B.dc_linear_workspace(m, k) + 3)
        work.fill_(0x5a)
        B.dc_linear_quantized(x, wq, ws, bias, got, relu, work[3:])
        bad = ~torch.isfinite(x.float()).all(1)
        assert torch.isnan(got[bad].float()).all() and torch.isnan(out[bad].float()).all()
        assert torch.equal(got[~bad], out[~bad])
        good = ~bad
        check = product64(q[good], s[good], wq, ws, bias, relu)
        T = half_step(dtype)
        assert ((got[good].double() - check[0]).abs() <= check[1] * (1 + T) + T * check[0].abs()).all()
        if m > 5:
            row = torch.where(bias < 0, torch.zeros_like(bias), bias) if relu else bias
            assert torch.equal(got[5], row.to(dtype))                  # a row of zeros leaves the bias


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", [(1, 1, 1), (1, 16, 3), (1, 17, 70), (1, 100, 50), (1, 1000, 300), (1, 4096, 4099), (1, 30001, 20), (2, 7, 5), (2, 512, 600), (2, 2049, 64),
                                   (2, 100000, 8), (3, 64, 64), (3, 333, 77), (4, 1024, 256), (5, 130, 9), (7, 585, 40), (8, 512, 1000), (8, 5, 3)])
def test_linear_of_one_row_and_of_a_few_short_ones(m, k, n, dtype):
    t = TYPES[dtype]
    x, _ = spread(make_map(m, k, t, m + k), k + 3 if k % 2 else k + 8, 5 if n % 2 else 0)
    if m > 2:
        x[1] = 0
        x[2, k // 2] = float("nan")
    if m > 4:
        x[3] = (x[3].float() * 2.0 ** -130).to(t)
        x[4] = (x[4].float() * 1e30).to(t)
    w, ws = random_q(n, k, k)
    bias = torch.randn(n, generator=gen(4), device="cuda") if n % 3 else None
    for relu in (False, True):
        out, buf = spread(torch.zeros(m, n, dtype=t, device="cuda"), n + 7, 1)
        B.dc_linear_quantized(x, w, ws, bias, out, relu, scratch(B.dc_linear_workspace(m, k)))
        q, s = quantise64(x)
        good = torch.isfinite(x.float()).all(1)
        want, bound = product64(q[good], s[good], w, ws, bias, relu)
        T = half_step(t)
        assert ((out[good].double() - want).abs() <= bound * (1 + T) + T * want.abs() + 1e-38).all()
        assert torch.isnan(out[~good].float()).all()
        rest = buf.clone()
        rest[1:1 + m * (n + 7)].view(m, n + 7)[:, :n] = 77
        assert (rest == 77).all()


@gpu
@pytest.mark.parametrize("m,k,n", [(1, 12688, 4098), (1, 12704, 4094), (1, 12704, 4090), (2, 2928, 4098), (2, 2944, 4077)])
def test_linear_on_either_side_of_the_single_launch(m, k, n):
    """Weights just above and just below what the single launch takes: the bits of the two steps."""
    x = make_map(m, k, torch.bfloat16, 2)
    wq, ws = random_q(n, k, 3)
    q, s, want, got = q_like(m, k), torch.empty(m, device="cuda"), torch.empty(m, n, dtype=torch.bfloat16, device="cuda"), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    B.dc_quantize_rows(x, q, s)
    B.dc_matmul_quantized(q, s, wq, ws, None, want)
    B.dc_linear_quantized(x, wq, ws, None, got, False, scratch(B.dc_linear_workspace(m, k)))
    assert torch.equal(got, want)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", [(1, 1024, 1024), (1, 4096, 4096), (1, 512, 9000), (1, 9000, 64), (2, 2048, 2048), (4, 1024, 256), (8, 512, 512), (64, 512, 512)])
def test_linear_over_its_own_input(m, k, n, dtype):
    """out over x, at its start, beginning in its middle and one element in front of it: the bits of an output apart."""
    t = TYPES[dtype]
    wide = max(k, n)
    wq, ws = random_q(n, k, 5)
    bias = torch.randn(n, generator=gen(6), device="cuda")
    work = scratch(B.dc_linear_workspace(m, k))
    data = make_map(m, k, t, m + n)
    want = torch.empty(m, n, dtype=t, device="cuda")
    B.dc_linear_quantized(data, wq, ws, bias, want, True, work)
    buf = torch.empty(3 * m * wide + 64, dtype=t, device="cuda")
    x = buf[m * wide:2 * m * wide].view(m, wide)[:, :k]
    for offset in (0, wide // 2, -1, wide - n, -m * wide + 8):
        for _ in range(5):
            x.copy_(data)
            out = buf[m * wide + offset:2 * m * wide + offset].view(m, wide)[:, :n]
            B.dc_linear_quantized(x, wq, ws, bias, out, True, work)
            assert torch.equal(out, want), offset
    x, out = buf[:m * (k + n)].view(m, k + n).split([k, n], 1)         # columns of one buffer: apart
    x.copy_(data)
    B.dc_linear_quantized(x, wq, ws, bias, out, True, work)
    assert torch.equal(out, want) and torch.equal(x, data)


@gpu
@pytest.mark.parametrize("k,n", [(20000, 33), (25088, 256), (70000, 16)])
def test_linear_of_long_rows(k, n):
    for m in (1, 3, 33):
        x = make_map(m, k, torch.bfloat16, m).relu()
        wq, ws = random_q(n, k, 5)
        out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
        B.dc_linear_quantized(x, wq, ws, None, out, False, scratch(B.dc_linear_workspace(m, k)))
        q, s = quantise64(x)
        want, bound = product64(q, s, wq, ws, None, False)
        T = half_step(torch.bfloat16)
        assert ((out.double() - want).abs() <= bound * (1 + T) + T * want.abs()).all()


# ---------------------------------------------------------------------------
# together, on streams, in graphs
# ---------------------------------------------------------------------------
def chain(x, gamma, beta, w1, s1, w2, s2, out, q, qs, mid, work):
    B.dc_layer_norm_quantize(x, gamma, beta, q, qs)
    B.dc_matmul_quantized(q, qs, w1, s1, None, mid, True)
    B.dc_linear_quantized(mid, w2, s2, beta, out, False, work)


def chain_buffers(m, c, seed, dtype=torch.bfloat16):
    wide = 4 * c
    w1, s1 = random_q(wide, c, seed + 1)
    w2, s2 = random_q(c, wide, seed + 2)
    g = gen(seed)
    return (make_map(m, c, dtype, seed), 1 + 0.1 * torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda"), w1, s1, w2, s2,
            torch.empty(m, c, dtype=dtype, device="cuda"), q_like(m, c), torch.empty(m, device="cuda"), torch.empty(m, wide, dtype=dtype, device="cuda"),
            scratch(B.dc_linear_workspace(m, wide)))


@gpu
@pytest.mark.parametrize("m", [1, 4, 50, 900])
def test_a_run_of_them_eager_on_another_stream_and_replayed(m):
    c = 96
    b = chain_buffers(m, c, 30 + m)
    x, gamma, beta, w1, s1, w2, s2, out, q, qs, mid, work = b
    chain(*b)
    eager = out.clone()
    y = torch.empty_like(x)
    B.dc_layer_norm(x, gamma, beta, y)
    q64, sc64 = quantise64(y)
    assert torch.equal(q, q64) and torch.equal(qs, sc64)
    q64, sc64 = quantise64(mid)
    want, bound = product64(q64, sc64, w2, s2, beta, False)
    T = half_step(torch.bfloat16)
    assert ((out.double() - want).abs() <= bound * (1 + T) + T * want.abs()).all()
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(*b)
    side.synchronize()
    assert torch.equal(out, eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(*b)
    keep = x.clone()
    for _ in range(3):
        x.copy_(torch.flip(keep, [0]))
        graph.replay()
        assert torch.equal(out, torch.flip(eager, [0]))
        x.copy_(keep)
        out.zero_()
        graph.replay()
        assert torch.equal(out, eager)


@gpu
def test_gradients_captured_into_a_graph():
    x, dy = make_map(400, 160, torch.bfloat16, 1), make_map(400, 160, torch.bfloat16, 2)
    _, mean, rstd, _ = norm64(x, None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    want = run_backward(dy, x, None, mean, rstd)
    dx, dg, db, work = torch.empty_like(x), torch.empty(160, device="cuda"), torch.empty(160, device="cuda"), scratch(B.dc_layer_norm_workspace(160))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.dc_layer_norm_backward(dy, x, None, mean, rstd, dx, dg, db, work)
    for _ in range(2):
        dx.zero_(), dg.zero_(), db.zero_()
        graph.replay()
        assert torch.equal(dx, want[0]) and torch.equal(dg, want[1]) and torch.equal(db, want[2])


@gpu
def test_two_calls_at_once_on_two_streams():
    a, b = chain_buffers(700, 128, 1), chain_buffers(333, 64, 2)
    chain(*a), chain(*b)
    want = a[7].clone(), b[7].clone()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    a[7].zero_(), b[7].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(s1):
            chain(*a)
        with torch.cuda.stream(s2):
            chain(*b)
    torch.cuda.synchronize()
    assert torch.equal(a[7], want[0]) and torch.equal(b[7], want[1])


@gpu
@pytest.mark.parametrize("m,k,n", [(1, 4096, 512), (20, 9216, 256), (300, 512, 300)])
def test_weights_written_just_before_the_product(m, k, n):
    """A product may start loading weights before the rows of x are ready, but not before what was enqueued in front of the call is done."""
    x = make_map(m, k, torch.bfloat16, 1)
    work, out = scratch(B.dc_linear_workspace(m, k)), torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    ws = [torch.randn(n, k, generator=gen(i), device="cuda") for i in range(4)]
    big = torch.randn(64 << 20, device="cuda")
    wq, sc = q_like(n, k), torch.empty(n, device="cuda")
    want, got = [], []
    for w in ws:
        B.dc_quantize_rows(w, wq, sc)
        torch.cuda.synchronize()
        B.dc_linear_quantized(x, wq, sc, None, out, False, work)
        torch.cuda.synchronize()
        want.append(out.clone())
    kept = [(q_like(n, k), torch.empty(n, device="cuda")) for _ in ws]
    for w, (q, s) in zip(ws, kept):
        B.dc_quantize_rows(w, q, s)
    for _ in range(5):
        for i, w in enumerate(ws):
            big.mul_(1.0)                                               # something long in front
            if i % 2:
                B.dc_quantize_rows(w, wq, sc)
            else:
                wq.copy_(kept[i][0]), sc.copy_(kept[i][1])
            o = torch.empty_like(out)
            B.dc_linear_quantized(x, wq, sc, None, o, False, work)
            got.append((i, o))
    assert all(torch.equal(o, want[i]) for i, o in got)


@gpu
@pytest.mark.parametrize("c", [256, 100, 1024])
def test_weights_that_the_kernel_before_writes(c):
    """gamma, beta, scales and biases are read after the kernel in front is done: here it is the last one of the gradients, which lets its successor
    start early."""
    rows = 3000
    x, dy = make_map(rows, c, torch.bfloat16, 1), make_map(rows, c, torch.bfloat16, 2)
    _, mean, rstd, _ = norm64(x, None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    _, dg, db = run_backward(dy, x, None, mean, rstd)
    y, q, s = torch.empty_like(x), q_like(rows, c), torch.empty(rows, device="cuda")
    B.dc_layer_norm(x, dg, db, y)
    B.dc_quantize_rows(y, q, s)
    w, _ = random_q(c, c, 3)
    out = torch.empty(rows, c, dtype=torch.bfloat16, device="cuda")
    B.dc_matmul_quantized(q, s, w, db, dg, out)
    few, want_few = q[:5], torch.empty(5, c, dtype=torch.bfloat16, device="cuda")
    B.dc_matmul_quantized(few, s[:5], w, db, dg, want_few)
    want_dx, _, _ = run_backward(dy, x, dg, mean, rstd)
    torch.cuda.synchronize()
    g, b, work = torch.empty(c, device="cuda"), torch.empty(c, device="cuda"), scratch(B.dc_layer_norm_workspace(c))
    got = []
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                                      # one right behind the other
        for i in range(40):
            g.fill_(-1.0), b.fill_(2.0)
            B.dc_layer_norm_backward(dy, x, None, mean, rstd, None, g, b, work)
            if i % 4 == 0:
                o = torch.empty_like(y)
                B.dc_layer_norm(x, g, b, o)
                got.append((o, y))
            elif i % 4 == 1:
                o = torch.empty_like(out)
                B.dc_matmul_quantized(q, s, w, b, g, o)
                got.append((o, out))
            elif i % 4 == 2:
                o = torch.empty_like(want_few)
                B.dc_matmul_quantized(few, s[:5], w, b, g, o)
                got.append((o, want_few))
            else:
                o = torch.empty_like(want_dx)
                B.dc_layer_norm_backward(dy, x, g, mean, rstd, o)
                got.append((o, want_dx))
    for _ in range(3):
        graph.replay()
    assert all(torch.equal(a, b) for a, b in got)


FIRST_CALL_IN_A_CAPTURE = """
import torch
from paper_1712_01670_b200 import binding as B
x = torch.randn(40, 4096, device="cuda").bfloat16()
w, s, out = torch.randint(-127, 128, (512, 4096), device="cuda").to(torch.int8), torch.rand(512, device="cuda"), torch.empty(40, 512, device="cuda").bfloat16()
big, o2 = torch.randn(20000, 96, device="cuda"), torch.empty(20000, 64, device="cuda")
w2 = torch.randint(-127, 128, (64, 96), device="cuda").to(torch.int8)
work, work2 = torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
y, mean, rstd = torch.empty_like(big), torch.empty(20000, device="cuda"), torch.empty(20000, device="cuda")
dg, db = torch.empty(96, device="cuda"), torch.empty(96, device="cuda")
torch.cuda.synchronize()
def run():
    B.dc_linear_quantized(x, w, s, None, out, True, work)
    B.dc_linear_quantized(big, w2, s[:64], None, o2, False, work2)
    B.dc_layer_norm(big, None, None, y, mean, rstd)
    B.dc_layer_norm_backward(big, big, None, mean, rstd, None, dg, db, work2)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    run()
g.replay()
torch.cuda.synchronize()
kept = [t.clone() for t in (out, o2, y, dg, db)]
run()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(kept, (out, o2, y, dg, db)))
print("the same")
"""


FIRST_CALLS_OF_THREADS = """
import threading
import torch
from paper_1712_01670_b200 import binding as B
N = 6
x = torch.randn(2100, 768, device="cuda").bfloat16()
w, s = torch.randint(-127, 128, (512, 768), device="cuda").to(torch.int8), torch.rand(512, device="cuda")
mean, rstd = x.float().mean(1), 1 / x.float().std(1)
bufs = [[torch.empty(n, dtype=torch.uint8, device="cuda") for n in (1 << 22, B.dc_layer_norm_workspace(768))] +
        [torch.empty(m, 512, device="cuda").bfloat16() for m in (1, 30, 2100)] + [torch.empty_like(x), torch.empty(768, device="cuda"), torch.empty(768, device="cuda")] for _ in range(N)]
streams = [torch.cuda.Stream() for _ in range(N)]
torch.cuda.synchronize()
gate, failed = threading.Barrier(N), []
def run(i):
    try:
        work, partial, one, few, many, dx, dg, db = bufs[i]
        gate.wait()
        with torch.cuda.stream(streams[i]):
            B.dc_linear_quantized(x[:1], w, s, None, one, True, work)
            B.dc_linear_quantized(x[:30], w, s, None, few, True, work)
            B.dc_linear_quantized(x, w, s, None, many, True, work)
            B.dc_layer_norm_backward(x, x, None, mean, rstd, dx, dg, db, partial)
    except Exception as e:
        failed.append(repr(e))
threads = [threading.Thread(target=run, args=(i,)) for i in range(N)]
for t in threads: t.start()
for t in threads: t.join()
torch.cuda.synchronize()
assert not failed, failed
assert all(torch.equal(p, q) for b in bufs[1:] for p, q in zip(bufs[0][2:], b[2:]))
assert torch.equal(bufs[0][4][:1], bufs[0][2]) and torch.equal(bufs[0][4][:30], bufs[0][3])
print("the same")
"""


@gpu
def test_the_first_calls_of_a_process_from_several_threads():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS_OF_THREADS], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "the same" in r.stdout, r.stdout + r.stderr


FIRST_C_CALLS_OF_THREADS = """
import ctypes as C
import threading
import time
import torch
from paper_1712_01670_b200 import binding as B
N, K, M = 6, 768, 2100
L = B.load()
xs = [torch.randn(M, K, device="cuda"), torch.randn(M, K, device="cuda").bfloat16()]
w, s = torch.randint(-127, 128, (512, K), device="cuda").to(torch.int8), torch.rand(512, device="cuda")
stats = [(x.float().mean(1), 1 / x.float().std(1)) for x in xs]
def buffers():
    per_type = [[torch.empty(m, 512, device="cuda").to(x.dtype) for m in (1, 30, 300, M) for relu in (0, 1)] + [torch.empty_like(x), torch.empty(K, device="cuda"), torch.empty(K, device="cuda")] for x in xs]
    return [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (1 << 22, B.dc_layer_norm_workspace(K))], per_type
def calls_of(bufs, stream):                    # arguments made beforehand: a thread only calls
    (work, partial), per_type = bufs
    st, got = stream.cuda_stream, []
    for dtype, x, (mean, rstd), outs in zip((B.DC_FP32, B.DC_BF16), xs, stats, per_type):
        pitch, out_pitch = K * x.element_size(), 512 * x.element_size()
        for i, m in enumerate((1, 30, 300, M)):
            for relu in (0, 1):
                got.append((L.dc_linear_quantized, (x.data_ptr(), pitch, w.data_ptr(), K, s.data_ptr(), None, m, 512, K, relu, dtype, outs[2 * i + relu].data_ptr(), out_pitch,
                                                    work.data_ptr(), 1 << 22, st)))
        got.append((L.dc_layer_norm_backward, (x.data_ptr(), pitch, x.data_ptr(), pitch, None, mean.data_ptr(), rstd.data_ptr(), M, K, dtype, outs[8].data_ptr(), pitch,
                                               outs[9].data_ptr(), outs[10].data_ptr(), partial.data_ptr(), partial.numel(), st)))
    return got
bufs = [buffers() for _ in range(N)]
streams = [torch.cuda.Stream() for _ in range(N)]
todo = [calls_of(b, t) for b, t in zip(bufs, streams)]
torch.cuda.synchronize()
gate, at, codes = threading.Barrier(N), [[] for _ in range(N)], [[] for _ in range(N)]
def run(i):
    for f, a in todo[i]:
        gate.wait()
        t = time.perf_counter_ns()
        codes[i].append(f(*a))
        at[i].append((t, time.perf_counter_ns()))
threads = [threading.Thread(target=run, args=(i,)) for i in range(N)]
for t in threads: t.start()
for t in threads: t.join()
torch.cuda.synchronize()
assert all(c == [0] * len(todo[0]) for c in codes), codes
at_once = sum(any(p is not q and max(p[0], q[0]) < min(p[1], q[1]) for p in spans for q in spans) for spans in zip(*at))
assert at_once > len(todo[0]) // 2, f"of {len(todo[0])} calls only {at_once} were made by two threads at once"
outs = [[t for p in b[1] for t in p] for b in bufs]
assert all(torch.equal(p, q) for o in outs[1:] for p, q in zip(outs[0], o))
again = [t.clone() for t in outs[0]]
for f, a in todo[0]:
    assert f(*a) == 0
torch.cuda.synchronize()
assert all(torch.equal(p, q) for p, q in zip(again, outs[0]))
print("the same")
"""


@gpu
def test_the_first_c_calls_of_a_process_overlap():
    """Through the C ABI, which holds no lock: the first calls of several threads are in the library at the same time, all succeed and agree."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_C_CALLS_OF_THREADS], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "the same" in r.stdout, r.stdout + r.stderr


@gpu
def test_the_first_call_of_a_process_inside_a_capture():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL_IN_A_CAPTURE], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "the same" in r.stdout, r.stdout + r.stderr


@gpu
def test_other_python_threads_run_during_a_call():
    """With no forced switches between threads, another thread can only have run between two calls if a call gave it the interpreter."""
    import sys
    import threading
    import time
    rows, c = 40, 64
    x = make_map(rows, c, torch.float32, 1)
    y, dx, q, s, out, work = torch.empty_like(x), torch.empty_like(x), q_like(rows, c), torch.empty(rows, device="cuda"), torch.empty(rows, 8, device="cuda"), scratch(1 << 20)
    w, ws = random_q(8, c, 2)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    calls = [lambda: B.dc_layer_norm(x, None, None, y), lambda: B.dc_layer_norm_backward(x, x, None, mean, rstd, dx), lambda: B.dc_quantize_rows(x, q, s),
             lambda: B.dc_layer_norm_quantize(x, None, None, q, s), lambda: B.dc_matmul_quantized(q, s, w, ws, None, out),
             lambda: B.dc_linear_quantized(x, w, ws, None, out, False, work)]
    turns, stop, before = [0], [], sys.getswitchinterval()

    def other():
        while not stop:
            turns[0] += 1
            time.sleep(0)                                              # hands the interpreter back

    for call in calls:
        call()
    torch.cuda.synchronize()
    sys.setswitchinterval(100.0)
    thread = threading.Thread(target=other)
    try:
        thread.start()
        seen = []
        for call in calls:
            t = turns[0]
            for _ in range(1000):
                call()
            seen.append(turns[0] - t)
    finally:
        stop.append(1)
        sys.setswitchinterval(before)
        thread.join()
    torch.cuda.synchronize()
    assert min(seen) > 0, seen


@gpu
def test_nothing_is_done_with_no_rows():
    x = torch.empty(0, 32, device="cuda")
    w, s = random_q(8, 32, 1)
    B.dc_layer_norm(x, None, None, x)
    q, qs = torch.empty(0, 32, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda")
    B.dc_quantize_rows(x, q, qs)
    B.dc_layer_norm_quantize(x, None, None, q, qs)
    out = torch.empty(0, 8, device="cuda")
    B.dc_matmul_quantized(q, qs, w, s, None, out)
    B.dc_linear_quantized(x, w, s, None, out, workspace=scratch(256))
    torch.cuda.synchronize()


@gpu
def test_maps_of_several_dimensions():
    x = make_map(2 * 5 * 7, 64, torch.float32, 1).view(2, 5, 7, 64)
    y, z = torch.empty_like(x), torch.empty(70, 64, device="cuda")
    B.dc_layer_norm(x, None, None, y)
    B.dc_layer_norm(x.reshape(70, 64), None, None, z)
    assert torch.equal(y.view(70, 64), z)
    with pytest.raises(ValueError):
        B.dc_layer_norm(x.transpose(1, 2), None, None, y.transpose(1, 2))


# ---------------------------------------------------------------------------
# refusals (no GPU: an argument is refused before any CUDA call)
# ---------------------------------------------------------------------------
P = C.c_void_p(1 << 20)                # an aligned address that nothing reads


def call(name, **kw):
    order = {
        "dc_layer_norm": ["x", "xp", "gamma", "beta", "rows", "c", "eps", "dtype", "y", "yp", "mean", "rstd", "stream"],
        "dc_layer_norm_backward": ["dy", "dyp", "x", "xp", "gamma", "mean", "rstd", "rows", "c", "dtype", "dx", "dxp", "dgamma", "dbeta", "work", "bytes", "stream"],
        "dc_quantize_rows": ["x", "xp", "rows", "c", "dtype", "q", "qp", "scale", "stream"],
        "dc_layer_norm_quantize": ["x", "xp", "gamma", "beta", "rows", "c", "eps", "dtype", "y", "yp", "q", "qp", "scale", "stream"],
        "dc_matmul_quantized": ["q", "qp", "scale", "w", "wp", "ws", "bias", "rows", "n", "c", "relu", "dtype", "y", "yp", "stream"],
        "dc_linear_quantized": ["x", "xp", "w", "wp", "ws", "bias", "rows", "n", "c", "relu", "dtype", "y", "yp", "work", "bytes", "stream"],
    }[name]
    base = dict(x=P, xp=256, gamma=P, beta=P, rows=0, c=64, n=64, eps=1e-5, dtype=B.DC_FP32, y=P, yp=256, mean=P, rstd=P, dy=P, dyp=256, dx=P, dxp=256, dgamma=P, dbeta=P,
                work=P, bytes=1 << 30, q=P, qp=64, scale=P, w=P, wp=64, ws=P, bias=P, relu=0, stream=None)
    base.update(kw)
    return getattr(B.load(), name)(*[base[k] for k in order])


ODD = C.c_void_p((1 << 20) + 2)
ODD1 = C.c_void_p((1 << 20) + 1)


@pytest.mark.parametrize("name,kw,status", [
    ("dc_layer_norm", dict(), B.DC_OK),                               # no rows
    ("dc_layer_norm", dict(rows=-1), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(c=0), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(c=16385), B.DC_ERR_LIMIT),
    ("dc_layer_norm", dict(dtype=2), B.DC_ERR_CONFIG),
    ("dc_layer_norm", dict(eps=-1e-9), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(eps=float("nan")), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(rows=2, x=None), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(rows=2, y=None), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(rows=2, xp=252), B.DC_ERR_ARG),            # rows would overlap
    ("dc_layer_norm", dict(rows=2, yp=0), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(rows=2, xp=258), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(rows=2, x=ODD), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(rows=2, x=ODD1, dtype=B.DC_BF16), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(rows=2, gamma=ODD), B.DC_ERR_ARG),
    ("dc_layer_norm", dict(rows=2, mean=ODD), B.DC_ERR_ARG),
    ("dc_layer_norm_backward", dict(rows=-5), B.DC_ERR_ARG),
    ("dc_layer_norm_backward", dict(c=20000), B.DC_ERR_LIMIT),
    ("dc_layer_norm_backward", dict(dtype=-1), B.DC_ERR_CONFIG),
    ("dc_layer_norm_backward", dict(rows=3, work=None), B.DC_ERR_ARG),
    ("dc_layer_norm_backward", dict(rows=3, bytes=296 * 8 * 64 - 1), B.DC_ERR_ARG),
    ("dc_layer_norm_backward", dict(rows=3, work=C.c_void_p((1 << 20) + 8)), B.DC_ERR_ARG),
    ("dc_layer_norm_backward", dict(rows=3, mean=None), B.DC_ERR_ARG),
    ("dc_layer_norm_backward", dict(rows=3, rstd=None), B.DC_ERR_ARG),
    ("dc_layer_norm_backward", dict(rows=3, dy=None), B.DC_ERR_ARG),
    ("dc_layer_norm_backward", dict(rows=3, dxp=128), B.DC_ERR_ARG),
    ("dc_layer_norm_backward", dict(rows=3, dx=None, dgamma=None, dbeta=None, work=None), B.DC_OK),   # nothing wanted
    ("dc_layer_norm", dict(rows=0x7ff00001), B.DC_ERR_LIMIT),
    ("dc_layer_norm", dict(rows=2, yp=1 << 32), B.DC_ERR_LIMIT),
    ("dc_layer_norm_backward", dict(rows=2, dyp=1 << 32), B.DC_ERR_LIMIT),
    ("dc_quantize_rows", dict(rows=2, xp=1 << 40), B.DC_ERR_LIMIT),
    ("dc_linear_quantized", dict(rows=2, xp=1 << 32), B.DC_ERR_LIMIT),
    ("dc_quantize_rows", dict(rows=-1), B.DC_ERR_ARG),
    ("dc_quantize_rows", dict(rows=2, q=None), B.DC_ERR_ARG),
    ("dc_quantize_rows", dict(rows=2, scale=None), B.DC_ERR_ARG),
    ("dc_quantize_rows", dict(rows=2, qp=72), B.DC_ERR_ARG),
    ("dc_quantize_rows", dict(rows=2, qp=48), B.DC_ERR_ARG),
    ("dc_quantize_rows", dict(rows=2, q=C.c_void_p((1 << 20) + 8)), B.DC_ERR_ARG),
    ("dc_quantize_rows", dict(rows=2, dtype=5), B.DC_ERR_CONFIG),
    ("dc_layer_norm_quantize", dict(rows=2, q=None), B.DC_ERR_ARG),
    ("dc_layer_norm_quantize", dict(rows=2, yp=4), B.DC_ERR_ARG),
    ("dc_layer_norm_quantize", dict(rows=2, c=16400, qp=16400, xp=65600, y=None), B.DC_ERR_LIMIT),
    ("dc_matmul_quantized", dict(rows=-1), B.DC_ERR_ARG),
    ("dc_matmul_quantized", dict(n=0), B.DC_ERR_ARG),
    ("dc_matmul_quantized", dict(c=0), B.DC_ERR_ARG),
    ("dc_matmul_quantized", dict(c=131072, qp=131072, wp=131072), B.DC_ERR_LIMIT),
    ("dc_matmul_quantized", dict(rows=1 << 31), B.DC_ERR_LIMIT),
    ("dc_matmul_quantized", dict(rows=2, scale=None), B.DC_ERR_ARG),
    ("dc_matmul_quantized", dict(rows=2, w=None), B.DC_ERR_ARG),
    ("dc_matmul_quantized", dict(rows=2, wp=56), B.DC_ERR_ARG),
    ("dc_matmul_quantized", dict(rows=2, qp=32), B.DC_ERR_ARG),
    ("dc_matmul_quantized", dict(rows=2, q=ODD), B.DC_ERR_ARG),
    ("dc_matmul_quantized", dict(rows=2, yp=128), B.DC_ERR_ARG),
    ("dc_matmul_quantized", dict(rows=2, dtype=7), B.DC_ERR_CONFIG),
    ("dc_linear_quantized", dict(rows=2, work=None), B.DC_ERR_ARG),
    ("dc_linear_quantized", dict(rows=2, bytes=2 * 68 + 255), B.DC_ERR_ARG),
    ("dc_linear_quantized", dict(rows=2, x=None), B.DC_ERR_ARG),
    ("dc_linear_quantized", dict(rows=2, xp=128), B.DC_ERR_ARG),
    ("dc_linear_quantized", dict(rows=2, bias=ODD), B.DC_ERR_ARG),
])
def test_refusals(name, kw, status):
    assert call(name, **kw) == status


@pytest.mark.parametrize("name,kw", [("dc_matmul_quantized", dict(rows=2, qp=1 << 40)), ("dc_matmul_quantized", dict(rows=2, wp=1 << 40)), ("dc_matmul_quantized", dict(rows=1, wp=1 << 60)),
                                     ("dc_linear_quantized", dict(rows=1, wp=1 << 40))])
def test_operands_too_far_apart_are_refused(name, kw):
    assert call(name, **kw) == B.DC_ERR_LIMIT


def test_workspaces():
    assert B.dc_layer_norm_workspace(100) == 296 * 2 * 4 * 100
    assert B.dc_linear_workspace(3, 17) == 3 * 36 + 256
    n = C.c_size_t()
    assert B.load().dc_layer_norm_workspace(0, C.byref(n)) == B.DC_ERR_ARG
    assert B.load().dc_linear_workspace(1, 0, C.byref(n)) == B.DC_ERR_ARG
    assert B.load().dc_linear_workspace(1, 1, None) == B.DC_ERR_ARG


def test_binding_refuses_what_does_not_fit_together():
    x, q, s = torch.zeros(3, 32), torch.zeros(3, 32, dtype=torch.int8), torch.zeros(3)
    with pytest.raises(ValueError):
        B.dc_layer_norm(x, None, None, torch.zeros(3, 31))
    with pytest.raises(TypeError):
        B.dc_layer_norm(x, None, None, torch.zeros(3, 32, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        B.dc_layer_norm(x.double(), None, None, x.double())
    with pytest.raises(ValueError):
        B.dc_layer_norm(x, torch.zeros(31), None, x)
    with pytest.raises(ValueError):
        B.dc_layer_norm(x.t(), None, None, x.t())
    with pytest.raises(ValueError):
        B.dc_layer_norm(x, None, None, x)                              # no CUDA tensors
    with pytest.raises(ValueError):
        B.dc_layer_norm_backward(x, x, None, None, s, x)
    with pytest.raises(ValueError):
        B.dc_quantize_rows(x, q[:2], s)
    with pytest.raises(TypeError):
        B.dc_quantize_rows(x, x, s)
    with pytest.raises(ValueError):
        B.dc_matmul_quantized(q, s, torch.zeros(5, 31, dtype=torch.int8), torch.zeros(5), None, torch.zeros(3, 5))
    with pytest.raises(ValueError):
        B.dc_matmul_quantized(q, s, torch.zeros(5, 32, dtype=torch.int8), torch.zeros(4), None, torch.zeros(3, 5))
    with pytest.raises(ValueError):
        B.dc_linear_quantized(x, torch.zeros(5, 32, dtype=torch.int8), torch.zeros(5), None, torch.zeros(3, 4))
