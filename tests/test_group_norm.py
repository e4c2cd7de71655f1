"""Group normalisation with an activation, channels last, and its gradients, against plain 64-bit implementations.

Tolerances: u = 2^-24 is half a step of float32, T(t) half a step of the map's type, relative to the value.  Values are added up as distances from one of them,
none larger than the group's range R.  A thread adds no more than 200 of them one behind another here, and at most 24 joins (threads, CTAs, chunks) follow,
so a sum of N terms is off by at most DEPTH u times the sum of their sizes, DEPTH = 224.
"""
import ctypes as C

import pytest
import torch

from paper_1712_01670_b200 import binding as B

U = 2.0 ** -24
DEPTH = 224
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = {"none": B.DC_ACT_NONE, "relu": B.DC_ACT_RELU, "silu": B.DC_ACT_SILU}
EPS = 1e-5
gpu = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make(maps, pixels, c, dtype, seed, shift=0.7):
    g = gen(seed)
    x = torch.randn(maps, pixels, c, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(c, generator=g, device="cuda")) + shift
    return x.to(dtype)


def weights(c, seed):
    g = gen(seed)
    return torch.randn(c, generator=g, device="cuda"), torch.randn(c, generator=g, device="cuda")


def scratch(maps, pixels, c, groups):
    return torch.full((B.dc_group_norm_workspace(maps, pixels, c, groups),), 0x7F, dtype=torch.uint8, device="cuda")


def spread(x, pitch, offset):
    """The same rows `pitch` elements apart, `offset` elements behind the start of an allocation."""
    maps, pixels, c = x.shape
    buf = torch.full((maps * pixels * pitch + offset + 64,), 77, dtype=x.dtype, device=x.device)
    view = buf[offset:offset + maps * pixels * pitch].view(maps, pixels, pitch)[..., :c]
    view.copy_(x)
    return view, buf


def untouched(buf, pitch, offset, c, rows):
    rest = buf.clone()
    rest[offset:offset + rows * pitch].view(rows, pitch)[:, :c] = 77
    return bool((rest == 77).all())


def split(x, groups):
    maps, pixels, c = x.shape
    return x.double().view(maps, pixels, groups, c // groups)


def wide(t, c):
    """[maps, groups] as [maps, 1, c]"""
    return t.repeat_interleave(c // t.shape[1], 1).unsqueeze(1)


def act64(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.where(z == z, torch.zeros_like(z), z))
    return z * torch.sigmoid(z) if act == "silu" else z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    p = torch.sigmoid(z)
    return p * (1 + z * (1 - p)) if act == "silu" else torch.ones_like(z)


def check_norm(x, groups, gamma, beta, act="none", eps=EPS, y=None):
    maps, pixels, c = x.shape
    y = torch.empty(maps, pixels, c, dtype=x.dtype, device="cuda") if y is None else y
    mean, rstd = torch.empty(maps, groups, device="cuda"), torch.empty(maps, groups, device="cuda")
    v = split(x, groups)
    wmean, n = v.mean((1, 3)), pixels * (c // groups)
    var = (v - wmean[:, None, :, None]).square().mean((1, 3))
    wrstd = (var + eps).rsqrt()
    size = v.abs().amax((1, 3))
    span = v.amax((1, 3)) - v.amin((1, 3))
    d = x.double() - wide(wmean, c)                       # before the call: y may be x
    B.dc_group_norm(x, groups, gamma, beta, y, mean, rstd, ACTS[act], eps, scratch(maps, pixels, c, groups))
    # the mean: a sum of distances, then the value that they were taken from; the squares: sums of squares up to R^2 and the mean's own square taken off
    dm = DEPTH * U * span + 4 * U * size
    dv = 4 * DEPTH * U * span.square() + 2 * dm * span * U
    dr = 0.5 * dv / (var + eps) + 8 * U                   # relative; the first term is far below 1 here
    assert n < 1 << 24 and dr.max() < 0.05
    assert ((mean.double() - wmean).abs() <= dm).all()
    assert ((rstd.double() - wrstd).abs() <= wrstd * dr * (1 + 2 * dr)).all()
    g = torch.ones(c, device="cuda", dtype=torch.float64) if gamma is None else gamma.double()
    b = torch.zeros(c, device="cuda", dtype=torch.float64) if beta is None else beta.double()
    xh = d * wide(wrstd, c)
    z = xh * g + b
    ez = g.abs() * (wide(wrstd * dm, c) + xh.abs() * (wide(dr * (1 + 2 * dr), c) + 4 * U)) + 2 * U * (z.abs() + b.abs())
    want = act64(z, act)
    # the slope of z sigmoid(z) is below 1.1; the sigmoid itself: the exponent's argument off by |z| u, an exponential and a reciprocal of a few steps
    bound = 1.1 * ez + ((z.abs() + 16) * U * want.abs() if act == "silu" else 0)
    T = torch.finfo(x.dtype).eps / 2
    over = (y.double() - want).abs() - (bound * (1 + T) + T * want.abs() + 1e-37)
    assert over.max() <= 0, f"off by {over.max():.3e} more than the bound"
    return y, mean, rstd


SHAPES = [(1, 1, 1, 1), (2, 1, 8, 8), (1, 3, 8, 1), (2, 5, 12, 4), (3, 49, 64, 32), (2, 100, 96, 32), (1, 49, 2048, 32), (4, 729, 260, 20), (2, 3025, 96, 32), (2, 200, 4096, 1),
          (1, 7, 16384, 2), (1, 33, 4098, 2), (5, 3, 257, 1), (3, 1000, 40, 5), (64, 2, 32, 4), (1, 20000, 16, 4), (2, 64, 24, 1), (40, 196, 64, 8), (1, 2500, 512, 32), (7, 31, 7, 7),
          (2, 900, 128, 32), (1, 16, 1032, 3), (3, 257, 48, 2), (1000, 1, 16, 2), (1, 1, 16384, 1), (2, 50, 640, 5), (70000, 1, 8, 2), (66000, 3, 6, 3), (2, 6000, 250, 5), (1, 17000, 32, 32), (2, 3000, 672, 32), (1, 3000, 130, 1),
          (3, 400, 66, 11), (2, 12000, 64, 32), (1, 30000, 64, 8), (4, 90, 96, 96)]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("maps,pixels,c,groups", SHAPES)
def test_norm(maps, pixels, c, groups, dtype):
    gamma, beta = weights(c, pixels + c)
    act = list(ACTS)[(maps + pixels + c) % 3]
    check_norm(make(maps, pixels, c, TYPES[dtype], pixels * 7 + c), groups, gamma, beta, act)


@gpu
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gamma,beta", [(True, True), (True, False), (False, True), (False, False)])
def test_norm_with_and_without_weights(gamma, beta, dtype, act):
    g, b = weights(96, 1)
    check_norm(make(3, 70, 96, TYPES[dtype], 2), 16, g if gamma else None, b if beta else None, act)


STRIDED = [(64, 64, 1), (64, 80, 0), (64, 72, 3), (64, 65, 0), (256, 264, 8), (96, 104, 4)]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c,pitch,offset", STRIDED)
def test_norm_of_strided_and_shifted_rows(c, pitch, offset, dtype):
    x, _ = spread(make(2, 30, c, TYPES[dtype], 9), pitch, offset)
    y, buf = spread(torch.zeros(2, 30, c, dtype=TYPES[dtype], device="cuda"), pitch, offset)
    gamma = torch.randn(c + 1, generator=gen(5), device="cuda")[1:]        # not 16-byte aligned either
    check_norm(x, 8, gamma, None, "silu", y=y)
    assert untouched(buf, pitch, offset, c, 60), "something beside the rows was written"


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("maps,pixels,c,groups", [(2, 64, 64, 8), (1, 3000, 48, 16), (3, 700, 260, 20)])
def test_norm_in_place(maps, pixels, c, groups, dtype):
    gamma, beta = weights(c, 3)
    x = make(maps, pixels, c, TYPES[dtype], 4)
    want = torch.empty_like(x)
    B.dc_group_norm(x, groups, gamma, beta, want, None, None, ACTS["relu"], EPS, scratch(maps, pixels, c, groups))
    B.dc_group_norm(x, groups, gamma, beta, x, None, None, ACTS["relu"], EPS, scratch(maps, pixels, c, groups))
    assert torch.equal(x, want)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_a_large_mean(dtype):
    """Values around 1000 whose spread is 1 (bfloat16: steps of 4 there, so a spread of 40): nothing is lost in a sum of squares."""
    s = 1.0 if dtype == "f32" else 40.0
    x = (1000.0 + s * torch.randn(2, 500, 64, generator=gen(11), device="cuda")).to(TYPES[dtype])
    check_norm(x, 8, None, None)


@gpu
@pytest.mark.parametrize("pixels", [1, 30, 5000])
def test_norm_of_equal_values(pixels):
    x = torch.full((2, pixels, 32), 3.5, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(2, 4, device="cuda"), torch.empty(2, 4, device="cuda")
    B.dc_group_norm(x, 4, None, None, y, mean, rstd, ACTS["none"], EPS, scratch(2, pixels, 32, 4))
    assert (y == 0).all() and (mean == 3.5).all() and ((rstd.double() - EPS ** -0.5).abs() <= 8 * U * EPS ** -0.5).all()


@gpu
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("pixels,c", [(40, 64), (4000, 64), (40, 63), (900, 24)])
def test_a_nan_stays_in_its_group(pixels, c, bad, act):
    groups = 8 if c % 8 == 0 else 9
    per = c // groups
    x = make(3, pixels, c, torch.float32, 12)
    clean, y = torch.empty_like(x), torch.empty_like(x)
    work = scratch(3, pixels, c, groups)
    B.dc_group_norm(x, groups, None, None, clean, None, None, ACTS[act], EPS, work)
    x[1, pixels // 2, 2 * per] = bad
    B.dc_group_norm(x, groups, None, None, y, None, None, ACTS[act], EPS, work)
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[1, :, 2 * per:3 * per] = True
    assert torch.isnan(y[hit]).all() and torch.equal(y[~hit], clean[~hit])


@gpu
def test_maps_of_more_dimensions_and_none():
    x = make(2, 6 * 5, 32, torch.float32, 1)
    a, b = torch.empty_like(x), torch.empty(2, 6, 5, 32, device="cuda")
    work = scratch(2, 30, 32, 4)
    B.dc_group_norm(x, 4, None, None, a, workspace=work)
    B.dc_group_norm(x.view(2, 6, 5, 32), 4, None, None, b, workspace=work)
    assert torch.equal(a.view_as(b), b)
    none = torch.empty(0, 9, 32, device="cuda")
    B.dc_group_norm(none, 4, None, None, none)
    dg, db = torch.full((32,), 5.0, device="cuda"), torch.full((32,), 5.0, device="cuda")
    B.dc_group_norm_backward(none, none, 4, None, None, torch.empty(0, 4, device="cuda"), torch.empty(0, 4, device="cuda"), None, dg, db)
    assert (dg == 0).all() and (db == 0).all()


# ---------------------------------------------------------------------------
# maps with a value far from all others
# ---------------------------------------------------------------------------
def check_statistics(x, groups):
    """Mean and rstd, off by what float32 sums of positive numbers are off by, whatever the values are.

    Distances are taken from some value c, and so that the mean is no farther from c than 2 sigma of the rows that are added up together, or from the mean itself: of Q, the squares
    of distances, at most 4/5 are taken off as the mean's.  Q is off by DEPTH u of itself, a sum of N distances by DEPTH u sqrt(N Q), so what is left, M >= Q/5, by
    DEPTH u (1 + 2 sqrt(4/5)) Q <= 14 DEPTH u M.  Where parts are joined, their means are off by DEPTH u sqrt(Q_i / N_i) and two roundings, which moves M by
    2 DEPTH u sqrt(5) M + 4 u sqrt(M N (var + mean^2)) at most.  Some roundings of sums that are there already: 16 u."""
    maps, pixels, c = x.shape
    v = split(x, groups)
    wmean = v.mean((1, 3))
    var = (v - wmean[:, None, :, None]).square().mean((1, 3))
    wrstd = (var + EPS).rsqrt()
    y, mean, rstd = torch.empty(maps, pixels, c, dtype=x.dtype, device="cuda"), torch.empty(maps, groups, device="cuda"), torch.empty(maps, groups, device="cuda")
    B.dc_group_norm(x, groups, None, None, y, mean, rstd, ACTS["none"], EPS, scratch(maps, pixels, c, groups))
    root = (var + wmean.square()).sqrt()
    dm = DEPTH * U * (5 * var).sqrt() + 16 * U * root
    dv = ((14 + 2 * 5 ** 0.5) * DEPTH + 16) * U + 4 * U * root / var.sqrt()
    dr = 0.5 * dv * (1 + 2 * dv) + 8 * U
    assert dv.max() < 4e-4, "the bound says nothing"
    assert ((mean.double() - wmean).abs() <= dm).all()
    off = ((rstd.double() - wrstd).abs() / wrstd - dr).max()
    assert off <= 0, f"rstd off by {off:.3e} of itself more than the bound"
    z = (x.double() - wide(wmean, c)) * wide(wrstd, c)
    T = torch.finfo(x.dtype).eps / 2
    over = (y.double() - z).abs() - ((wide(wrstd * dm, c) + z.abs() * (wide(dr, c) + 4 * U) + 2 * U * z.abs()) * (1 + T) + T * z.abs())
    assert over.max() <= 0, f"off by {over.max():.3e} more than the bound"


# one launch and two, whole vectors to a group and not, rows of two elements and of one, groups wider than a CTA
FAR = [(1, 3136, 64, 8), (4, 3136, 256, 32), (3, 900, 24, 8), (2, 3025, 96, 32), (1, 20000, 16, 4), (1, 30000, 64, 8), (2, 700, 4096, 2), (2, 4000, 66, 11), (2, 4000, 33, 3), (2, 6000, 250, 5),
       (40, 196, 64, 8)]


@gpu
@pytest.mark.parametrize("where", ["first", "any", "row", "channel"])
@pytest.mark.parametrize("far", [30.0, 1e3, 3e4])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("maps,pixels,c,groups", FAR)
def test_norm_with_values_far_from_the_rest(maps, pixels, c, groups, dtype, far, where):
    """A group's first value, any one, its first row or its first channel `far` standard deviations away."""
    g = gen(pixels + c)
    x = torch.randn(maps, pixels, c, generator=g, device="cuda")
    v = x.view(maps, pixels, groups, c // groups)
    if where == "first":
        v[:, 0, :, 0] += far
    elif where == "any":
        at = torch.randint(0, pixels, (maps,), generator=g, device="cuda")
        v[torch.arange(maps, device="cuda"), at, :, (c // groups) // 2] -= far
    elif where == "row":
        v[:, 0] += far
    else:
        v[..., 0] += far
    check_statistics(x.to(TYPES[dtype]), groups)


# ---------------------------------------------------------------------------
# gradients
# ---------------------------------------------------------------------------
def gradients64(dy, x, groups, gamma, beta, mean, rstd, act):
    """(dx, dgamma, dbeta) and bounds of their errors before rounding to the map's type"""
    maps, pixels, c = x.shape
    g = torch.ones(c, device="cuda", dtype=torch.float64) if gamma is None else gamma.double()
    b = torch.zeros(c, device="cuda", dtype=torch.float64) if beta is None else beta.double()
    r, dy = wide(rstd.double(), c), dy.double()
    xh = (x.double() - wide(mean.double(), c)) * r        # off by two roundings
    z = xh * g + b
    ez = 4 * U * ((xh * g).abs() + b.abs())
    dz = dy * slope64(z, act)
    # the slope's own slope is below 0.5; its factors as above; ReLU: either side where z cannot be told from zero
    ed = {"none": 0 * dz, "relu": dy.abs() * (z.abs() <= ez), "silu": dy.abs() * (0.5 * ez + (z.abs() + 16) * U * (1 + z.abs()))}[act]
    gz, eg = dz * g, ed * g.abs() + 2 * U * (dz * g).abs()
    of = lambda t: wide(t.reshape(maps, pixels, groups, c // groups).mean((1, 3)), c)
    m1, m2 = of(gz), of(gz * xh)
    e1 = of(eg) + (DEPTH + 4) * U * of(gz.abs())
    e2 = of(eg * xh.abs()) + (DEPTH + 8) * U * of((gz * xh).abs())
    dx = r * (gz - m1 - xh * m2)
    ex = r * (eg + e1 + xh.abs() * e2 + 8 * U * (gz.abs() + m1.abs() + (xh * m2).abs()))
    sums = lambda t: t.sum((0, 1))
    return (dx, sums(dz * xh), sums(dz)), (ex, sums(ed * xh.abs()) + (DEPTH + 8) * U * sums((dz * xh).abs()), sums(ed) + (DEPTH + 4) * U * sums(dz.abs()))


def check_backward(dy, x, groups, gamma, beta, act, dx=None):
    maps, pixels, c = x.shape
    v = split(x, groups)
    m64 = v.mean((1, 3))
    mean, rstd = m64.float(), ((v - m64[:, None, :, None]).square().mean((1, 3)) + EPS).rsqrt().float()
    (wx, wg, wb), (ex, eg, eb) = gradients64(dy, x, groups, gamma, beta, mean, rstd, act)
    dx = torch.empty(maps, pixels, c, dtype=x.dtype, device="cuda") if dx is None else dx
    dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    B.dc_group_norm_backward(dy, x, groups, gamma, beta, mean, rstd, dx, dg, db, ACTS[act], scratch(maps, pixels, c, groups))
    T = torch.finfo(x.dtype).eps / 2
    over = (dx.double() - wx).abs() - (ex * (1 + T) + T * wx.abs() + 1e-37)
    assert over.max() <= 0, f"dx off by {over.max():.3e} more than the bound"
    assert ((dg.double() - wg).abs() <= eg + 2 * U * wg.abs()).all() and ((db.double() - wb).abs() <= eb + 2 * U * wb.abs()).all()
    return dx, dg, db, mean, rstd


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("maps,pixels,c,groups", SHAPES)
def test_backward(maps, pixels, c, groups, dtype):
    gamma, beta = weights(c, pixels + c)
    act = list(ACTS)[(maps + pixels + c + 1) % 3]
    check_backward(make(maps, pixels, c, TYPES[dtype], 3, 0.1), make(maps, pixels, c, TYPES[dtype], pixels * 7 + c), groups, gamma, beta, act)


@gpu
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gamma,beta", [(True, True), (True, False), (False, True), (False, False)])
def test_backward_with_and_without_weights(gamma, beta, dtype, act):
    g, b = weights(96, 1)
    check_backward(make(3, 70, 96, TYPES[dtype], 5, 0.0), make(3, 70, 96, TYPES[dtype], 2), 16, g if gamma else None, b if beta else None, act)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c,pitch,offset", STRIDED)
def test_backward_of_strided_and_shifted_rows(c, pitch, offset, dtype):
    x, _ = spread(make(2, 30, c, TYPES[dtype], 9), pitch, offset)
    dy, _ = spread(make(2, 30, c, TYPES[dtype], 8), pitch, offset)
    dx, buf = spread(torch.zeros(2, 30, c, dtype=TYPES[dtype], device="cuda"), pitch, offset)
    gamma = torch.randn(c + 1, generator=gen(5), device="cuda")[1:]
    check_backward(dy, x, 8, gamma, None, "silu", dx=dx)
    assert untouched(buf, pitch, offset, c, 60), "something beside the rows was written"


@gpu
@pytest.mark.parametrize("maps,pixels,c,groups", [(2, 64, 64, 8), (1, 3000, 48, 16), (3, 700, 260, 20)])
def test_backward_in_place_of_either_and_of_parts(maps, pixels, c, groups):
    gamma, beta = weights(c, 3)
    x, dy = make(maps, pixels, c, torch.bfloat16, 4), make(maps, pixels, c, torch.bfloat16, 6, 0.0)
    dx, dg, db, mean, rstd = check_backward(dy, x, groups, gamma, beta, "silu")
    work = scratch(maps, pixels, c, groups)
    call = lambda a, b, *out: B.dc_group_norm_backward(a, b, groups, gamma, beta, mean, rstd, *out, ACTS["silu"], work)
    a, b = dy.clone(), x.clone()
    call(a, x, a, None, None)
    call(dy, b, b, None, None)
    assert torch.equal(a, dx) and torch.equal(b, dx)
    g, t = torch.full_like(dg, 9), torch.full_like(db, 9)
    call(dy, x, None, g, None)
    call(dy, x, None, None, t)
    assert torch.equal(g, dg) and torch.equal(t, db)
    call(dy, x, None, None, None)


@gpu
@pytest.mark.parametrize("act", list(ACTS))
def test_backward_against_differences(act):
    """The gradients against differences of the 64-bit forward pass along random directions: second-order differences are off by h^2 times a third derivative, far below the tolerance
    of 1e-4 with h = 1e-4 (values and derivatives are of order one; ReLU: no z within 1e-3 of its bend moves across it)."""
    g = gen(21)
    x, dy = torch.randn(2, 6, 12, generator=g, device="cuda"), torch.randn(2, 6, 12, generator=g, device="cuda")
    gamma, beta = weights(12, 2)

    def loss(x, gamma, beta):
        v = x.view(2, 6, 4, 3)
        d = v - v.mean((1, 3), keepdim=True)
        z = (d * (d.square().mean((1, 3), keepdim=True) + EPS).rsqrt()).view(2, 6, 12) * gamma + beta
        return (act64(z, act) * dy.double()).sum(), z

    if act == "relu":
        near = loss(x.double(), gamma.double(), beta.double())[1].abs() < 2e-3
        dy[near] = 0
    y, mean, rstd = torch.empty_like(x), torch.empty(2, 4, device="cuda"), torch.empty(2, 4, device="cuda")
    work = scratch(2, 6, 12, 4)
    B.dc_group_norm(x, 4, gamma, beta, y, mean, rstd, ACTS[act], EPS, work)
    dx, dg, db = torch.empty_like(x), torch.empty(12, device="cuda"), torch.empty(12, device="cuda")
    B.dc_group_norm_backward(dy, x, 4, gamma, beta, mean, rstd, dx, dg, db, ACTS[act], work)
    h = 1e-4
    for k in range(6):
        v, w, t = torch.randn(2, 6, 12, generator=g, device="cuda").double(), torch.randn(12, generator=g, device="cuda").double(), torch.randn(12, generator=g, device="cuda").double()
        up = loss(x.double() + h * v, gamma.double() + h * w, beta.double() + h * t)[0]
        down = loss(x.double() - h * v, gamma.double() - h * w, beta.double() - h * t)[0]
        got = (dx.double() * v).sum() + (dg.double() * w).sum() + (db.double() * t).sum()
        size = (dx.double() * v).abs().sum() + (dg.double() * w).abs().sum() + (db.double() * t).abs().sum()
        assert abs((up - down) / (2 * h) - got) <= 1e-4 * size


@gpu
def test_relu_backward_keeps_what_the_forward_pass_kept():
    x, dy = make(2, 4000, 64, torch.float32, 31), torch.ones(2, 4000, 64, device="cuda")
    gamma, beta = weights(64, 32)
    y, mean, rstd = torch.empty_like(x), torch.empty(2, 8, device="cuda"), torch.empty(2, 8, device="cuda")
    work = scratch(2, 4000, 64, 8)
    B.dc_group_norm(x, 8, gamma, beta, y, mean, rstd, ACTS["relu"], EPS, work)
    db = torch.empty(64, device="cuda")
    B.dc_group_norm_backward(dy, x, 8, gamma, beta, mean, rstd, None, None, db, ACTS["relu"], work)
    assert torch.equal(db, (y > 0).sum((0, 1)).float())      # sums of ones: exact


@gpu
@pytest.mark.parametrize("shift", [0, 1, 100, 255])
@pytest.mark.parametrize("maps,pixels,c,groups", [(3, 196, 64, 8), (2, 30000, 64, 8), (1, 20000, 16, 4), (2, 50, 4096, 2)])
def test_a_workspace_of_any_alignment(maps, pixels, c, groups, shift):
    """As many bytes as asked for, from any one on: the same bits, and nothing beside them is written."""
    x, dy = make(maps, pixels, c, torch.bfloat16, 4), make(maps, pixels, c, torch.bfloat16, 6, 0.0)
    gamma, beta = weights(c, 3)
    need = B.dc_group_norm_workspace(maps, pixels, c, groups)

    def both(work):
        y, dx, numbers = torch.empty_like(x), torch.empty_like(x), torch.empty(2, maps, groups, device="cuda")
        gradients = torch.empty(2, c, device="cuda")
        B.dc_group_norm(x, groups, gamma, beta, y, *numbers, ACTS["silu"], EPS, work)
        B.dc_group_norm_backward(dy, x, groups, gamma, beta, *numbers, dx, *gradients, ACTS["silu"], work)
        return y, numbers, dx, gradients

    want = both(scratch(maps, pixels, c, groups))
    room = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    at = -room.data_ptr() % 256 + shift
    assert all(torch.equal(a, b) for a, b in zip(want, both(room[at:at + need])))
    assert (room[:at] == 0x5A).all() and (room[at + need:] == 0x5A).all()


# ---------------------------------------------------------------------------
# streams, graphs, refusals
# ---------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("maps,pixels,c,groups", [(2, 600, 64, 8), (1, 1200, 40, 8), (4, 300, 33, 3), (2, 700, 4096, 2)])
def test_rows_behind_four_gigabytes(maps, pixels, c, groups, dtype):
    t, pitch = TYPES[dtype], 1 << 21
    def far():
        m = torch.empty(maps * pixels * pitch, dtype=t, device="cuda").view(maps, pixels, pitch)[:, :, :c]
        assert (maps * pixels - 1) * pitch * m.element_size() > 1 << 32
        return m
    gamma, beta = weights(c, 3)
    x, dy = make(maps, pixels, c, t, 4), make(maps, pixels, c, t, 5)
    y, dx, numbers = torch.empty_like(x), torch.empty_like(x), [torch.empty(2, maps, groups, device="cuda") for _ in range(2)]
    gradients = [torch.empty(2, c, device="cuda") for _ in range(2)]
    work = scratch(maps, pixels, c, groups)
    B.dc_group_norm(x, groups, gamma, beta, y, *numbers[0], ACTS["silu"], EPS, work)
    B.dc_group_norm_backward(dy, x, groups, gamma, beta, *numbers[0], dx, *gradients[0], ACTS["silu"], work)
    far_x, far_dy, far_y, far_dx = far(), far(), far(), far()
    far_x.copy_(x), far_dy.copy_(dy)
    B.dc_group_norm(far_x, groups, gamma, beta, far_y, *numbers[1], ACTS["silu"], EPS, work)
    B.dc_group_norm_backward(far_dy, far_x, groups, gamma, beta, *numbers[1], far_dx, *gradients[1], ACTS["silu"], work)
    # (rows of 33 elements lie on fewer bytes than those 2^21 apart: sums in another order there)
    if c % 8 == 0:
        assert torch.equal(far_y, y) and torch.equal(far_dx, dx) and torch.equal(numbers[0], numbers[1]) and torch.equal(gradients[0], gradients[1])
    else:
        check_norm(far_x, groups, gamma, beta, "silu")
        check_backward(far_dy, far_x, groups, gamma, beta, "silu")


@gpu
def test_equal_calls_give_equal_bits_on_streams_and_in_graphs():
    maps, pixels, c, groups = 4, 900, 96, 32
    gamma, beta = weights(c, 3)
    xs = [make(maps, pixels, c, torch.bfloat16, s) for s in (1, 2)]
    dy = make(maps, pixels, c, torch.bfloat16, 3, 0.0)

    def outputs():
        return dict(y=torch.empty_like(dy), mean=torch.empty(maps, groups, device="cuda"), rstd=torch.empty(maps, groups, device="cuda"), dx=torch.empty_like(dy),
                    dg=torch.empty(c, device="cuda"), db=torch.empty(c, device="cuda"), work=scratch(maps, pixels, c, groups))

    def both(x, o):
        B.dc_group_norm(x, groups, gamma, beta, o["y"], o["mean"], o["rstd"], ACTS["silu"], EPS, o["work"])
        B.dc_group_norm_backward(dy, x, groups, gamma, beta, o["mean"], o["rstd"], o["dx"], o["dg"], o["db"], ACTS["silu"], o["work"])

    want = [outputs() for _ in xs]
    for x, o in zip(xs, want):
        both(x, o)
    torch.cuda.synchronize()
    # two streams at once, each with a workspace of its own
    got, streams = [outputs() for _ in xs], [torch.cuda.Stream() for _ in xs]
    for _ in range(3):
        for x, o, s in zip(xs, got, streams):
            with torch.cuda.stream(s):
                both(x, o)
    torch.cuda.synchronize()
    names = ("y", "mean", "rstd", "dx", "dg", "db")
    assert all(torch.equal(a[k], b[k]) for a, b in zip(want, got) for k in names)
    # captured, and replayed on other values
    o, x = outputs(), xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(x, o)
    x.copy_(xs[1])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(want[1][k], o[k]) for k in names)


def test_refusals_of_the_c_abi():
    lib = B.load()
    buf = (C.c_char * 4096)()
    at = (C.addressof(buf) + 255) & ~255
    n = C.c_size_t()
    assert lib.dc_group_norm_workspace(1, 1, 8, 2, None) == B.DC_ERR_ARG
    assert lib.dc_group_norm_workspace(1, 1, 8, 3, C.byref(n)) == B.DC_ERR_ARG
    assert lib.dc_group_norm_workspace(1, 1, 16392, 1, C.byref(n)) == B.DC_ERR_LIMIT
    assert lib.dc_group_norm_workspace(1 << 20, 1 << 20, 8, 1, C.byref(n)) == B.DC_ERR_LIMIT
    assert lib.dc_group_norm_workspace(2, 9, 8, 2, C.byref(n)) == B.DC_OK and n.value > 0
    room = n.value

    def norm(x=at, x_pitch=32, gamma=None, beta=None, maps=2, pixels=9, c=8, groups=2, eps=1e-5, act=0, dtype=B.DC_FP32, y=at, y_pitch=32, mean=None, rstd=None, work=at, bytes_=room):
        return lib.dc_group_norm(x, x_pitch, gamma, beta, maps, pixels, c, groups, eps, act, dtype, y, y_pitch, mean, rstd, work, bytes_, None)

    def back(dy=at, dy_pitch=32, x=at, x_pitch=32, gamma=None, beta=None, mean=at, rstd=at, maps=2, pixels=9, c=8, groups=2, act=0, dtype=B.DC_FP32, dx=at, dx_pitch=32, dg=at, db=at,
             work=at, bytes_=room):
        return lib.dc_group_norm_backward(dy, dy_pitch, x, x_pitch, gamma, beta, mean, rstd, maps, pixels, c, groups, act, dtype, dx, dx_pitch, dg, db, work, bytes_, None)

    for call in (norm, back):
        assert call(dtype=2) == B.DC_ERR_CONFIG and call(act=3) == B.DC_ERR_CONFIG and call(act=-1) == B.DC_ERR_CONFIG
        assert call(groups=3) == B.DC_ERR_ARG and call(groups=0) == B.DC_ERR_ARG and call(c=0) == B.DC_ERR_ARG
        assert call(maps=-1) == B.DC_ERR_ARG and call(pixels=-1) == B.DC_ERR_ARG
        assert call(x=None) == B.DC_ERR_ARG and call(x=at + 2) == B.DC_ERR_ARG and call(x_pitch=28) == B.DC_ERR_ARG and call(x_pitch=34) == B.DC_ERR_ARG
        assert call(x_pitch=1 << 32) == B.DC_ERR_LIMIT and call(pixels=1 << 31) == B.DC_ERR_LIMIT and call(c=16400) == B.DC_ERR_LIMIT
        assert call(work=None) == B.DC_ERR_ARG and call(bytes_=room - 1) == B.DC_ERR_ARG
        assert call(gamma=at + 1) == B.DC_ERR_ARG and call(beta=at + 2) == B.DC_ERR_ARG and call(mean=at + 2) == B.DC_ERR_ARG and call(rstd=at + 1) == B.DC_ERR_ARG
    assert norm(y=None) == B.DC_ERR_ARG and norm(y_pitch=16) == B.DC_ERR_ARG and norm(eps=-1.0) == B.DC_ERR_ARG and norm(eps=float("nan")) == B.DC_ERR_ARG
    assert norm(maps=0) == B.DC_OK and norm(pixels=0, x=None, y=None, work=None, bytes_=0) == B.DC_OK
    assert back(dy=None) == B.DC_ERR_ARG and back(mean=None) == B.DC_ERR_ARG and back(dx=at + 1) == B.DC_ERR_ARG and back(dg=at + 1) == B.DC_ERR_ARG
    assert back(dx=None, dg=None, db=None) == B.DC_OK


@gpu
def test_refusals_of_tensors():
    x = torch.zeros(2, 9, 8, device="cuda")
    work = scratch(2, 9, 8, 2)
    y = torch.empty_like(x)
    for bad in [dict(x=x.cpu()), dict(x=x.half()), dict(y=torch.empty(2, 9, 7, device="cuda")), dict(y=y.bfloat16()), dict(x=x.transpose(1, 2)), dict(x=torch.zeros(2, 18, 8, device="cuda")[:, :9]),
                dict(gamma=torch.zeros(7, device="cuda")), dict(mean=torch.zeros(3, device="cuda")), dict(work=work[::2])]:
        a = dict(x=x, y=y, gamma=None, mean=None, work=work)
        a.update(bad)
        with pytest.raises((TypeError, ValueError)):
            B.dc_group_norm(a["x"], 2, a["gamma"], None, a["y"], a["mean"], None, 0, EPS, a["work"])
    for bad in (dict(groups=3), dict(work=None), dict(work=work[:16]), dict(activation=7)):
        a = dict(groups=2, work=work, activation=0)
        a.update(bad)
        with pytest.raises(B.DeepCacheError):
            B.dc_group_norm(x, a["groups"], None, None, y, None, None, a["activation"], EPS, a["work"])
