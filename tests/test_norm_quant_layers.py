"""Layer normalisation and 8-bit convolutions as layers of a cache: the oracle's pins, and the CUDA path layer by layer.

A stored map that differs in its last bit may turn a value next to a half to the other step, so each layer is checked from the very map that
the library has stored for its input: then every step, and every sum, is known exactly, and what is left are the float32 roundings
behind the sum and the rounding to the map's type.
"""
import ctypes

import numpy as np
import pytest
import torch
import torch.nn.functional as F

import parity_util as P
from oracle import deepcache_oracle as orc
from paper_1712_01670_b200 import binding as B
from paper_1712_01670_b200.engine import DeepCache
from paper_1712_01670_b200.synth import configs, nets

gpu = pytest.mark.gpu
U = 2.0 ** -24


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


# ---------------------------------------------------------------------------
# the oracle (CPU)
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("c", [1, 5, 64])
def test_oracle_layer_norm_equals_torch_float64(c):
    g = rng(c)
    x, gamma, beta = g.normal(2.0, 3.0, size=(6, 7, c)), g.normal(size=c), g.normal(size=c)
    want = F.layer_norm(torch.from_numpy(x), (c,), torch.from_numpy(gamma), torch.from_numpy(beta), 1e-5).numpy()
    assert np.abs(orc.layer_norm(x, gamma, beta, 1e-5, orc.QUANT_NONE) - want).max() < 1e-12
    want = F.layer_norm(torch.from_numpy(x), (c,), None, None, 0.3).numpy()
    assert np.abs(orc.layer_norm(x, None, None, 0.3, orc.QUANT_NONE) - want).max() < 1e-12


def test_oracle_rows_in_8_bits():
    q, s = orc.quantise_rows(np.array([[127.0, 0.5, 1.5, -2.5, -126.5], [0, 0, 0, 0, 0], [-2, 1, 0, 0, 0]]))
    assert q.tolist() == [[127, 0, 2, -2, -126], [0] * 5, [-127, 64, 0, 0, 0]]
    assert s.tolist() == [1.0, 0.0, float(np.float32(2 / 127))]


def test_oracle_8_bit_convolution_is_near_the_convolution_and_exact_on_its_own_steps():
    g = rng(3)
    x, w, b = g.normal(size=(5, 6, 48)), g.normal(size=(24, 1, 1, 48)).astype(np.float32), g.normal(size=24)
    L = dict(kind=orc.KIND_CONV_QUANT, kh=1, kw=1, sh=1, sw=1, ph=0, pw=0, cin=48, cout=24, relu=0, in0=-1, in1=-1, out_h=5, out_w=6)
    out, reused = orc.conv_quant(x, L, w, b, orc.QUANT_NONE)
    exact = x @ w.reshape(24, 48).T.astype(np.float64) + b
    # half a step of either side, summed up: |x| half a weight step + |w| half a pixel step, per term
    step_x, step_w = np.abs(x).max(-1) / 254, np.abs(w).reshape(24, 48).max(-1) / 254
    bound = np.abs(x).sum(-1)[..., None] * step_w + np.abs(w).reshape(24, 48).sum(-1) * step_x[..., None] + 48 * step_x[..., None] * step_w
    assert (np.abs(out - exact) <= bound * 1.001).all() and not reused.any()
    xi = g.integers(-127, 128, size=(5, 6, 48)).astype(np.float64)
    xi[..., 0] = 127
    wi = g.integers(-127, 128, size=(24, 1, 1, 48)).astype(np.float32)
    wi[..., 0] = -127
    out, _ = orc.conv_quant(xi, dict(L, relu=1), wi, b, orc.QUANT_NONE)
    assert np.abs(out - np.maximum(xi @ wi.reshape(24, 48).T + b, 0)).max() < 1e-9


def test_region_rules():
    regs = np.zeros(2, orc.REGION_DTYPE)
    regs[0] = (3, 4, 10, 6, 1, 5)
    point = dict(kind=orc.KIND_CONV_QUANT, kh=1, kw=1, sh=1, sw=1, ph=0, pw=0, cin=8, cout=8, relu=0, in0=-1, in1=-1, out_h=20, out_w=30)
    assert (orc.propagate_layer(point, 20, 30, regs) == regs).all()
    assert (orc.propagate_layer(dict(point, kind=orc.KIND_LAYER_NORM), 20, 30, regs) == regs).all()
    whole = dict(point, kh=20, kw=30, out_h=1, out_w=1)
    assert (orc.propagate_layer(whole, 20, 30, regs)["w"] == 0).all()


def test_oracle_reuses_8_bit_pixels():
    """The same frame again: everything in rectangles comes from the cache, so the pointwise layers' outputs are bit-equal."""
    w = configs.small_cnn_stream()
    w.layers = nets.norm_quant_net(64, 64, 16, 1)
    w = P.crop_workload(w, 64, 64)
    o = P.make_oracles(w, 1)[0]
    frame = w.streams(1, 1).frame(0)[0]
    a = o.infer_frame(frame)
    b = o.infer_frame(frame)
    for i, l in enumerate(w.layers):
        assert np.array_equal(a["maps"][i], b["maps"][i])
        if l["kind"] == orc.KIND_CONV_QUANT and l["out_h"] > 1:
            assert b["reused"][i].mean() > 0.5


def refused(l, dtype=0):
    cfg = B.dc_config(width=64, height=64, channels=3, n_streams=1, block=8, range=4, search=1, skip_k=1, expire_n=10, psnr_db=20.0, dtype=dtype, max_regions=0)
    base = dict(kind=0, kh=3, kw=3, sh=1, sw=1, ph=1, pw=1, cin=3, cout=16, relu=1, in0=-1, in1=-1, out_h=64, out_w=64)
    q = dict(kind=B.DC_CONV_QUANT, kh=1, kw=1, sh=1, sw=1, ph=0, pw=0, cin=16, cout=32, relu=1, in0=0, in1=-1, out_h=64, out_w=64)
    q.update(l)
    out = ctypes.c_void_p()
    return B.load().dc_cache_create(ctypes.byref(cfg), B.make_layers([base, q]), 2, None, None, None, ctypes.byref(out))


@pytest.mark.parametrize("l", [dict(cin=8), dict(kh=3, kw=3, ph=1, pw=1), dict(sh=2, sw=2, out_h=32, out_w=32), dict(cout=6), dict(groups=2), dict(out_w=63),
                               dict(kh=64, kw=64, out_h=1, out_w=2), dict(kind=B.DC_LAYER_NORM, cout=17), dict(kind=B.DC_LAYER_NORM, cout=16, out_h=32),
                               dict(kind=10), dict(kh=64, kw=64, out_h=1, out_w=1, cout=10, cin=15)])
def test_layer_tables_that_are_refused(l):
    assert refused(l) == B.DC_ERR_CONFIG
    assert refused(dict(l), dtype=1) == B.DC_ERR_CONFIG


def test_epsilon_needs_a_cache():
    assert B.load().dc_cache_set_norm_epsilon(None, 0, 1e-5) == B.DC_ERR_ARG


# ---------------------------------------------------------------------------
# the CUDA path
# ---------------------------------------------------------------------------
def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rows64(x):
    x = x.double()
    most = x.abs().amax(-1, keepdim=True)
    q = torch.round(127.0 * x / torch.where(most > 0, most, torch.ones_like(most)))
    return q, (most[..., 0] / 127.0).float().double()


def quant_layer64(x, l, w, b):
    """(out, bound) of an 8-bit convolution on the stored map x [S, H, W, C] (torch, on the GPU)."""
    S = x.shape[0]
    rows = x.reshape(S, 1, 1, -1) if l["kh"] > 1 or l["out_h"] * l["out_w"] == 1 else x
    q, s = rows64(rows)
    wq, ws = rows64(torch.as_tensor(w, device="cuda").reshape(l["cout"], -1))
    acc = (q @ wq.t()) * s[..., None] * ws
    out = acc + torch.as_tensor(b, device="cuda").double()
    bound = 4 * U * acc.abs() + U * out.abs()
    return (out.clamp_min(0) if l["relu"] else out), bound


def norm_layer64(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    g = 1.0 if gamma is None else torch.as_tensor(gamma, device="cuda").double()
    b = 0.0 if beta is None else torch.as_tensor(beta, device="cuda").double()
    y = d * rstd * g + b
    dm = 82 * U * x.abs().mean(-1, keepdim=True)          # as in test_operators.norm64
    g, b = torch.as_tensor(g).abs(), torch.as_tensor(b).abs()
    return y, g * rstd * (dm * (1 + (d * rstd).abs() * dm * rstd) + d.abs() * 48 * U) + 2 * U * (y.abs() + b)


def assert_near(got, want, bound, what):
    T = half_step(got.dtype)
    over = (got.double() - want).abs() - (bound * (1 + T) + T * want.abs() + 1e-38)
    assert float(over.max()) <= 0, f"{what}: off by {float(over.max()):.3e} more than the bound"


def frames_of(h, w, n, S, seed):
    """A textured stream that moves by whole pixels, with a block drawn anew every frame."""
    g = rng(seed)
    big = np.kron(g.integers(0, 256, size=(S, h // 4 + 24, w // 4 + 24, 3)), np.ones((1, 4, 4, 1))).astype(np.uint8)
    out = []
    for t in range(n):
        f = big[:, 2 * t:2 * t + h, 3 * t:3 * t + w].copy()
        f[:, 5:17, 9:25] = g.integers(0, 256, size=(S, 12, 16, 3))
        out.append(f)
    return out


def check_frames(layers, h, w, S, dtype, frames, announce=False, host=False, **kw):
    weights, biases = nets.random_weights(layers, 5)
    dc = DeepCache(w, h, layers, weights, biases, n_streams=S, block=8, search_range=8, dtype=dtype, expire_n=4, **kw)
    prev, reused_any = {}, 0
    try:
        for t, f in enumerate(frames):
            f = torch.as_tensor(f).cuda()
            out, stats = dc.infer_frame(f, want_stats=True)
            if announce and t + 1 < len(frames):
                nxt = torch.as_tensor(frames[t + 1]).cuda()
                B.dc_lookahead_frame(dc.handle, nxt, w * 3)
                frames[t + 1] = nxt
            maps = [dc.layer_map(i) for i in range(len(layers))]
            maps.append((f.double() / 255).to(maps[0].dtype))            # [-1]: the frame as a map
            assert torch.equal(out, maps[-2])
            for i, l in enumerate(layers):
                what = f"frame {t} layer {i}"
                if l["kind"] == nets.KIND_LAYER_NORM:
                    x = maps[l["in0"]]
                    want, bound = norm_layer64(x, weights[i], biases[i], 1e-5)
                    assert_near(maps[i], want, bound, what)
                elif l["kind"] == nets.KIND_CONV_QUANT:
                    want, bound = quant_layer64(maps[l["in0"]], l, weights[i], biases[i])
                    fresh = torch.ones(S, l["out_h"], l["out_w"], dtype=torch.bool, device="cuda")
                    if not stats[0].refreshed and l["out_h"] > 1:
                        regs, n = dc.layer_regions(i)
                        for s in range(S):
                            for r in regs[s, :int(n[s])].cpu().tolist():
                                x0, y0, rw, rh, sx, sy = r
                                if rw > 0:
                                    assert torch.equal(maps[i][s, y0:y0 + rh, x0:x0 + rw], prev[i][s, sy:sy + rh, sx:sx + rw]), what
                                    fresh[s, y0:y0 + rh, x0:x0 + rw] = False
                            share = 1 - float(fresh[s].double().mean())
                            assert abs(stats[s].reuse_ratio[i] - share) < 1e-6
                            reused_any += share > 0
                    else:
                        assert all(stats[s].reuse_ratio[i] == 0 for s in range(S))
                    assert_near(maps[i][fresh], want[fresh], bound[fresh], what)
            prev = dict(enumerate(maps))
            assert dc.status() == B.DC_OK
        if len(frames) > 1:
            assert reused_any, "no pixel was reused: the test's frames do not match"
    finally:
        dc.close()


@gpu
@pytest.mark.parametrize("dtype", [B.DC_FP32, B.DC_BF16])
@pytest.mark.parametrize("h,w,S,width", [(64, 64, 1, 32), (56, 72, 3, 16), (60, 76, 2, 32), (40, 44, 5, 64)])
def test_frames(h, w, S, width, dtype):
    """Maps of widths that are multiples of 8 and ones that are not, full frames and cached ones, several streams."""
    layers = nets.norm_quant_net(h, w, width, 2)
    check_frames(layers, h, w, S, dtype, frames_of(h, w, 6, S, h + w))


@gpu
def test_frames_announced():
    layers = nets.norm_quant_net(64, 80, 32, 1)
    check_frames(layers, 64, 80, 2, B.DC_BF16, frames_of(64, 80, 5, 2, 1), announce=True)


@gpu
@pytest.mark.parametrize("dtype", [B.DC_FP32, B.DC_BF16])
def test_layers_that_read_the_frame_and_each_other(dtype):
    """A normalisation with two readers, an 8-bit convolution of three channels, one behind another, and on the resized frame."""
    b = nets.NetBuilder(52, 60)
    n = b.layer_norm(-1)
    a = b.conv_quant(n, 24)
    c = b.conv_quant(n, 24, relu=0)
    d = b.conv_quant(-1, 24)
    x = b.add(b.add(a, c), d)
    x = b.conv_quant(x, 40)
    x = b.layer_norm(x)
    x = b.conv_quant(x, 16, whole=True)
    x = b.conv_quant(x, 24)                                        # a map of one pixel
    b.layer_norm(x)
    check_frames(b.layers, 52, 60, 2, dtype, frames_of(52, 60, 4, 2, 3))


@gpu
@pytest.mark.parametrize("dtype", [B.DC_FP32, B.DC_BF16])
def test_layers_that_read_the_resized_frame(dtype):
    """A normalisation and an 8-bit convolution that read the frame behind an area resize, with an ordinary convolution beside them."""
    b = nets.NetBuilder(80, 96)
    r = b.resize_area(-1, 40, 48)
    n = b.layer_norm(r)
    x = b.add(b.conv_quant(n, 24), b.conv_quant(r, 24, relu=0))
    x = b.add(x, b.conv(r, 24, 3, 1, 1))
    b.conv_quant(b.layer_norm(x), 16)
    g = rng(6)
    big = np.kron(g.integers(0, 256, size=(2, 30, 34, 3)), np.ones((1, 4, 4, 1))).astype(np.uint8)
    frames = [big[:, 4 * t:4 * t + 80, 8 * t:8 * t + 96].copy() for t in range(4)]
    layers, weights, biases = b.layers, *nets.random_weights(b.layers, 5)
    dc = DeepCache(96, 80, layers, weights, biases, n_streams=2, block=8, search_range=8, dtype=dtype, expire_n=4)
    prev, reused_any = {}, 0.0
    try:
        for t, f in enumerate(frames):
            _, stats = dc.infer_frame(torch.as_tensor(f).cuda(), want_stats=True)
            maps = [dc.layer_map(i) for i in range(len(layers))]
            for i, l in enumerate(layers):
                what = f"frame {t} layer {i}"
                if l["kind"] == nets.KIND_LAYER_NORM:
                    assert_near(maps[i], *norm_layer64(maps[l["in0"]], weights[i], biases[i], 1e-5), what)
                elif l["kind"] == nets.KIND_CONV_QUANT:
                    want, bound = quant_layer64(maps[l["in0"]], l, weights[i], biases[i])
                    fresh = torch.ones(2, l["out_h"], l["out_w"], dtype=torch.bool, device="cuda")
                    if not stats[0].refreshed:
                        regs, n_regs = dc.layer_regions(i)
                        for s in range(2):
                            for x0, y0, rw, rh, sx, sy in regs[s, :int(n_regs[s])].cpu().tolist():
                                if rw > 0:
                                    assert torch.equal(maps[i][s, y0:y0 + rh, x0:x0 + rw], prev[i][s, sy:sy + rh, sx:sx + rw]), what
                                    fresh[s, y0:y0 + rh, x0:x0 + rw] = False
                    reused_any += 1 - float(fresh.double().mean())
                    assert_near(maps[i][fresh], want[fresh], bound[fresh], what)
            prev = dict(enumerate(maps))
            assert dc.status() == B.DC_OK
        assert reused_any > 0, "no pixel was reused: the test's frames do not match"
    finally:
        dc.close()


@gpu
@pytest.mark.parametrize("dtype", [B.DC_FP32, B.DC_BF16])
@pytest.mark.parametrize("h,w,cin,cout,S", [(33, 45, 24, 40, 2), (16, 24, 64, 256, 4), (7, 7, 512, 128, 3)])
def test_partial_convolution_with_a_callers_rectangles(h, w, cin, cout, S, dtype):
    """dc_conv_partial on an 8-bit layer: a caller's maps and rectangles, a whole map, and a bad rectangle."""
    t = torch.bfloat16 if dtype == B.DC_BF16 else torch.float32
    b = nets.NetBuilder(h, w)
    x = b.conv(-1, cin, 1)
    q = b.conv_quant(x, cout)
    weights, biases = nets.random_weights(b.layers, 9)
    dc = DeepCache(w, h, b.layers, weights, biases, n_streams=S, block=8, dtype=dtype, max_regions=6)
    try:
        assert B.dc_cache_layer_conv_scheme(dc.handle, q) == 11
        g = torch.Generator(device="cuda")
        g.manual_seed(h)
        inp = torch.randn(S, h, w, cin, generator=g, device="cuda").relu().to(t)
        inp[0, 0, 0] = 0
        prev = torch.randn(S, h, w, cout, generator=g, device="cuda").to(t)
        want, bound = quant_layer64(inp, b.layers[q], weights[q], biases[q])
        assert_near(dc.conv_partial(q, inp), want, bound, "whole map")
        regs = torch.zeros(S, 6, 6, dtype=torch.int32, device="cuda")
        n = torch.zeros(S, dtype=torch.int32, device="cuda")
        rects = {0: [(0, 0, w, 3, 0, 2), (2, 4, 3, 2, 1, 1)], 1: [(0, 0, w, h, 0, 0)]}
        for s, rs in rects.items():
            for k, r in enumerate(rs):
                regs[s, k] = torch.tensor(r, dtype=torch.int32)
            n[s] = len(rs)
        got = dc.conv_partial(q, inp, prev, regs, n)
        fresh = torch.ones(S, h, w, dtype=torch.bool, device="cuda")
        for s, rs in rects.items():
            for x0, y0, rw, rh, sx, sy in rs:
                assert torch.equal(got[s, y0:y0 + rh, x0:x0 + rw], prev[s, sy:sy + rh, sx:sx + rw])
                fresh[s, y0:y0 + rh, x0:x0 + rw] = False
        assert_near(got[fresh], want[fresh], bound[fresh], "the rest")
        assert dc.status() == B.DC_OK
        regs[0, 0] = torch.tensor((0, 0, w + 1, 2, 0, 0), dtype=torch.int32)           # does not lie inside the map: computed, and said so
        got = dc.conv_partial(q, inp, prev, regs, n)
        assert_near(got[0, :2], want[0, :2], bound[0, :2], "a bad rectangle's pixels")
        assert dc.status() == B.DC_ERR_ARG
        with pytest.raises(B.DeepCacheError):
            B.dc_conv_partial(dc.handle, q, inp, prev, regs, n, prev)                  # out is the cached map
    finally:
        dc.close()


@gpu
@pytest.mark.parametrize("dtype", [B.DC_FP32, B.DC_BF16])
def test_partial_convolution_of_rows_longer_than_registers(dtype):
    """Rows of more channels than a CTA holds, read one by one, behind 4 lines of a caller's rectangles each: of the rows that a CTA takes
    (296 apart on 148 SMs, which is 4 lines of 74 pixels) every second one is reused.  A row's largest value is reduced in a slot of shared memory that the
    CTA's next row but one uses again."""
    t = torch.bfloat16 if dtype == B.DC_BF16 else torch.float32
    h, w, cin, cout, S = 20, 74, 8200, 16, 2
    b = nets.NetBuilder(h, w)
    q = b.conv_quant(b.conv(-1, cin, 1), cout)
    weights, biases = nets.random_weights(b.layers, 3)
    dc = DeepCache(w, h, b.layers, weights, biases, n_streams=S, block=8, dtype=dtype, max_regions=4)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(8)
        inp = torch.empty(S * h * w * cin + 1, dtype=t, device="cuda")[1:].view(S, h, w, cin)      # not 16-byte aligned: single elements
        inp.copy_(torch.randn(S, h, w, cin, generator=g, device="cuda") * torch.exp(2 * torch.randn(S, h, w, 1, generator=g, device="cuda")))
        prev = torch.randn(S, h, w, cout, generator=g, device="cuda").to(t)
        regs = torch.zeros(S, 4, 6, dtype=torch.int32, device="cuda")
        for k, y in enumerate((4, 12)):
            regs[:, k] = torch.tensor((0, y, w, 4, 0, y), dtype=torch.int32)
        n = torch.full((S,), 2, dtype=torch.int32, device="cuda")
        fresh = torch.ones(S, h, w, dtype=torch.bool, device="cuda")
        fresh[:, 4:8] = fresh[:, 12:16] = False
        want, bound = quant_layer64(inp, b.layers[q], weights[q], biases[q])
        first = None
        for _ in range(10):
            got = dc.conv_partial(q, inp, prev, regs, n)
            assert_near(got[fresh], want[fresh], bound[fresh], "computed pixels")
            assert torch.equal(got[~fresh], prev[~fresh])
            first = got.clone() if first is None else first
            assert torch.equal(got, first)
        assert dc.status() == B.DC_OK
    finally:
        dc.close()


@gpu
def test_whole_map_layers_ignore_rectangles():
    b = nets.NetBuilder(6, 5)
    q = b.conv_quant(-1, 32, relu=0, whole=True)
    weights, biases = nets.random_weights(b.layers, 2)
    dc = DeepCache(5, 6, b.layers, weights, biases, n_streams=3, block=4, dtype=B.DC_FP32, max_regions=1)
    try:
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        inp, prev = torch.rand(3, 6, 5, 3, generator=g, device="cuda"), torch.rand(3, 1, 1, 32, generator=g, device="cuda")
        regs = torch.tensor([[0, 0, 1, 1, 0, 0]] * 3, dtype=torch.int32, device="cuda").view(3, 1, 6)
        want, bound = quant_layer64(inp, b.layers[q], weights[q], biases[q])
        for args in ((), (prev, regs, torch.ones(3, dtype=torch.int32, device="cuda"))):
            assert_near(dc.conv_partial(q, inp, *args), want, bound, "whole map")
    finally:
        dc.close()


@gpu
@pytest.mark.parametrize("dtype", [B.DC_FP32, B.DC_BF16])
def test_frames_from_the_host_have_the_bits_of_those_on_the_device(dtype):
    """dc_infer_frame_host, with the next frame announced, on a table whose last layer is an 8-bit convolution."""
    h, w, S = 48, 52, 2
    b = nets.NetBuilder(h, w)
    x = b.conv(-1, 32, 3, 1, 1)
    x = b.layer_norm(x)
    b.conv_quant(x, 16)
    weights, biases = nets.random_weights(b.layers, 5)
    frames = frames_of(h, w, 6, S, 8)
    a, c = (DeepCache(w, h, b.layers, weights, biases, n_streams=S, block=8, search_range=8, dtype=dtype, expire_n=4) for _ in range(2))
    try:
        t = torch.bfloat16 if dtype == B.DC_BF16 else torch.float32
        pinned = [torch.as_tensor(f).pin_memory() for f in frames]
        out = torch.empty(a.out_shape(-1), dtype=t).pin_memory()
        for i, f in enumerate(pinned):
            want = a.infer_frame(f.cuda())
            if i + 1 < len(pinned):
                B.dc_prefetch_frame_host(c.handle, pinned[i + 1].data_ptr(), w * 3)
            B.dc_infer_frame_host(c.handle, f.data_ptr(), w * 3, out.data_ptr())
            assert torch.equal(out.cuda(), want), f"frame {i}"
        assert a.status() == c.status() == B.DC_OK
    finally:
        a.close(), c.close()


@gpu
def test_epsilon_is_set_and_empties_the_cache():
    b = nets.NetBuilder(24, 24)
    x = b.conv(-1, 16, 3, 1, 1)
    n = b.layer_norm(x)
    weights, biases = nets.random_weights(b.layers, 2)
    weights[n] = biases[n] = None                                  # ones, zeros
    dc = DeepCache(24, 24, b.layers, weights, biases, block=8, dtype=B.DC_FP32)
    try:
        f = torch.randint(0, 256, (1, 24, 24, 3), dtype=torch.uint8, device="cuda")
        dc.infer_frame(f)
        for eps in (0.25, 1e-5):
            dc.set_norm_epsilon(n, eps)
            out, stats = dc.infer_frame(f, want_stats=True)
            assert stats[0].refreshed == 1
            want, bound = norm_layer64(dc.layer_map(x), None, None, eps)
            assert_near(out, want, bound, f"epsilon {eps}")
        for layer, eps in ((x, 1e-5), (n, -1.0), (7, 1e-5), (n, float("nan"))):
            with pytest.raises(B.DeepCacheError):
                dc.set_norm_epsilon(layer, eps)
    finally:
        dc.close()


@gpu
def test_products_beside_an_inference_on_cta_pairs(monkeypatch):
    """Few rows, short reductions, on another stream than an inference whose convolutions run on CTA pairs with all of tensor memory and whose next frame is
    matched meanwhile (they then leave the most shared memory free): both end, with the results that they have alone."""
    monkeypatch.setenv("DC_CONV_SCHEME", "7")
    h, w, S = 480, 640, 5                                           # blocks of 4: enough of them for the overlapped pass
    b = nets.NetBuilder(h, w)
    x = b.resize_area(-1, 56, 56)
    x = b.conv(x, 64, 3, 1, 1)
    pairs = [b.conv(x, 256, 3, 1, 1)]
    pairs.append(b.conv(pairs[0], 256, 3, 1, 1))
    weights, biases = nets.random_weights(b.layers, 4)
    frames = [torch.as_tensor(f).cuda() for f in frames_of(h, w, 6, S, 2)]
    m, k, n = 8, 512, 4096
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    a, wq = (torch.randint(-127, 128, (r, k), generator=g, device="cuda", dtype=torch.int32).to(torch.int8) for r in (m, n))
    sa, sw = torch.rand(m, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda")
    want, out = (torch.empty(m, n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.dc_matmul_quantized(a, sa, wq, sw, None, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()

    def run(beside):
        dc = DeepCache(w, h, b.layers, weights, biases, n_streams=S, block=4, search_range=4, dtype=B.DC_BF16, expire_n=3)
        try:
            assert [B.dc_cache_layer_conv_scheme(dc.handle, i) for i in pairs] == [7, 7]
            outs = []
            for rounds in range(4):
                for t, f in enumerate(frames):
                    outs.append(dc.infer_frame(f))
                    B.dc_lookahead_frame(dc.handle, frames[(t + 1) % len(frames)], w * 3)
                    if beside:
                        with torch.cuda.stream(side):
                            for _ in range(40):
                                B.dc_matmul_quantized(a, sa, wq, sw, None, out)
            torch.cuda.synchronize()
            assert dc.status() == B.DC_OK
            return outs
        finally:
            dc.close()

    alone, beside = run(False), run(True)
    assert all(torch.equal(p, q) for p, q in zip(alone, beside))
    assert torch.equal(out, want)
