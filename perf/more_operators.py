"""Times group normalisation with an activation (forward, backward) and matrix products in 8-bit floating point with a scale for each block of 128.

What a case stands for: maps are [streams, pixels, channels], channels last.  Group normalisation takes its statistics from all pixels of one stream's map
and the channels of one group.  Blocks: 128 values along the reduction share a scale, in activations and gradients for each row, in weights for 128 output
channels at once.  ``run`` computes a case in elementary torch operations where ``own`` is false, and through the library's entry points where it is true.
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 128
E4M3 = torch.float8_e4m3fn
MOST = 448.0                                              # the largest value of that type
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTIVATIONS = ["none", "relu", "silu"]
_binding = None


def _library():
    global _binding
    if _binding is None:
        from paper_1712_01670_b200 import binding
        _binding = binding
    return _binding


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _norm(name, op, maps, pixels, c, groups, act, dtype):
    return dict(name=name, op=op, maps=maps, pixels=pixels, c=c, groups=groups, act=act, dtype=dtype)


def _quantize(name, m, k, block, dtype):
    return dict(name=name, op="quantize", m=m, k=k, block=block, dtype=dtype)


def _linear(name, op, m, k, n, dtype, relu=False):
    return dict(name=name, op=op, m=m, k=k, n=n, dtype=dtype, relu=relu)


def listed():
    return [
        # the first AlexNet map of 16 streams, 55 x 55 of 96 channels in 32 groups of three
        _norm("group_norm_55x55x96_16streams", "norm", 16, 55 * 55, 96, 32, "relu", "f32"),
        # the widest map of ResNet-50, 56 x 56 of 256 channels, 32 streams
        _norm("group_norm_56x56x256_32streams", "norm", 32, 56 * 56, 256, 32, "silu", "bf16"),
        # gradients: an odd map, 27 x 27 of 260 channels in 20 groups, four streams
        _norm("group_norm_backward_27x27x260_4streams", "backward", 4, 27 * 27, 260, 20, "none", "f32"),
        # the widest map again
        _norm("group_norm_backward_56x56x256_32streams", "backward", 32, 56 * 56, 256, 32, "silu", "bf16"),
        # one stream's 14 x 14 map on its way into 8 bits
        _quantize("quantize_196x1024", 196, 1024, 1, "bf16"),
        # 32 streams' 28 x 28 maps, as rows for the product and as columns for the weights' gradient
        _quantize("quantize_28x28x512_32streams", 32 * 28 * 28, 512, 1, "bf16"),
        # the first fully connected layer behind the AlexNet trunk (6 x 6 x 256), one stream: a single row
        _linear("linear_9216to4096_1row", "linear", 1, 9216, 4096, "bf16", True),
        # the one behind the VGG-16 trunk (7 x 7 x 512), 32 streams
        _linear("linear_25088to4096_32rows", "linear", 32, 25088, 4096, "bf16", True),
        # the largest product: 8192 rows through a square layer
        _linear("linear_8192_4096to4096", "linear", 8192, 4096, 4096, "bf16"),
        # normalisation with its activation and the fourfold widening behind it: one stream's 14 x 14 map
        _linear("group_norm_linear_14x14", "norm_linear", 196, 384, 1536, "bf16", True),
        # both gradients of a layer: odd sizes, a few rows; 32 streams of 14 x 14 pixels
        _linear("linear_backward_1000_333to777", "linear_backward", 1000, 333, 777, "f32"),
        _linear("linear_backward_14x14_512to2048_32streams", "linear_backward", 32 * 196, 512, 2048, "bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "backward", "backward", "quantize", "linear", "linear", "linear", "norm_linear", "linear_backward"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op in ("norm", "backward"):
        groups = rng.choice([1, 4, 8, 16, 32, 32, 32, 5, 20])
        per = _log(rng, 1, 64)
        if rng.random() < 0.6:
            per = max(4, per // 4 * 4)                    # most maps have such channel counts, some do not
        c, maps = groups * per, _log(rng, 1, 32)
        pixels = _log(rng, 1, max(1, min(56 * 56 * 4, 32 * 56 * 56 * 256 // (c * maps) // (2 if dtype == "f32" else 1))))
        return dict(op=op, maps=maps, pixels=pixels, c=c, groups=groups, act=rng.choice(ACTIVATIONS), dtype=dtype)
    k = _log(rng, 16, 16384 if op in ("linear", "quantize") else 2048)
    if rng.random() < 0.7:
        k = max(32, k // 32 * 32)
    if op == "quantize":
        return dict(op=op, m=_log(rng, 1, min(100352, 16 * 1024 * 1024 // k)), k=k, block=rng.choice([1, 1, BLOCK]), dtype=dtype)
    n = _log(rng, 8, 4096)
    if rng.random() < 0.7:
        n = max(8, n // 8 * 8)
    m = _log(rng, 1, min(100352, 8192 * 4096 * 4096 // (k * n), 32 * 1024 * 1024 // k, 32 * 1024 * 1024 // n))
    if op == "linear_backward":
        m = min(m, 25088)
    if op == "norm_linear":
        dtype, k = "bf16", max(32, k // 32 * 32)
    return dict(op=op, m=m, k=k, n=n, dtype=dtype, relu=op != "linear_backward" and rng.random() < 0.5)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _activations(g, rows, c, dtype, positive):
    """A map as a network has it: channels of different size, a few large ones; behind a ReLU (positive) half is zero, and here and
    there a pixel has nothing left."""
    dev = torch.device("cuda")
    size = torch.exp(0.5 * torch.randn(c, generator=g, device=dev))
    size[torch.randint(0, c, (max(1, c // 64),), generator=g, device=dev)] *= 8.0
    x = torch.randn(rows, c, generator=g, device=dev) * size
    if positive:
        x = x.clamp_min_(0.0)
        x[torch.rand(rows, generator=g, device=dev) < 0.01] = 0.0
    else:
        x += 0.5 * torch.randn(1, c, generator=g, device=dev)
    return x.to(dtype)


def _up(v, to):
    return (v + to - 1) // to * to


def _bytes_like(rows, k):
    """Room for rows of 8-bit values, a multiple of 16 bytes apart."""
    return torch.zeros(rows, _up(k, 16), dtype=torch.uint8, device="cuda").view(E4M3)[:, :k]


def _weights(g, n, k):
    """A layer's weights as a program keeps them: 8-bit values and a scale for each 128 x 128 of them, the block's largest value over 448."""
    dev = torch.device("cuda")
    w = torch.randn(n, k, generator=g, device=dev) * math.sqrt(2.0 / k)
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    padded = torch.zeros(nb * BLOCK, kb * BLOCK, device=dev)
    padded[:n, :k] = w
    scale = padded.view(nb, BLOCK, kb, BLOCK).abs().amax((1, 3)) / MOST
    wide = scale.repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)[:n, :k]
    kept = _bytes_like(n, k)
    kept.copy_((w / wide).clamp_(-MOST, MOST).to(E4M3))
    return kept, scale


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dtype, op = TYPES[case["dtype"]], case["op"]
    s = dict(case)
    B = None
    if own:
        B = _library()
    if op in ("norm", "backward"):
        maps, pixels, c, groups = case["maps"], case["pixels"], case["c"], case["groups"]
        s["x"] = _activations(g, maps * pixels, c, dtype, False).view(maps, pixels, c)
        s["gamma"] = 1.0 + 0.2 * torch.randn(c, generator=g, device=dev)
        s["beta"] = 0.1 * torch.randn(c, generator=g, device=dev)
        s["out"] = torch.empty_like(s["x"])
        if op == "norm":
            s["mean"], s["rstd"] = torch.empty(maps, groups, device=dev), torch.empty(maps, groups, device=dev)
        else:
            x = s["x"].double().view(maps, pixels, groups, c // groups)           # what the forward pass has left
            mean = x.mean((1, 3))
            s["mean"], s["rstd"] = mean.float(), torch.rsqrt((x - mean[:, None, :, None]).square().mean((1, 3)) + EPS).float()
            s["dy"] = (0.02 * torch.randn(maps, pixels, c, generator=g, device=dev)).to(dtype)
            s["dgamma"], s["dbeta"] = torch.empty(c, device=dev), torch.empty(c, device=dev)
        if own:
            s["work"] = torch.empty(B.dc_group_norm_workspace(maps, pixels, c, groups), dtype=torch.uint8, device=dev)
        return s
    m, k = case["m"], case["k"]
    mb, kb = -(-m // BLOCK), -(-k // BLOCK)
    s["x"] = _activations(g, m, k, dtype, op in ("linear", "quantize", "linear_backward"))
    if op == "quantize":
        s["q"], s["q_t"] = _bytes_like(m, k), _bytes_like(k, m)
        s["scale"] = torch.empty(-(-m // case["block"]), kb, device=dev)
        s["scale_t"] = torch.empty(-(-k // case["block"]), mb, device=dev)
        return s
    n = case["n"]
    nb = -(-n // BLOCK)
    s["w"], s["w_scale"] = _weights(g, n, k)
    if op == "linear_backward":
        s["dy"] = (0.02 * torch.randn(m, n, generator=g, device=dev)).to(dtype)
        s["w_t"] = _bytes_like(k, n)                      # the same weights, turned, for the gradient of x
        s["w_t"].copy_(s["w"].t())
        s["w_t_scale"] = s["w_scale"].t().contiguous()
        s["dx"], s["dw"] = torch.empty(m, k, dtype=dtype, device=dev), torch.empty(n, k, device=dev)
        s["q"], s["q_scale"], s["q_t"], s["q_t_scale"] = _bytes_like(m, n), torch.empty(m, nb, device=dev), _bytes_like(n, m), torch.empty(n, mb, device=dev)
        s["x_t"], s["x_t_scale"] = _bytes_like(k, m), torch.empty(k, mb, device=dev)
        return s
    s["bias"] = 0.05 * torch.randn(n, generator=g, device=dev)
    s["out"] = torch.empty(m, n, dtype=dtype, device=dev)
    if op == "norm_linear":
        s["x"] = s["x"].view(1, m, k)
        s["gamma"] = 1.0 + 0.2 * torch.randn(k, generator=g, device=dev)
        s["beta"] = 0.1 * torch.randn(k, generator=g, device=dev)
        s["y"] = torch.empty_like(s["x"])
    if own:
        room = B.dc_linear_blocks_workspace(m, k)
        if op == "norm_linear":
            room = max(room, B.dc_group_norm_workspace(1, m, k, 32))
        s["work"] = torch.empty(room, dtype=torch.uint8, device=dev)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _plain_act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _plain_norm(x, s, groups, act):
    maps, pixels, c = x.shape
    v = x.reshape(maps, pixels, groups, c // groups)
    mean = v.mean((1, 3), keepdim=True)
    d = v - mean
    rstd = 1.0 / torch.sqrt((d * d).mean((1, 3), keepdim=True) + EPS)
    z = (d * rstd).reshape(maps, pixels, c) * s["gamma"] + s["beta"]
    return _plain_act(z, act), mean.reshape(maps, groups), rstd.reshape(maps, groups)


def _plain_norm_backward(s):
    x, dy = s["x"].float(), s["dy"].float()
    maps, pixels, c = x.shape
    groups = s["groups"]
    per = c // groups
    xh = ((x.reshape(maps, pixels, groups, per) - s["mean"][:, None, :, None]) * s["rstd"][:, None, :, None]).reshape(maps, pixels, c)
    z = xh * s["gamma"] + s["beta"]
    if s["act"] == "relu":
        dy = torch.where(z > 0, dy, torch.zeros_like(dy))
    elif s["act"] == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        dy = dy * p * (1.0 + z * (1.0 - p))
    gy = (dy * s["gamma"]).reshape(maps, pixels, groups, per)
    xg = xh.reshape(maps, pixels, groups, per)
    dx = (gy - gy.mean((1, 3), keepdim=True) - xg * (gy * xg).mean((1, 3), keepdim=True)) * s["rstd"][:, None, :, None]
    return dx.reshape(maps, pixels, c), (dy * xh).sum((0, 1)), dy.sum((0, 1))


def _plain_blocks(x, block):
    """(8-bit values, scales) of x [rows, k]: blocks of `block` rows by 128 columns share the smallest power of two that takes their largest value to 448 or below."""
    rows, k = x.shape
    rb, kb = -(-rows // block), -(-k // BLOCK)
    padded = torch.zeros(rb * block, kb * BLOCK, device=x.device)
    padded[:rows, :k] = x
    tiles = padded.view(rb, block, kb, BLOCK)
    most = tiles.abs().amax((1, 3))
    half, e = torch.frexp(most)                           # most = half * 2^e, half in [0.5, 1)
    e = torch.clamp(e - 9 + (half > 0.875).int(), min=-126).double()
    scale = torch.where(most > 0, torch.exp2(e).float(), torch.zeros_like(most))
    q = (tiles * torch.exp2(-e).float()[:, None, :, None]).to(E4M3)
    return q.view(rb * block, kb * BLOCK)[:rows, :k], scale


def _plain_values(q, scale, block):
    """What 8-bit values and the scales of their blocks stand for."""
    rows, k = q.shape
    return q.float() * scale.repeat_interleave(block, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :k]


def _plain_linear(x, s):
    y = _plain_values(*_plain_blocks(x, 1), 1) @ _plain_values(s["w"], s["w_scale"], BLOCK).t() + s["bias"]
    return _plain_act(y, "relu") if s["relu"] else y


def run(s):
    op = s["op"]
    if own:
        B = _library()
        act = {"none": B.DC_ACT_NONE, "relu": B.DC_ACT_RELU, "silu": B.DC_ACT_SILU}
        if op == "norm":
            B.dc_group_norm(s["x"], s["groups"], s["gamma"], s["beta"], s["out"], s["mean"], s["rstd"], act[s["act"]], EPS, s["work"])
            return s["out"], s["mean"], s["rstd"]
        if op == "backward":
            B.dc_group_norm_backward(s["dy"], s["x"], s["groups"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["out"], s["dgamma"], s["dbeta"], act[s["act"]], s["work"])
            return s["out"], s["dgamma"], s["dbeta"]
        if op == "quantize":
            B.dc_quantize_blocks(s["x"], s["q"], s["scale"], s["q_t"], s["scale_t"], s["block"])
            return s["q"], s["scale"], s["q_t"], s["scale_t"]
        if op == "linear_backward":
            B.dc_quantize_blocks(s["dy"], s["q"], s["q_scale"], s["q_t"], s["q_t_scale"])
            B.dc_quantize_blocks(s["x"], None, None, s["x_t"], s["x_t_scale"])
            B.dc_matmul_blocks(s["q"], s["q_scale"], s["w_t"], s["w_t_scale"], None, s["dx"])
            B.dc_matmul_blocks(s["q_t"], s["q_t_scale"], s["x_t"], s["x_t_scale"], None, s["dw"])
            return s["dx"], s["dw"]
        x = s["x"]
        if op == "norm_linear":
            B.dc_group_norm(x, 32, s["gamma"], s["beta"], s["y"], None, None, act["silu"], EPS, s["work"])
            x = s["y"][0]
        B.dc_linear_blocks(x, s["w"], s["w_scale"], s["bias"], s["out"], s["relu"], s["work"])
        return s["out"]
    dtype = s["x"].dtype
    if op == "norm":
        y, mean, rstd = _plain_norm(s["x"].float(), s, s["groups"], s["act"])
        return y.to(dtype), mean, rstd
    if op == "backward":
        dx, dgamma, dbeta = _plain_norm_backward(s)
        return dx.to(dtype), dgamma, dbeta
    x = s["x"].float()
    if op == "quantize":
        return (*_plain_blocks(x, s["block"]), *_plain_blocks(x.t(), s["block"]))
    if op == "linear_backward":
        dy = s["dy"].float()
        dx = _plain_values(*_plain_blocks(dy, 1), 1) @ _plain_values(s["w_t"], s["w_t_scale"], BLOCK).t()
        dw = _plain_values(*_plain_blocks(dy.t(), 1), 1) @ _plain_values(*_plain_blocks(x.t(), 1), 1).t()
        return dx.to(dtype), dw
    if op == "norm_linear":
        x = _plain_norm(x, s, 32, "silu")[0][0].to(dtype).float()                 # the map between the two is of the maps' type
    return _plain_linear(x, s).to(dtype)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    e, op = 2 if case["dtype"] == "bf16" else 4, case["op"]
    if op in ("norm", "backward"):
        values = case["maps"] * case["pixels"] * case["c"]
        stats = 8 * case["maps"] * case["groups"]
        if op == "norm":
            return {"bytes": 2 * values * e + stats + 8 * case["c"], "flops": 10 * values}
        return {"bytes": 3 * values * e + stats + 16 * case["c"], "flops": 24 * values}
    m, k = case["m"], case["k"]
    mb, kb = -(-m // BLOCK), -(-k // BLOCK)
    if op == "quantize":
        return {"bytes": m * k * (e + 2) + 4 * (-(-m // case["block"]) * kb + -(-k // case["block"]) * mb), "flops": 4 * m * k}
    n = case["n"]
    weights = n * k + 4 * -(-n // BLOCK) * kb
    if op == "linear_backward":
        return {"bytes": (m * n + 2 * m * k) * e + weights + 4 * n * k, "flops": 4 * m * k * n}
    return {"bytes": (m * k + m * n) * e + weights + 4 * n + (8 * k if op == "norm_linear" else 0), "flops": 2 * m * k * n}


def _exact_e4m3(v):
    """The nearest value of the type, of two the one with the even last bit: three bits behind the leading one, steps of 2^-9 at least."""
    _, e = torch.frexp(v)
    step = torch.exp2(torch.clamp(e.double() - 4.0, min=-9.0))
    return torch.round(v / step) * step


def _exact_blocks(x, block):
    """(q, scale) in 64 bits, block by block along the columns."""
    rows = x.shape[0]
    qs, scales = [], []
    for part in torch.split(x, BLOCK, dim=1):
        most = torch.stack([t.abs().max() for t in torch.split(part, block, dim=0)]) if block > 1 else torch.linalg.vector_norm(part, ord=float("inf"), dim=1)
        step = torch.exp2(torch.clamp(torch.ceil(torch.log2(most / MOST)), min=-126.0))
        step = torch.where(step * MOST < most, step * 2.0, step)                  # should the logarithm have been rounded over a whole number
        step = torch.where((step * (MOST / 2) >= most) & (step > 2.0 ** -126), step / 2.0, step)
        step = torch.where(most > 0, step, torch.zeros_like(step))
        wide = step.repeat_interleave(block)[:rows, None] if block > 1 else step[:, None]
        qs.append(torch.where(wide > 0, _exact_e4m3(part / torch.where(wide > 0, wide, torch.ones_like(wide))), torch.zeros_like(part)))
        scales.append(step)
    return torch.cat(qs, 1), torch.stack(scales, 1)


def _exact_product(a, a_scale, b, b_scale):
    """Sums of each block of the reduction, scaled and added up; the scales of b are for 128 of its rows, or for each."""
    rows = torch.arange(b.shape[0], device=b.device)
    if b_scale.shape[0] != b.shape[0]:
        rows = rows // BLOCK
    out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device=a.device)
    for j, (p, w) in enumerate(zip(torch.split(a, BLOCK, dim=1), torch.split(b, BLOCK, dim=1))):
        out += torch.einsum("mk,nk->mn", p * a_scale[:, j:j + 1], w * b_scale[rows, j:j + 1])
    return out


def _exact_norm(x, gamma, beta, groups, act):
    maps, pixels, c = x.shape
    v = x.view(maps, pixels, groups, -1).permute(0, 2, 1, 3).reshape(maps, groups, -1)
    var, mean = torch.var_mean(v, dim=2, correction=0)
    rstd = (var + EPS).pow(-0.5)
    y = ((v - mean[..., None]) * rstd[..., None]).view(maps, groups, pixels, -1).permute(0, 2, 1, 3).reshape(maps, pixels, c)
    y = torch.addcmul(beta, y, gamma)
    if act != "none":
        y = y.clamp(min=0.0) if act == "relu" else y * torch.sigmoid(y)
    return y, mean, rstd


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    x = s["x"].to(torch.float64)
    if op == "norm":
        return _exact_norm(x, s["gamma"].double(), s["beta"].double(), s["groups"], s["act"])
    if op == "backward":
        # the gradient of sum(dy * act(y)) by the chain rule through each group's centred values u and their scale r
        maps, pixels, c = x.shape
        groups = s["groups"]
        gamma, beta, dy = s["gamma"].double(), s["beta"].double(), s["dy"].double()
        per = c // groups
        wide = lambda t: t.double().repeat_interleave(per, 1).unsqueeze(1)
        r, u = wide(s["rstd"]), x - wide(s["mean"])
        z = torch.addcmul(beta, u * r, gamma)
        if s["act"] == "relu":
            dy = dy * (z > 0)
        elif s["act"] == "silu":
            p = torch.sigmoid(z)
            dy = dy * (p + z * p * (1.0 - p))
        of_group = lambda t: t.view(maps, pixels, groups, per).sum((1, 3)).repeat_interleave(per, 1).unsqueeze(1)
        d_hat, count = dy * gamma, pixels * per
        d_u = d_hat * r - u * r.pow(3) * of_group(d_hat * u) / count
        return d_u - of_group(d_hat) * r / count, torch.einsum("npc,npc,npc->c", dy, u, r.expand_as(u)), dy.sum((0, 1))
    if op == "quantize":
        return (*_exact_blocks(x, s["block"]), *_exact_blocks(x.t(), s["block"]))
    if op == "linear_backward":
        dy = s["dy"].double()
        return (_exact_product(*_exact_blocks(dy, 1), s["w_t"].to(torch.float64), s["w_t_scale"].double()),
                _exact_product(*_exact_blocks(dy.t(), 1), *_exact_blocks(x.t(), 1)))
    if op == "norm_linear":
        x = _exact_norm(x, s["gamma"].double(), s["beta"].double(), 32, "silu")[0][0].to(TYPES[case["dtype"]]).to(torch.float64)
    y = _exact_product(*_exact_blocks(x, 1), s["w"].to(torch.float64), s["w_scale"].double()) + s["bias"].double()
    return y.clamp(min=0.0) if s["relu"] else y
