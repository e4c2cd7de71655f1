"""Times layer normalisation over a pixel's channels (forward, backward) and matrix products in 8-bit integers.

What a case stands for: maps are [rows, channels], a row being a pixel (of every stream) or, in front of a fully connected
layer, a stream.  ``run`` computes a case in elementary torch operations where ``own`` is false, and through the
library's entry points where it is true.
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
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
def _norm(name, op, rows, c, dtype):
    return dict(name=name, op=op, rows=rows, c=c, dtype=dtype)


def _linear(name, op, m, k, n, dtype, relu):
    return dict(name=name, op=op, m=m, k=k, n=n, dtype=dtype, relu=relu)


def listed():
    return [
        # one stream's last ResNet-50 map, 7 x 7 pixels of 2048 channels: a latency
        _norm("norm_7x7x2048", "norm", 49, 2048, "bf16"),
        # the first AlexNet map of 16 streams, 55 x 55 of 96 channels
        _norm("norm_55x55x96_16streams", "norm", 16 * 55 * 55, 96, "f32"),
        # the widest map of ResNet-50, 56 x 56 of 256 channels, 32 streams
        _norm("norm_56x56x256_32streams", "norm", 32 * 56 * 56, 256, "bf16"),
        # gradients: one stream's 14 x 14 map of 1024 channels
        _norm("backward_14x14x1024", "backward", 196, 1024, "bf16"),
        # an odd map, 27 x 27 of 257 channels, four streams
        _norm("backward_27x27x257_4streams", "backward", 4 * 27 * 27, 257, "f32"),
        # the widest map again
        _norm("backward_56x56x256_32streams", "backward", 32 * 56 * 56, 256, "bf16"),
        # the first fully connected layer behind the AlexNet trunk (6 x 6 x 256), one stream: a single row
        _linear("linear_9216to4096_1row", "linear", 1, 9216, 4096, "bf16", True),
        # the one behind the VGG-16 trunk (7 x 7 x 512), 32 streams
        _linear("linear_25088to4096_32rows", "linear", 32, 25088, 4096, "bf16", True),
        # a 1 x 1 convolution that widens: 56 x 56 pixels, 64 to 256 channels, 7 streams
        _linear("linear_56x56_64to256", "linear", 7 * 56 * 56, 64, 256, "f32", False),
        # the largest product: 8192 rows through a square layer
        _linear("linear_8192_4096to4096", "linear", 8192, 4096, 4096, "bf16", False),
        # normalisation and the fourfold widening behind it: one stream of 14 x 14, 32 streams of 28 x 28
        _linear("norm_linear_14x14", "norm_linear", 196, 384, 1536, "bf16", True),
        _linear("norm_linear_28x28_32streams", "norm_linear", 32 * 28 * 28, 512, 2048, "bf16", True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "backward", "linear", "linear", "norm_linear"])
    if op in ("norm", "backward"):
        c = _log(rng, 16, 4096)
        if rng.random() < 0.6:
            c = max(16, c // 16 * 16)                    # most maps have such channel counts, some do not
        rows = _log(rng, 1, min(200000, 32 * 56 * 56 * 256 // c))
        return dict(op=op, rows=rows, c=c, dtype=rng.choice(["f32", "bf16"]) if rows * c * 2 <= 32 * 56 * 56 * 256 else "bf16")
    k, n = _log(rng, 16, 16384 if op == "linear" else 2048), _log(rng, 8, 4096)
    if rng.random() < 0.7:
        k, n = max(16, k // 16 * 16), max(8, n // 8 * 8)
    m = _log(rng, 1, min(100352, 8192 * 4096 * 4096 // (k * n), 32 * 1024 * 1024 // k, 32 * 1024 * 1024 // n))
    dtype = "bf16" if op == "norm_linear" else rng.choice(["f32", "bf16"])
    return dict(op=op, m=m, k=k, n=n, dtype=dtype, relu=rng.random() < 0.5)


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
        x += 0.5 * torch.randn(rows, 1, generator=g, device=dev)
    return x.to(dtype)


def _weights(g, n, k):
    """A layer's weights as a program keeps them: 8-bit integers, one scale per output channel, rows 16 bytes apart or a multiple."""
    dev = torch.device("cuda")
    w = torch.randn(n, k, generator=g, device=dev) * math.sqrt(2.0 / k)
    scale = w.abs().amax(1) / 127.0
    kept = torch.zeros(n, (k + 15) // 16 * 16, dtype=torch.int8, device=dev)
    kept[:, :k] = torch.round(w / scale[:, None]).clamp_(-127, 127).to(torch.int8)
    return kept[:, :k], scale


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dtype = TYPES[case["dtype"]]
    s = dict(case)
    if case["op"] in ("norm", "backward"):
        rows, c = case["rows"], case["c"]
        s["x"] = _activations(g, rows, c, dtype, False)
        s["gamma"] = 1.0 + 0.2 * torch.randn(c, generator=g, device=dev)
        s["beta"] = 0.1 * torch.randn(c, generator=g, device=dev)
        if case["op"] == "norm":
            s["out"] = torch.empty(rows, c, dtype=dtype, device=dev)
        else:
            x = s["x"].double()                           # what the forward pass has left
            mean = x.mean(1)
            s["mean"], s["rstd"] = mean.float(), torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS).float()
            s["dy"] = (0.02 * torch.randn(rows, c, generator=g, device=dev)).to(dtype)
            s["out"] = torch.empty(rows, c, dtype=dtype, device=dev)
        s["stat"] = torch.empty(2, rows if case["op"] == "norm" else c, device=dev)
        # scratch memory, as much as two rows of gradients for each SM twice
        s["work"] = torch.empty(2 * 4 * c * 2 * 148 if case["op"] == "backward" else 0, dtype=torch.uint8, device=dev)
        return s
    m, k, n = case["m"], case["k"], case["n"]
    s["x"] = _activations(g, m, k, dtype, case["op"] == "linear")
    s["w"], s["w_scale"] = _weights(g, n, k)
    s["bias"] = 0.05 * torch.randn(n, generator=g, device=dev)
    s["out"] = torch.empty(m, n, dtype=dtype, device=dev)
    s["scale"] = torch.empty(m, device=dev)
    s["q"] = torch.empty(m, (k + 15) // 16 * 16, dtype=torch.int8, device=dev)[:, :k]
    if case["op"] == "norm_linear":
        s["gamma"] = 1.0 + 0.2 * torch.randn(k, generator=g, device=dev)
        s["beta"] = 0.1 * torch.randn(k, generator=g, device=dev)
    else:
        s["work"] = torch.empty(m * ((k + 15) // 16 * 16 + 4) + 256, dtype=torch.uint8, device=dev)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _plain_norm(x, gamma, beta):
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    return d * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def _plain_linear(x, s):
    """Each row of x in 127 steps of its largest value either way; 64 bits, because values lie on the border between two steps."""
    x = x.double()
    most = x.abs().amax(1, keepdim=True)
    q = torch.round(x * 127.0 / torch.where(most > 0, most, torch.ones_like(most))).float()
    y = (q @ s["w"].float().t()) * (most / 127.0).float() * s["w_scale"] + s["bias"]
    return torch.relu(y) if s["relu"] else y


def run(s):
    op = s["op"]
    if own:
        B = _library()
        if op == "norm":
            B.dc_layer_norm(s["x"], s["gamma"], s["beta"], s["out"], s["stat"][0], s["stat"][1], EPS)
            return s["out"], s["stat"][0], s["stat"][1]
        if op == "backward":
            B.dc_layer_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["out"], s["stat"][0], s["stat"][1], s["work"])
            return s["out"], s["stat"][0], s["stat"][1]
        if op == "linear":
            B.dc_linear_quantized(s["x"], s["w"], s["w_scale"], s["bias"], s["out"], s["relu"], s["work"])
        else:
            B.dc_layer_norm_quantize(s["x"], s["gamma"], s["beta"], s["q"], s["scale"], None, EPS)
            B.dc_matmul_quantized(s["q"], s["scale"], s["w"], s["w_scale"], s["bias"], s["out"], s["relu"])
        return s["out"]
    dtype = s["x"].dtype
    x = s["x"].float()
    if op == "norm":
        y, mean, rstd = _plain_norm(x, s["gamma"], s["beta"])
        return y.to(dtype), mean, rstd
    if op == "backward":
        dy = s["dy"].float()
        xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
        gy = dy * s["gamma"]
        dx = (gy - gy.mean(1, keepdim=True) - xhat * (gy * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
        return dx.to(dtype), (dy * xhat).sum(0), dy.sum(0)
    if op == "norm_linear":
        x = _plain_norm(x, s["gamma"], s["beta"])[0].to(dtype)      # the map between the two is of the maps' type
    return _plain_linear(x, s).to(dtype)


# ---------------------------------------------------------------------------
# what a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        rows, c = case["rows"], case["c"]
        return {"bytes": 2 * rows * c * e + 8 * rows + 8 * c, "flops": 8 * rows * c}
    if case["op"] == "backward":
        rows, c = case["rows"], case["c"]
        return {"bytes": 3 * rows * c * e + 8 * rows + 12 * c, "flops": 14 * rows * c}
    m, k, n = case["m"], case["k"], case["n"]
    return {"bytes": m * k * e + n * k + 8 * n + m * n * e + (8 * k if case["op"] == "norm_linear" else 0), "flops": 2 * m * k * n}


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].to(torch.float64)
    n = x.shape[1]
    if case["op"] == "backward":
        # the gradient of sum(dy * y) by the chain rule through the centred row u, its scale r and the affine map
        dy, r, u = s["dy"].to(torch.float64), s["rstd"].to(torch.float64), x - s["mean"].to(torch.float64).unsqueeze(1)
        d_hat = dy * s["gamma"].to(torch.float64)
        d_u = d_hat * r.unsqueeze(1)
        d_r = torch.einsum("rc,rc->r", d_hat, u)
        d_u = d_u - u * (d_r * r.pow(3) / n).unsqueeze(1)
        dx = d_u - d_hat.sum(1, keepdim=True) * r.unsqueeze(1) / n
        return dx, torch.einsum("rc,rc,r->c", dy, u, r), torch.einsum("rc->c", dy)
    if case["op"] in ("norm", "norm_linear"):
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + EPS).pow(-0.5)
        y = torch.addcmul(s["beta"].to(torch.float64), (x - mean.unsqueeze(1)) * rstd.unsqueeze(1), s["gamma"].to(torch.float64))
        if case["op"] == "norm":
            return y, mean, rstd
        x = y.to(TYPES[case["dtype"]]).to(torch.float64)
    most = torch.linalg.vector_norm(x, ord=float("inf"), dim=1)
    q = torch.nan_to_num((x * 127.0).div(most.unsqueeze(1)), nan=0.0).round()
    y = torch.einsum("mk,nk->mn", q, s["w"].to(torch.float64))
    y = y * torch.outer(most / 127.0, s["w_scale"].to(torch.float64)) + s["bias"].to(torch.float64)
    return y.clamp(min=0.0) if case["relu"] else y
