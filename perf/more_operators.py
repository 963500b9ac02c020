"""Calls of the operators that stand on both sides of window attention in a network's block: the layer norm over each pixel's
channels, the point-wise product with bias, activation and residual in its epilogue, both with their gradients, and dropout with the
residual added, its mask drawn from a counter-based generator and never stored.  One dict per case; inputs are made on the GPU from a seed.

`run` computes a case in its plain form, elementary torch operations in 32 bits, or, where `own` is set, through the public
entry points (paper_2503_06671_amd.binding).  `exact` is the same result in 64 bits, written from the definition.

Sizes are those of the other calls this library is measured on: feature maps of 720p outputs, training batches of 64x64 crops,
photographs of no particular size; 64 channels with 128 hidden ones, 192 with 576, and the widest parameters of the optimiser's cases.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _norm(train, dtype, C, H, W, N=1, affine=True, skip=False):
    return dict(kind="norm", train=train, dtype=dtype, N=N, C=C, H=H, W=W, affine=affine, skip=skip)


def _product(train, dtype, K, M, H, W, N=1, act="none", bias=True, residual=False):
    return dict(kind="product", train=train, dtype=dtype, N=N, K=K, M=M, H=H, W=W, act=act, bias=bias, residual=residual)


def _dropout(train, dtype, C, H, W, N=1, p=0.1, over="element", residual=True):
    return dict(kind="dropout", train=train, dtype=dtype, N=N, C=C, H=H, W=W, p=p, over=over, residual=residual)


def listed():
    def named(name, c):
        return dict(c, name=name)

    return [
        # one small tile of an image: latency and the host's own time
        named("norm_64x64_f32", _norm(False, "f32", 64, 64, 64)),
        # the larger model's norm on the feature map of a 720p output
        named("norm_180x320_c192_bf16", _norm(False, "bf16", 192, 180, 320)),
        # training on a batch of crops: the norm in front of attention, its gradients and the skip connection's added
        named("norm_train_64x64x64_bf16", _norm(True, "bf16", 64, 64, 64, N=64, skip=True)),
        # photographs of odd size, channels that fill no group
        named("norm_train_2x339x511_c45_f32", _norm(True, "f32", 45, 339, 511, N=2)),
        # queries, keys and values of one small tile: latency
        named("product_64x64_64_192_f32", _product(False, "f32", 64, 192, 64, 64, bias=False)),
        # the larger model's queries, keys and values on the feature map of a 720p output
        named("product_180x320_192_576_bf16", _product(False, "bf16", 192, 576, 180, 320)),
        # the way back from attention to the residual stream, a photograph of odd size
        named("product_339x511_64_64_res_f32", _product(False, "f32", 64, 64, 339, 511, residual=True)),
        # training on a batch of crops: a feed-forward network's first layer with all gradients
        named("product_train_64x64x64_64_128_gelu_bf16", _product(True, "bf16", 64, 128, 64, 64, N=64, act="gelu")),
        # crops of odd size in fp32, channels that fill no tile, activation and residual
        named("product_train_5x50x61_96_45_silu_res_f32", _product(True, "f32", 96, 45, 50, 61, N=5, act="silu", residual=True)),
        # a wide model's layer: the matrix units' rate
        named("product_train_16x64x64_640_1280_gelu_bf16", _product(True, "bf16", 640, 1280, 64, 64, N=16, act="gelu")),
        # the larger model's branch in a small batch, stochastic depth over whole images: latency
        named("dropout_4x64x64_c192_images_f32", _dropout(False, "f32", 192, 64, 64, N=4, p=0.2, over="image")),
        # training on a batch of crops: elements dropped, the residual added, and the way back
        named("dropout_train_64x64x64_bf16", _dropout(True, "bf16", 64, 64, 64, N=64)),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "product", "product", "dropout"))
    while True:
        dtype, train = rng.choice(("f32", "bf16")), rng.random() < 0.5
        N, H, W = _log(rng, 1, 64), _log(rng, 1, 360), _log(rng, 1, 640)
        if rng.random() < 0.15:  # a single token of each sequence
            H = W = 1
        pixels = N * H * W
        if kind == "product":
            c = _product(train, dtype, _log(rng, 3, 1280), _log(rng, 3, 1280), H, W, N=N, act=rng.choice(("none", "gelu", "silu")), bias=rng.random() < 0.7,
                         residual=rng.random() < 0.4)
            if pixels * c["K"] * c["M"] * (3 if train else 1) <= 1.6e11 and pixels * (c["K"] + c["M"]) <= 1.2e8:
                return c
            continue
        C = _log(rng, 3, 1280)
        if pixels * C > 2e7:
            continue
        if kind == "norm":
            return _norm(train, dtype, C, H, W, N=N, affine=rng.random() < 0.8, skip=train and rng.random() < 0.5)
        return _dropout(train, dtype, C, H, W, N=N, p=round(rng.uniform(0.0, 0.9), 3), over=rng.choice(("element", "element", "plane", "image")),
                        residual=rng.random() < 0.7)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, N, H, W = DTYPES[c["dtype"]], c["N"], c["H"], c["W"]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)

    s = dict(case=c)
    if c["kind"] == "norm":
        # a residual stream: every channel with a mean and a size of its own
        C = c["C"]
        size = torch.exp(0.7 * torch.randn(C, 1, 1, device="cuda", generator=g))
        mean = torch.randn(C, 1, 1, device="cuda", generator=g)
        s["x"] = (torch.randn(N, C, H, W, device="cuda", generator=g) * size + mean).to(dt)
        s["weight"] = 1.0 + normal(C, scale=0.2, dtype=torch.float32) if c["affine"] else None
        s["bias"] = normal(C, scale=0.2, dtype=torch.float32) if c["affine"] else None
        s["grad_out"] = normal(N, C, H, W) if c["train"] else None
        s["grad_skip"] = normal(N, C, H, W) if c["skip"] else None
    elif c["kind"] == "product":
        K, M = c["K"], c["M"]
        s["x"] = normal(N, K, H, W)
        s["w"] = normal(M, K, scale=K ** -0.5, dtype=torch.float32)
        s["b"] = normal(M, scale=0.2, dtype=torch.float32) if c["bias"] else None
        s["residual"] = normal(N, M, H, W) if c["residual"] else None
        s["grad_out"] = normal(N, M, H, W) if c["train"] else None
    else:
        s["x"] = normal(N, c["C"], H, W)
        s["residual"] = normal(N, c["C"], H, W) if c["residual"] else None
        s["grad_out"] = normal(N, c["C"], H, W) if c["train"] else None
        # the key, and how many calls the generator has seen (beyond 32 bits in a long training)
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 * (seed + 1) % 2 ** 63, 2 ** 32 + 5 * seed
    return s


def _sum_pixels(x):
    """[N, C, H, W] -> [C]: a long sum."""
    return x.sum((2, 3)).double().sum(0).float()


def _norm_plain(s):
    c, dt = s["case"], s["x"].dtype
    x = s["x"].float()
    each = (1, -1, 1, 1)
    d = x - x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    xh = d * r
    y = xh if s["weight"] is None else xh * s["weight"].view(each) + s["bias"].view(each)
    out = {"out": y.to(dt)}
    if not c["train"]:
        return out
    g = s["grad_out"].float()
    a = g if s["weight"] is None else g * s["weight"].view(each)
    gx = r * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    if s["grad_skip"] is not None:
        gx = gx + s["grad_skip"].float()
    out["grad_x"] = gx.to(dt)
    if s["weight"] is not None:
        out["grad_weight"], out["grad_bias"] = _sum_pixels(g * xh), _sum_pixels(g)
    return out


def _norm_own(s):
    from paper_2503_06671_amd import binding

    c = s["case"]
    if not c["train"]:
        return {"out": binding.layernorm_forward(s["x"], s["weight"], s["bias"], eps=EPS)}
    if "saved" not in s:  # the buffers that a training program keeps
        s["saved"] = binding.new_layernorm_saved(c["N"], c["H"], c["W"])
        s["ws"] = binding.new_layernorm_backward_workspace(c["N"], c["C"], c["H"], c["W"])
    out = binding.layernorm_forward(s["x"], s["weight"], s["bias"], eps=EPS, saved=s["saved"])
    grads = binding.layernorm_backward(s["x"], s["grad_out"], s["saved"], s["ws"], s["weight"], s["bias"], grad_skip=s["grad_skip"])
    return {"out": out, **{n: grads[n] for n in ("grad_x", "grad_weight", "grad_bias") if n in grads}}


def _activation(act, pre):
    if act == "gelu":
        return 0.5 * pre * (1.0 + torch.erf(pre * math.sqrt(0.5)))
    return pre / (1.0 + torch.exp(-pre)) if act == "silu" else pre


def _slope(act, pre):
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(pre * math.sqrt(0.5))) + pre * torch.exp(-0.5 * pre * pre) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-pre))
    return sig * (1.0 + pre * (1.0 - sig))


def _product_plain(s):
    c, dt = s["case"], s["x"].dtype
    N, K, M, H, W = (c[n] for n in ("N", "K", "M", "H", "W"))
    x = s["x"].float().reshape(N, K, H * W)
    pre = torch.matmul(s["w"], x)
    if s["b"] is not None:
        pre = pre + s["b"].view(-1, 1)
    y = _activation(c["act"], pre).reshape(N, M, H, W)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"out": y.to(dt)}
    if not c["train"]:
        return out
    gp = s["grad_out"].float().reshape(N, M, H * W)
    if c["act"] != "none":
        gp = gp * _slope(c["act"], pre)
    del pre
    out["grad_x"] = torch.matmul(s["w"].t().contiguous(), gp).reshape(N, K, H, W).to(dt)
    out["grad_w"] = torch.matmul(gp, x.transpose(1, 2).contiguous()).double().sum(0).float()
    if s["b"] is not None:
        out["grad_b"] = _sum_pixels(gp.reshape(N, M, H, W))
    return out


def _product_own(s):
    from paper_2503_06671_amd import binding

    c = s["case"]
    out = {"out": binding.pointwise_forward(s["x"], s["w"], s["b"], act=c["act"], residual=s["residual"])}
    if not c["train"]:
        return out
    if "ws" not in s:  # the buffer that a training program keeps
        s["ws"] = binding.new_pointwise_backward_workspace(c["N"], c["K"], c["M"], c["H"], c["W"], s["x"].dtype, act=c["act"])
    grads = binding.pointwise_backward(s["x"], s["grad_out"], s["w"], s["ws"], s["b"], act=c["act"])
    return {**out, **{n: grads[n] for n in ("grad_x", "grad_w", "grad_b") if n in grads}}


def _words(count, seed, offset):
    """`count` generator blocks of four 32-bit words: Philox4x32 with ten rounds, counter (block, offset), key the seed."""
    low = 0xFFFFFFFF
    block = torch.arange(count, device="cuda")
    x = [block & low, block >> 32, torch.full_like(block, offset & low), torch.full_like(block, offset >> 32 & low)]
    k0, k1 = seed & low, seed >> 32 & low

    def round_(x, k0, k1):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        return [(b >> 32 & low) ^ x[1] ^ k0, b & low, (a >> 32 & low) ^ x[3] ^ k1, a & low]

    for _ in range(10):
        x = round_(x, k0, k1)
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(x, 1)


def _dropped_of(p):
    """How many of the 65536 values of a draw drop."""
    return int(math.floor(p * 65536.0 + 0.5))


def _kept(s):
    c = s["case"]
    units = {"element": c["N"] * c["C"] * c["H"] * c["W"], "plane": c["N"] * c["C"], "image": c["N"]}[c["over"]]
    words = _words((units + 7) // 8, s["seed"], s["offset"])
    draws = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:units]
    keep = draws >= _dropped_of(c["p"])
    shape = {"element": (c["N"], c["C"], c["H"], c["W"]), "plane": (c["N"], c["C"], 1, 1), "image": (c["N"], 1, 1, 1)}[c["over"]]
    return keep.reshape(shape)


def _dropout_plain(s):
    c, dt = s["case"], s["x"].dtype
    keep, scale = _kept(s), 65536.0 / (65536 - _dropped_of(c["p"]))
    zero = torch.zeros((), device="cuda")
    y = torch.where(keep, s["x"].float() * scale, zero)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"out": y.to(dt)}
    if c["train"]:
        out["grad_x"] = torch.where(keep, s["grad_out"].float() * scale, zero).to(dt)
    return out


def _dropout_own(s):
    from paper_2503_06671_amd import binding

    c = s["case"]
    kw = dict(p=c["p"], seed=s["seed"], offset=s["offset"], over=c["over"])
    out = {"out": binding.dropout_forward(s["x"], residual=s["residual"], **kw)}
    if c["train"]:
        out["grad_x"] = binding.dropout_backward(s["grad_out"], **kw)
    return out


def run(state):
    kind = state["case"]["kind"]
    if kind == "norm":
        return (_norm_own if own else _norm_plain)(state)
    if kind == "product":
        return (_product_own if own else _product_plain)(state)
    return (_dropout_own if own else _dropout_plain)(state)


def work(case):
    c = case
    size = 4.0 if c["dtype"] == "f32" else 2.0
    pixels = float(c["N"] * c["H"] * c["W"])
    if c["kind"] == "norm":
        tensors = 2 + (2 + c["skip"] if c["train"] else 0)  # x and out; the gradients of out, of x and the skip connection's
        weights = (16.0 if c["train"] else 8.0) * c["C"] if c["affine"] else 0.0
        return {"bytes": tensors * pixels * c["C"] * size + weights, "flops": (20.0 if c["train"] else 8.0) * pixels * c["C"]}
    if c["kind"] == "product":
        K, M = c["K"], c["M"]
        planes = (K + M) * (2 if c["train"] else 1) + (M if c["residual"] else 0)
        weights = 4.0 * (K * M + (M if c["bias"] else 0)) * (2 if c["train"] else 1)
        return {"bytes": planes * pixels * size + weights, "flops": (6.0 if c["train"] else 2.0) * pixels * K * M}
    tensors = 2 + c["residual"] + (2 if c["train"] else 0)
    return {"bytes": tensors * pixels * c["C"] * size, "flops": (3.0 if c["train"] else 2.0) * pixels * c["C"]}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "product": _exact_product, "dropout": _exact_dropout}[case["kind"]](s)


def _exact_norm(s):
    """Pixels as rows of a matrix; the gradient by the Jacobian's two projections."""
    c = s["case"]
    N, C, H, W = (c[n] for n in ("N", "C", "H", "W"))

    def rows(t):
        return t.double().permute(0, 2, 3, 1).reshape(-1, C)

    def back(t):
        return t.reshape(N, H, W, C).permute(0, 3, 1, 2).contiguous()

    x = rows(s["x"])
    mean = x.sum(1, keepdim=True) / C
    std = (((x - mean) ** 2).sum(1, keepdim=True) / C + EPS).sqrt()
    unit = (x - mean) / std
    w = torch.ones(C, device="cuda", dtype=torch.float64) if s["weight"] is None else s["weight"].double()
    out = {"out": back(unit * w + (0.0 if s["bias"] is None else s["bias"].double()))}
    if c["train"]:
        g = rows(s["grad_out"])
        along = g * w
        along = along - along.sum(1, keepdim=True) / C
        gx = back((along - unit * (along * unit).sum(1, keepdim=True) / C) / std)
        out["grad_x"] = gx if s["grad_skip"] is None else gx + s["grad_skip"].double()
        if s["weight"] is not None:
            out["grad_weight"], out["grad_bias"] = (g * unit).sum(0), g.sum(0)
    return out


def _exact_product(s):
    """Image by image."""
    c = s["case"]
    w = s["w"].double()
    b = 0.0 if s["b"] is None else s["b"].double()[:, None]
    parts, grad_w, grad_b = {"out": [], "grad_x": []}, 0.0, 0.0
    for n in range(c["N"]):
        x = s["x"][n].double().flatten(1)
        pre = w @ x + b
        if c["act"] == "gelu":
            phi = torch.special.erfc(-pre / math.sqrt(2.0)) / 2
            y, slope = pre * phi, phi + pre * torch.exp(-pre ** 2 / 2) / math.sqrt(2 * math.pi)
        elif c["act"] == "silu":
            sig = torch.sigmoid(pre)
            y, slope = pre * sig, sig + pre * sig * torch.sigmoid(-pre)
        else:
            y, slope = pre, None
        y = y.reshape(c["M"], c["H"], c["W"])
        parts["out"].append(y if s["residual"] is None else y + s["residual"][n].double())
        if c["train"]:
            g = s["grad_out"][n].double().flatten(1)
            g = g if slope is None else g * slope
            parts["grad_x"].append((w.t() @ g).reshape(c["K"], c["H"], c["W"]))
            grad_w, grad_b = grad_w + g @ x.t(), grad_b + g.sum(1)
    out = {"out": torch.stack(parts["out"])}
    if c["train"]:
        out["grad_x"], out["grad_w"] = torch.stack(parts["grad_x"]), grad_w
        if s["b"] is not None:
            out["grad_b"] = grad_b
    return out


def _exact_dropout(s):
    """The generator on the host, its 64-bit products in unsigned numbers."""
    c = s["case"]
    shape = dict(element=(c["N"], c["C"], c["H"], c["W"]), plane=(c["N"], c["C"], 1, 1), image=(c["N"], 1, 1, 1))[c["over"]]
    units = math.prod(shape)
    n = np.arange(-(-units // 8), dtype=np.uint64)
    half, low = np.uint64(32), np.uint64(0xFFFFFFFF)
    state = np.stack([n & low, n >> half, np.full_like(n, s["offset"] % 2 ** 32), np.full_like(n, s["offset"] // 2 ** 32 % 2 ** 32)])
    for turn in range(10):
        key = [np.uint64((s["seed"] // 2 ** (32 * i) + turn * weyl) % 2 ** 32) for i, weyl in enumerate((0x9E3779B9, 0xBB67AE85))]
        first, second = state[0] * np.uint64(0xD2511F53), state[2] * np.uint64(0xCD9E8D57)
        state = np.stack([second >> half ^ state[1] ^ key[0], second & low, first >> half ^ state[3] ^ key[1], first & low])
    draws = np.ascontiguousarray(state.T.astype("<u4")).view("<u2").reshape(-1)[:units]
    dropped = round(c["p"] * 65536)
    share = torch.from_numpy((draws >= dropped).reshape(shape)).cuda().double() * (65536 / (65536 - dropped))
    y = s["x"].double() * share
    out = {"out": y if s["residual"] is None else y + s["residual"].double()}
    if c["train"]:
        out["grad_x"] = s["grad_out"].double() * share
    return out
