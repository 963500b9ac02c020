"""Plain float64 forms of the layer norm, the point-wise product and dropout, and what fp32 arithmetic may be off by.

E is half a step of fp32, 2^-24: a rounded result is off by E of itself at most.  A sum of n values in any order of fp32 additions is off by
n E of the sum of magnitudes at most; the matrix cores' sums are given twice that, as they need not round to nearest."""
import math

import torch

E = 2.0 ** -24
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
ACTS = {"none": lambda v: v, "gelu": lambda v: 0.5 * v * torch.special.erfc(-v / math.sqrt(2)), "silu": lambda v: v * torch.sigmoid(v)}


def slope(act, v):
    if act == "gelu":
        return 0.5 * torch.special.erfc(-v / math.sqrt(2)) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(v)
        return s * (1 + v * (1 - s))
    return torch.ones_like(v)


def each(t):
    return t.double().view(1, -1, 1, 1)


def norm(x, weight=None, bias=None, eps=1e-5, grad_out=None, skip=None):
    """{name: (value, how far a result of x's type may be off)}; cpu or gpu tensors."""
    C, half, dtype = x.shape[1], HALF_STEP[x.dtype], x.dtype
    pixels = x.numel() // C
    n = (C + 16) * E  # (a sum over the channels, in any order, and a few operations more)
    x = x.double()
    w = torch.ones(C, device=x.device).double() if weight is None else weight.double()
    w, b = each(w), each(torch.zeros(C, device=x.device) if bias is None else bias)
    mean = x.mean(1, keepdim=True)
    r = 1 / ((x - mean).square().mean(1, keepdim=True) + eps).sqrt()
    u = (x - mean) * r
    size = r * x.abs().mean(1, keepdim=True)   # the mean is off by n of mean |x|, and u by that times r
    off_u = n * (size + 2 * u.abs())            # (r: half of what the mean of squares is off by, and the square root)
    out = w * u + b
    res = {"out": (out, w.abs() * off_u + 4 * E * ((w * u).abs() + b.abs()) + half * out.abs())}
    if grad_out is None:
        return res
    g = grad_out.double()
    a = w * g
    sa, sau = a.mean(1, keepdim=True), (a * u).mean(1, keepdim=True)
    gx = r * (a - sa - u * sau)
    off = gx.abs() * n * (2 + size) + r * (8 * E * (a.abs() + sa.abs() + (u * sau).abs()) + n * a.abs().mean(1, keepdim=True) + sau.abs() * off_u
                                           + u.abs() * (n * (a * u).abs().mean(1, keepdim=True) + (a.abs() * off_u).mean(1, keepdim=True)))
    if skip is not None:
        gx = gx + skip.double()
        off = off + 2 * E * gx.abs()
    res["grad_x"] = gx, off + half * gx.abs()
    depth = (pixels / 64 + 64) * E  # (no thread adds more than a 64th of the pixels, then come sums of threads and blocks)
    res["grad_weight"] = (g * u).sum((0, 2, 3)), (g.abs() * off_u).sum((0, 2, 3)) + (depth + 4 * E) * (g * u).abs().sum((0, 2, 3))
    res["grad_bias"] = g.sum((0, 2, 3)), depth * g.abs().sum((0, 2, 3))
    assert dtype in HALF_STEP
    return res


def product(x, w, b=None, act="none", residual=None, grad_out=None):
    """As above.  Left out of a product at most: fp32 2^-21 (terms beyond the sixth product); bf16 2^-16 (what two terms of a weight leave)."""
    f32, half = x.dtype == torch.float32, HALF_STEP[x.dtype]
    M, K = w.shape
    pixels = x.numel() // K
    x, w = x.double(), w.double()

    def apply(m, t):
        return torch.einsum("mk,nkhw->nmhw", m, t)

    pre, size = apply(w, x), apply(w.abs(), x.abs())
    if b is not None:
        pre, size = pre + each(b), size + each(b).abs()
    sums = (K + 16) * 2 * E
    y = ACTS[act](pre)
    # |act'| <= 1.13; gelu itself within 3.4e-7 + 8.1e-8 |v|, silu within a few steps and |v| steps of the exponential's argument
    off = 1.13 * (2.0 ** (-21 if f32 else -16) + sums) * size
    off = off + (3.4e-7 + 1e-7 * pre.abs() if act == "gelu" else 8 * E * (1 + pre.abs()) * y.abs() if act == "silu" else 0)
    out = y if residual is None else y + residual.double()
    res = {"out": (out, off + E * out.abs() + half * out.abs())}
    if grad_out is None:
        return res
    go = grad_out.double()
    gp = go * slope(act, pre)
    # |act''| <= 0.8; the slope itself within 1e-6
    off_gp = go.abs() * (0.8 * (2.0 ** -21 + sums) * size + 1e-6) if act != "none" else torch.zeros_like(gp)
    gx, gsize = apply(w.t(), gp), apply(w.t().abs(), gp.abs())
    terms = 2.0 ** -21 if f32 else 2.0 ** -16 + (2.0 ** -16 if act != "none" else 0)  # (bf16: two terms of a weight, and of gp)
    res["grad_x"] = gx, apply(w.t().abs(), off_gp) + (terms + (M + 16) * 2 * E) * gsize + half * gx.abs()
    depth = (pixels / 16 + 64) * 2 * E
    res["grad_w"] = (torch.einsum("nmhw,nkhw->mk", gp, x),
                     torch.einsum("nmhw,nkhw->mk", off_gp, x.abs()) + (2.0 ** -21 + depth) * torch.einsum("nmhw,nkhw->mk", gp.abs(), x.abs()))
    res["grad_b"] = gp.sum((0, 2, 3)), off_gp.sum((0, 2, 3)) + depth * gp.abs().sum((0, 2, 3))
    return res


def check(got, want, what=""):
    """A result against (value, tolerance)."""
    value, off = want
    assert got.shape == value.shape, (what, got.shape, value.shape)
    d = (got.double() - value.to(got.device)).abs()
    bad = ~(d <= off.to(got.device))
    assert not bad.any(), (what, int(bad.sum()), d[bad].max().item(), off.to(got.device)[bad].min().item())


def dropped_of(p):
    return int(math.floor(p * 65536 + 0.5))


def philox(block, offset, seed):
    """Four 32-bit words of one block, in whole numbers of Python."""
    low = 2 ** 32 - 1
    x = [block & low, block >> 32, offset & low, offset >> 32]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(b >> 32) ^ x[1] ^ k[0], b & low, (a >> 32) ^ x[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return x


def draws(units, seed, offset, first=0):
    """The 16-bit draws of units first, first + 1, ..."""
    out, held, words = [], None, None
    for u in range(first, first + units):
        if u // 8 != held:
            held, words = u // 8, philox(u // 8, offset, seed)
        out.append(words[u % 8 // 2] >> 16 * (u % 2) & 0xFFFF)
    return torch.tensor(out)


def kept(shape, p, seed, offset, over):
    N, C, H, W = shape
    sizes = {"element": shape, "plane": (N, C, 1, 1), "image": (N, 1, 1, 1)}[over]
    return (draws(math.prod(sizes), seed, offset) >= dropped_of(p)).view(sizes).expand(shape)


def dropout(x, p, seed, offset, over, residual=None):
    """The same fp32 operations one by one: results are equal."""
    scale = torch.tensor(65536 / (65536 - dropped_of(p)), dtype=torch.float64).float()
    y = torch.where(kept(x.shape, p, seed, offset, over), x.float() * scale, torch.zeros(()))
    return (y if residual is None else y + residual.float()).to(x.dtype)
