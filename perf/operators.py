"""Calls of the operators that stand around the module in a network and its training: self-attention over windows of a
feature map with a learned relative position bias, that attention with its gradients, and the AdamW step over all of a
network's parameters.  One dict per case; inputs are made on the GPU from a seed.

`run` computes a case in its plain form, elementary torch operations in 32 bits, or, where `own` is set, through the public
entry points (paper_2503_06671_amd.binding).  `exact` is the same result in 64 bits, written from the definition window by
window and tensor by tensor.

Sizes are those of the other calls this library is measured on (feature maps of 720p outputs, training batches of 64x64
crops, photographs of no particular size), with the windows of the network (32x32; 48x48 with 192 channels) and smaller ones.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 256        # elements of a tensor that share a scale where the optimiser's states are held in 8 bits
CODE_MAX = 448.0   # the largest value of torch.float8_e4m3fn
TINY = 2.0 ** -100  # blocks whose magnitudes all lie below this hold zeros


def _attn(kind, dtype, H, W, N=1, heads=4, kv_heads=None, d=16, win=(32, 32), edges=0, masked=False):
    return dict(kind=kind, dtype=dtype, N=N, H=H, W=W, heads=heads, kv_heads=kv_heads or heads, d=d, win_h=win[0], win_w=win[1],
                edges=edges, masked=masked)


def _adamw(states, grads, blocks, modules, channels, hidden):
    return dict(kind="adamw", states=states, grads=grads, blocks=blocks, modules=modules, channels=channels, hidden=hidden)


def listed():
    def named(name, c):
        return dict(c, name=name)

    return [
        # one small tile of an image: latency, launches and the host's own time
        named("attend_64x64_f32", _attn("attend", "f32", 64, 64)),
        # the feature map of a 720p output at x4, the usual inference call, in both storage types
        named("attend_180x320_f32", _attn("attend", "f32", 180, 320)),
        named("attend_180x320_bf16", _attn("attend", "bf16", 180, 320)),
        # the larger model on the same map: 192 channels, windows of 48x48
        named("attend_180x320_c192_w48_bf16", _attn("attend", "bf16", 180, 320, heads=6, d=32, win=(48, 48))),
        # photographs padded to one size, windows that do not divide it, shared key and value heads, one empty image
        named("attend_3x339x511_w13_bf16", _attn("attend", "bf16", 339, 511, N=3, heads=6, kv_heads=2, d=8, win=(13, 13), masked=True)),
        # whole rows as windows: long sequences, with buckets that widen with the distance
        named("attend_rows_4x2039_f32", _attn("attend", "f32", 4, 2039, N=2, heads=4, kv_heads=2, d=32, win=(1, 2048), edges=15)),
        # training on a batch of crops: the forward and all gradients, bf16 activations
        named("train_64x64x64_bf16", _attn("train", "bf16", 64, 64, N=64)),
        # the batch that falls to one of several workers, fp32, smaller windows
        named("train_8x64x64_w16_f32", _attn("train", "f32", 64, 64, N=8, win=(16, 16))),
        # crops padded to one size, windows that do not divide them, shared heads, buckets
        named("train_5x50x61_w20_f32", _attn("train", "f32", 50, 61, N=5, heads=6, kv_heads=3, d=24, win=(20, 20), edges=9, masked=True)),
        # the optimiser on the network's own few hundred tensors, most of them small: latency
        named("adamw_c64_f32", _adamw("f32", "f32", 5, 5, 64, 128)),
        # the larger model's parameters, states in 8 bits
        named("adamw_c192_8bit", _adamw("8bit", "f32", 8, 5, 192, 384)),
        # a model of a hundred million parameters, 8-bit states and bf16 gradients
        named("adamw_wide_8bit_bf16", _adamw("8bit", "bf16", 12, 6, 640, 1280)),
    ]


def _pairs(c):
    """Queries times keys over the windows of one image's one head, pixels that a mask hides included."""
    rows = sum(min(c["win_h"], c["H"] - y) ** 2 for y in range(0, c["H"], c["win_h"]))
    cols = sum(min(c["win_w"], c["W"] - x) ** 2 for x in range(0, c["W"], c["win_w"]))
    return rows * cols


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "train", "adamw"))
    if kind == "adamw":
        return _adamw(rng.choice(("f32", "8bit")), rng.choice(("f32", "bf16")), rng.randint(1, 8), rng.randint(1, 6),
                      2 * _log(rng, 16, 160), _log(rng, 16, 500))
    dtype = rng.choice(("f32", "bf16"))
    while True:
        heads = rng.choice((1, 2, 3, 4, 6, 8))
        kv = rng.choice([h for h in range(1, heads + 1) if heads % h == 0])
        if rng.random() < 0.25:  # rows as sequences
            H, W, win = rng.randint(1, 4), _log(rng, 1, 4096), (1, _log(rng, 16, 4096))
        else:
            H, W, win = _log(rng, 8, 360), _log(rng, 8, 640), (_log(rng, 2, 48), _log(rng, 2, 48))
        c = _attn(kind, dtype, H, W, N=_log(rng, 1, 32), heads=heads, kv_heads=kv, d=rng.choice((8, 12, 16, 24, 32, 33, 48, 64)), win=win,
                  edges=rng.choice((0, 0, 4, 9, 15)), masked=rng.random() < 0.4)
        # no more than the largest listed: pairs of tokens and heads, the plain form's memory and its many small windows
        cost = c["N"] * heads * _pairs(c)
        if cost * (c["d"] + 16) <= (3e9 if kind == "train" else 8e9) and c["N"] * heads * H * W * c["d"] <= 4e7:
            return c


def _edges(n, far):
    """n bucket edges: distances one by one at first, then wider and wider up to `far`."""
    out = [1]
    for i in range(1, n):
        out.append(max(out[-1] + 1, int(round((far / 2.0) ** (i / max(1, n - 1))))))
    return out


def _case_edges(c):
    return _edges(c["edges"], max(c["win_h"], c["win_w"])) if c["edges"] else None


def _sizes(c):
    """Element counts of the network's parameters: per module ConvFFN, estimator, fuse; per block attention's bias and
    projections; one shared large kernel."""
    C, Ch, h, Ca = c["channels"], c["hidden"], 8, max(1, c["channels"] // 4)
    module = [(Ch * C, 1), (Ch, 0), (Ch * 9, 1), (Ch, 0), (C * Ch, 1), (C, 0), (h * Ca, 1), (h, 0), (9 * Ca * h, 1), (9 * Ca, 0), (C * C, 1), (C, 0)]
    block = [(4 * 63 * 63, 0), (3 * C * C, 1), (C * C, 1), (C, 0), (C, 0)]
    return [(16 * 16 * 169, 1)] + (module * c["modules"] + block) * c["blocks"]


def _places(c):
    """(start, elements, decays) of every tensor in the flat buffers, starts a multiple of four elements, and the total."""
    at, out = 0, []
    for n, decays in _sizes(c):
        out.append((at, n, bool(decays)))
        at += (n + 3) // 4 * 4
    return out, at


HYPER = dict(lr=5e-4, beta1=0.9, beta2=0.9, eps=1e-8, weight_decay=1e-2, step=7, grad_scale=0.5)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)

    if c["kind"] == "adamw":
        places, total = _places(c)
        s = dict(case=c, places=places, total=total, done=0)
        s["p"] = normal(total, scale=0.05)
        s["g"] = normal(total, scale=1e-3, dtype=DTYPES[c["grads"]])
        m, v = normal(total, scale=1e-4), normal(total, scale=1e-4).square()
        # each tensor's blocks: (index of the block of every element) in the order of the tensors
        starts = torch.tensor([a for a, n, _ in places], device="cuda")
        counts = torch.tensor([n for a, n, _ in places], device="cuda")
        blocks = (counts + BLOCK - 1) // BLOCK
        first = torch.cumsum(blocks, 0) - blocks
        s["n_blocks"], s["first"], s["blocks"] = int(blocks.sum()), first.tolist(), blocks.tolist()
        which = torch.repeat_interleave(torch.arange(len(places), device="cuda"), (counts + 3) // 4 * 4)
        inside = torch.arange(total, device="cuda") - starts[which]
        s["block_of"] = torch.clamp(inside // BLOCK, max=blocks[which] - 1) + first[which]
        s["real"] = inside < counts[which]
        # the elements of each block, the place behind the last where a block has no more
        s["slots"] = torch.full((s["n_blocks"], BLOCK), total, device="cuda")
        s["slots"].view(-1)[(s["block_of"] * BLOCK + inside - (s["block_of"] - first[which]) * BLOCK)[s["real"]]] = torch.arange(total, device="cuda")[s["real"]]
        s["decay"] = torch.tensor([HYPER["weight_decay"] if d else 0.0 for _, _, d in places], device="cuda", dtype=torch.float64)[which]
        for name in ("p", "g"):
            s[name] = torch.where(s["real"], s[name], torch.zeros_like(s[name]))
        m, v = torch.where(s["real"], m, 0 * m), torch.where(s["real"], v, 0 * v)
        if c["states"] == "8bit":
            s["m"], s["m_scale"] = _held(s, m, False)
            s["v"], s["v_scale"] = _held(s, torch.sqrt(v), True)
        else:
            s["m"], s["v"] = m, v
        return s
    C, Ckv, dt = c["heads"] * c["d"], c["kv_heads"] * c["d"], DTYPES[c["dtype"]]
    N, H, W = c["N"], c["H"], c["W"]
    # one tensor with queries, keys and values, as the point-wise layer in front writes it
    qkv = normal(N, C + 2 * Ckv, H, W, dtype=dt)
    s = dict(case=c, mask=None, edges=_case_edges(c), scale=1.0 / math.sqrt(c["d"]))
    nb = [2 * c["edges"] + 1 if c["edges"] else 2 * w - 1 for w in (c["win_h"], c["win_w"])]
    s["bias"] = normal(c["heads"], *nb, scale=0.5)
    if c["masked"]:
        # pixels that an image of the batch has: its own height and width, some holes, and no pixel of the last image
        hw = torch.rand(N, 2, device="cuda", generator=g) * 0.7 + 0.3
        ok = (torch.arange(H, device="cuda")[None, :, None] < hw[:, 0, None, None] * H) & (torch.arange(W, device="cuda")[None, None, :] < hw[:, 1, None, None] * W)
        ok = ok & (torch.rand(N, H, W, device="cuda", generator=g) > 0.02)
        if N > 1:
            ok[-1] = False
        s["mask"] = ok.to(torch.uint8)
        qkv = torch.where(ok[:, None], qkv, torch.full_like(qkv, float("nan")))  # nobody has written there
    s["q"], s["k"], s["v"] = qkv[:, :C], qkv[:, C:C + Ckv], qkv[:, C + Ckv:]
    if c["kind"] == "train":
        s["grad_out"] = normal(N, C, H, W, dtype=dt)
    return s


def _held(s, x, up):
    """Values in 8 bits, a scale for each block; `up`: a value that is not zero does not become zero."""
    size = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    top = torch.nn.functional.pad(size, (0, 1))[s["slots"]].amax(1)
    full = top >= TINY
    scale = torch.where(full, top / CODE_MAX, torch.zeros_like(top))
    inverse = torch.where(full, CODE_MAX / top, torch.zeros_like(top))
    y = x * inverse[s["block_of"]]
    if up:
        y = torch.where((y > 0) & (y < 2.0 ** -9), torch.full_like(y, 2.0 ** -9), y)
    return y.to(torch.float8_e4m3fn), scale


def _adamw_plain(s):
    c, h = s["case"], HYPER
    s["done"] += 1
    t = h["step"] + s["done"]
    f = torch.float32
    at = s["block_of"]
    if c["states"] == "8bit":
        m = s["m"].to(f) * s["m_scale"][at]
        v = (s["v"].to(f) * s["v_scale"][at]).square()
    else:
        m, v = s["m"], s["v"]

    def const(x):
        return torch.tensor(x, dtype=torch.float64, device="cuda").to(f)

    g = s["g"].to(f) * const(h["grad_scale"])
    m = const(h["beta1"]) * m + const(1 - h["beta1"]) * g
    v = const(h["beta2"]) * v + const(1 - h["beta2"]) * (g * g)
    r = torch.sqrt(v)
    update = m / (r * const(1 / math.sqrt(1 - h["beta2"] ** t)) + const(h["eps"]))
    p = s["p"] * (1.0 - h["lr"] * s["decay"]).to(f) - const(h["lr"] / (1 - h["beta1"] ** t)) * update
    s["p"].copy_(p)
    if c["states"] == "8bit":
        for name, x, up in (("m", m, False), ("v", r, True)):
            codes, scale = _held(s, x, up)
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


def _adamw_own(s):
    from paper_2503_06671_amd import binding

    c, h = s["case"], HYPER
    opt = s.get("opt")
    if opt is None:  # the plan that a training program makes once
        def views(name, scales=False):
            if scales:
                return [s[name][b:b + n] for b, n in zip(s["first"], s["blocks"])]
            return [s[name][a:a + n] for a, n, _ in s["places"]]

        scales = dict(m_scale=views("m_scale", True), v_scale=views("v_scale", True)) if c["states"] == "8bit" else {}
        opt = s["opt"] = binding.AdamW(views("p"), views("g"), states=c["states"], m=views("m"), v=views("v"),
                                       weight_decay=[h["weight_decay"] if d else 0.0 for _, _, d in s["places"]], step=h["step"], **scales)
    opt.step(h["lr"], beta1=h["beta1"], beta2=h["beta2"], eps=h["eps"], grad_scale=h["grad_scale"])


def _adamw_outputs(s):
    names = ("p", "m", "v", "m_scale", "v_scale") if s["case"]["states"] == "8bit" else ("p", "m", "v")
    return {n: s[n] for n in names}


def _grid(c):
    """Windows down and across."""
    return -(-c["H"] // c["win_h"]), -(-c["W"] // c["win_w"])


def _windows(c, x, heads):
    """[N, heads d, H, W] -> [N gy gx, heads, tokens, d], pixels beyond the map as zeros."""
    gy, gx = _grid(c)
    x = torch.nn.functional.pad(x, (0, gx * c["win_w"] - c["W"], 0, gy * c["win_h"] - c["H"]))
    x = x.reshape(c["N"], heads, -1, gy, c["win_h"], gx, c["win_w"]).permute(0, 3, 5, 1, 4, 6, 2)
    return x.reshape(c["N"] * gy * gx, heads, c["win_h"] * c["win_w"], -1)


def _map(c, x):
    """The way back: [N gy gx, heads, tokens, d] -> [N, heads d, H, W]."""
    gy, gx = _grid(c)
    x = x.reshape(c["N"], gy, gx, x.shape[1], c["win_h"], c["win_w"], -1).permute(0, 3, 6, 1, 4, 2, 5)
    return x.reshape(c["N"], x.shape[1] * x.shape[2], gy * c["win_h"], gx * c["win_w"])[:, :, :c["H"], :c["W"]]


def _bucket(offsets, edges):
    """The bucket of offsets along one axis, zero for the most negative."""
    if edges is None:
        return offsets - offsets.min()
    e = torch.tensor(edges, device=offsets.device)
    return len(edges) + torch.sign(offsets) * torch.searchsorted(e, offsets.abs().contiguous(), right=True)


def _places_in_table(c, edges, columns):
    """The table's element that holds the bias of each (query, key) of a window."""
    y = torch.arange(c["win_h"], device="cuda").repeat_interleave(c["win_w"])
    x = torch.arange(c["win_w"], device="cuda").repeat(c["win_h"])
    return _bucket(y[None, :] - y[:, None], edges) * columns + _bucket(x[None, :] - x[:, None], edges)


def _attention_plain(s):
    c, f = s["case"], torch.float32
    group = c["heads"] // c["kv_heads"]
    here = torch.ones(c["N"], 1, c["H"], c["W"], device="cuda", dtype=torch.bool) if s["mask"] is None else s["mask"][:, None] != 0

    def split(x, heads):
        return _windows(c, torch.where(here, x.to(f), torch.zeros((), device="cuda")), heads)

    q = split(s["q"], c["heads"])
    k, v = (split(s[n], c["kv_heads"]).repeat_interleave(group, 1) for n in ("k", "v"))
    at = _places_in_table(c, s["edges"], s["bias"].shape[2])
    seen = _windows(c, here.to(f), 1)[:, :, :, 0] != 0  # [windows, 1, tokens]
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"] + s["bias"].reshape(c["heads"], -1)[:, at]
    score = torch.where(seen[:, :, None, :], score, torch.full((), -math.inf, device="cuda"))
    top = torch.amax(score, -1, keepdim=True)
    e = torch.exp(score - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    del score
    total = e.sum(-1, keepdim=True)
    p = torch.where(seen[:, :, :, None] & (total > 0), e / total, torch.zeros((), device="cuda"))
    del e
    o = torch.matmul(p, v)
    dt = s["q"].dtype
    out = {"out": _map(c, o).to(dt)}
    if c["kind"] == "attend":
        return out
    do = split(s["grad_out"], c["heads"])
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = p * (dp - (do * o).sum(-1, keepdim=True))
    del dp
    shared = (-1, c["kv_heads"], group, q.shape[2], q.shape[3])
    out["grad_q"] = _map(c, torch.matmul(ds, k) * s["scale"]).to(dt)
    out["grad_k"] = _map(c, (torch.matmul(ds.transpose(2, 3).contiguous(), q) * s["scale"]).reshape(shared).sum(2)).to(dt)
    out["grad_v"] = _map(c, torch.matmul(p.transpose(2, 3).contiguous(), do).reshape(shared).sum(2)).to(dt)
    # first the sums of equal offsets, then those of a bucket's offsets
    per_offset = torch.zeros(c["heads"], (2 * c["win_h"] - 1) * (2 * c["win_w"] - 1), device="cuda", dtype=torch.float64)
    offsets = _places_in_table(c, None, 2 * c["win_w"] - 1)
    per_offset.index_add_(1, offsets.reshape(-1), ds.double().sum(0).reshape(c["heads"], -1))
    if s["edges"] is not None:
        y, x = (_bucket(torch.arange(-w + 1, w, device="cuda"), s["edges"]) for w in (c["win_h"], c["win_w"]))
        at = (y[:, None] * s["bias"].shape[2] + x[None, :]).reshape(-1)
        per_offset = torch.zeros_like(s["bias"], dtype=torch.float64).reshape(c["heads"], -1).index_add_(1, at, per_offset)
    out["grad_bias"] = per_offset.reshape(s["bias"].shape).to(f)
    return out


def _attention_own(s):
    from paper_2503_06671_amd import binding

    c = s["case"]
    window = (c["win_h"], c["win_w"])
    kw = dict(bias=s["bias"], edges=s["edges"], mask=s["mask"], scale=s["scale"], kv_heads=c["kv_heads"])
    if c["kind"] == "attend":
        return {"out": binding.window_attention_forward(s["q"], s["k"], s["v"], c["heads"], window, **kw)}
    if "ws" not in s:  # the buffers that a training program keeps
        s["saved"] = binding.new_window_attention_saved(c["N"], c["heads"], c["d"], c["H"], c["W"], s["q"].dtype)
        s["ws"] = binding.new_window_attention_backward_workspace(c["N"], c["heads"], c["d"], c["H"], c["W"], window)
    out = binding.window_attention_forward(s["q"], s["k"], s["v"], c["heads"], window, saved=s["saved"], **kw)
    grads = binding.window_attention_backward(s["q"], s["k"], s["v"], out, s["grad_out"], s["saved"], c["heads"], window, s["ws"], **kw)
    return {"out": out, **{n: grads[n] for n in ("grad_q", "grad_k", "grad_v", "grad_bias")}}


def run(state):
    if state["case"]["kind"] == "adamw":
        (_adamw_own if own else _adamw_plain)(state)
        return _adamw_outputs(state)
    return (_attention_own if own else _attention_plain)(state)


def work(case):
    c = case
    if c["kind"] == "adamw":
        n = sum(k for k, _ in _sizes(c))
        state = 4 if c["states"] == "8bit" else 16  # both states, read and written
        scales = 16.0 * sum(-(-k // BLOCK) for k, _ in _sizes(c)) if c["states"] == "8bit" else 0.0
        return {"bytes": n * (8.0 + (4 if c["grads"] == "f32" else 2) + state) + scales, "flops": 16.0 * n}
    size = 4 if c["dtype"] == "f32" else 2
    pixels = c["N"] * c["H"] * c["W"]
    C, Ckv = c["heads"] * c["d"], c["kv_heads"] * c["d"]
    nb = [2 * c["edges"] + 1 if c["edges"] else 2 * w - 1 for w in (c["win_h"], c["win_w"])]
    table = 4.0 * c["heads"] * nb[0] * nb[1]
    mask = pixels if c["masked"] else 0
    products = c["N"] * c["heads"] * float(_pairs(c)) * c["d"]  # of two values each, a score or an output's share
    if c["kind"] == "attend":
        return {"bytes": pixels * size * 2.0 * (C + Ckv) + table + mask, "flops": 4.0 * products}
    return {"bytes": pixels * size * (4.0 * C + 4.0 * Ckv) + 2 * table + mask, "flops": 14.0 * products}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_adamw(s) if case["kind"] == "adamw" else _exact_attention(s)


def _exact_adamw(s):
    h, t = HYPER, HYPER["step"] + 1
    out = {n: torch.zeros_like(x, dtype=torch.float64) for n, x in _adamw_outputs(s).items()}
    eight = s["case"]["states"] == "8bit"
    for i, (a, n, decays) in enumerate(s["places"]):
        at, b = slice(a, a + n), slice(s["first"][i], s["first"][i] + s["blocks"][i])
        p, g, m, v = (s[k][at].double() for k in ("p", "g", "m", "v"))
        if eight:
            each = torch.arange(n, device="cuda") // BLOCK
            m, v = m * s["m_scale"][b].double()[each], (v * s["v_scale"][b].double()[each]) ** 2
        g = g * h["grad_scale"]
        m = h["beta1"] * m + (1 - h["beta1"]) * g
        v = h["beta2"] * v + (1 - h["beta2"]) * g ** 2
        hat = m / (1 - h["beta1"] ** t) / ((v / (1 - h["beta2"] ** t)).sqrt() + h["eps"])
        out["p"][at] = p * (1 - h["lr"] * (h["weight_decay"] if decays else 0.0)) - h["lr"] * hat
        if eight:
            for name, x in (("m", m), ("v", v.sqrt())):
                pad = torch.nn.functional.pad(x.abs(), (0, s["blocks"][i] * BLOCK - n)).reshape(-1, BLOCK)
                scale = pad.amax(1) / CODE_MAX
                scale = torch.where(scale * CODE_MAX >= TINY, scale, torch.zeros_like(scale))
                out[name + "_scale"][b] = scale
                y = torch.where(scale[each] > 0, x / scale[each], torch.zeros_like(x))
                # to the nearest of the format's values: three bits behind the leading one, steps of 2^-9 below 2^-6
                step = torch.exp2(torch.floor(torch.log2(torch.clamp(y.abs(), min=2.0 ** -6))) - 3)
                q = torch.round(y / step) * step
                out[name][at] = torch.where((q == 0) & (y > 0) & (name == "v"), torch.full_like(q, 2.0 ** -9), q)
        else:
            out["m"][at], out["v"][at] = m, v
    return out


def _exact_attention(s):
    c, D = s["case"], torch.float64
    train = c["kind"] == "train"
    group, d, scale = c["heads"] // c["kv_heads"], c["d"], s["scale"]
    N, H, W = c["N"], c["H"], c["W"]
    if -(-H // c["win_h"]) * -(-W // c["win_w"]) > 4000:
        return None  # too many windows to go through one by one
    table = s["bias"].double()
    ok = torch.ones(N, H, W, device="cuda", dtype=torch.bool) if s["mask"] is None else s["mask"].bool()
    out = {"out": torch.zeros(N, c["heads"], d, H, W, device="cuda", dtype=D)}
    if train:
        out["grad_q"] = torch.zeros_like(out["out"])
        out["grad_k"] = torch.zeros(N, c["kv_heads"], d, H, W, device="cuda", dtype=D)
        out["grad_v"] = torch.zeros_like(out["grad_k"])
        out["grad_bias"] = torch.zeros_like(table)

    def bucket(offset, full):
        if s["edges"] is None:
            return offset + full - 1
        return len(s["edges"]) + (1 if offset > 0 else -1) * sum(e <= abs(offset) for e in s["edges"])

    def axis(n, full):
        by = torch.tensor([bucket(o, full) for o in range(-n + 1, n)], device="cuda")
        i = torch.arange(n, device="cuda")
        return by[i[None, :] - i[:, None] + n - 1]  # [query, key]

    for y0 in range(0, H, c["win_h"]):
        for x0 in range(0, W, c["win_w"]):
            h, w = min(c["win_h"], H - y0), min(c["win_w"], W - x0)
            at = (slice(None), slice(None), slice(None), slice(y0, y0 + h), slice(x0, x0 + w))
            here = ok[:, y0:y0 + h, x0:x0 + w].reshape(N, 1, h * w)

            def tokens(name, heads):
                x = s[name].reshape(N, heads, d, H, W)[at].reshape(N, heads, d, h * w).double()
                return torch.where(here[:, :, None], x, torch.zeros_like(x))

            q = tokens("q", c["heads"]).reshape(N, c["kv_heads"], group, d, h * w)
            k, v = (tokens(n, c["kv_heads"])[:, :, None] for n in ("k", "v"))
            by, bx = axis(h, c["win_h"]), axis(w, c["win_w"])
            spot = (by[:, None, :, None] * table.shape[2] + bx[None, :, None, :]).reshape(h * w, h * w)
            bias = table.flatten(1)[:, spot].reshape(c["kv_heads"], group, h * w, h * w)
            z = torch.matmul(q.transpose(3, 4).contiguous(), k.expand(-1, -1, group, -1, -1).contiguous()) * scale + bias
            pair = here[:, :, None, :, None] & here[:, :, None, None, :]
            z = z.masked_fill(~pair, -math.inf)
            p = torch.nan_to_num(torch.softmax(z, -1), nan=0.0)
            del z
            o = torch.matmul(v.expand(-1, -1, group, -1, -1).contiguous(), p.transpose(3, 4).contiguous())
            out["out"][at] = o.reshape(N, c["heads"], d, h, w)
            if not train:
                continue
            do = tokens("grad_out", c["heads"]).reshape(N, c["kv_heads"], group, d, h * w)
            dp = torch.matmul(do.transpose(3, 4).contiguous(), v.expand(-1, -1, group, -1, -1).contiguous())
            ds = p * (dp - (p * dp).sum(-1, keepdim=True))
            out["grad_q"][at] = (torch.matmul(k.expand(-1, -1, group, -1, -1).contiguous(), ds.transpose(3, 4).contiguous()) * scale).reshape(N, c["heads"], d, h, w)
            out["grad_k"][at] = (torch.matmul(q, ds).sum(2) * scale).reshape(N, c["kv_heads"], d, h, w)
            out["grad_v"][at] = torch.matmul(do, p).sum(2).reshape(N, c["kv_heads"], d, h, w)
            out["grad_bias"].reshape(c["heads"], -1).index_add_(1, spot.reshape(-1), ds.sum(0).reshape(c["heads"], -1))
    return {n: x if n == "grad_bias" else x.reshape(N, -1, H, W) for n, x in out.items()}
