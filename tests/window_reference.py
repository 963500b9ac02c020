"""Window attention and its gradients in float64, window by window and head by head from the definition, with the sums of
magnitudes that bound what rounding can do; the AdamW step with every fp32 operation by itself.  CPU only, shares no code with the GPU path."""
import math

import torch

D = torch.float64


def bucket(o, full, edges):
    if edges is None:
        return o + full - 1
    return len(edges) + (o > 0) * sum(e <= o for e in edges) - (o < 0) * sum(e <= -o for e in edges)


def bias_of_window(table, h, w, window, edges):
    """[heads, h w, h w] and the bucket of each pair."""
    by = torch.tensor([[bucket(kj - qi, window[0], edges) for kj in range(h)] for qi in range(h)])
    bx = torch.tensor([[bucket(kj - qi, window[1], edges) for kj in range(w)] for qi in range(w)])
    at = (by[:, None, :, None] * table.shape[2] + bx[None, :, None, :]).reshape(h * w, h * w)
    return table.reshape(table.shape[0], -1)[:, at], at


def attention(q, k, v, heads, window, bias=None, edges=None, mask=None, scale=None, kv_heads=None, grad_out=None):
    """Tensors as the binding takes them, on the CPU.  Returns a dict of float64 results and, under "..._abs", of the sums of the
    magnitudes of their terms."""
    kv_heads = kv_heads or heads
    N, C, H, W = q.shape
    d = C // heads
    scale = d ** -0.5 if scale is None else scale
    ok = torch.ones(N, H, W, dtype=torch.bool) if mask is None else mask.bool()

    def clean(x):
        return torch.where(ok[:, None], x.to(D), torch.zeros((), dtype=D))

    q, k, v = clean(q), clean(k), clean(v)
    names = ["out"] + (["grad_q", "grad_k", "grad_v"] if grad_out is not None else [])
    r = {n: torch.zeros_like(q if n in ("out", "grad_q") else k) for n in names}
    r.update({n + "_abs": torch.zeros_like(r[n]) for n in names})
    r["score_abs"] = 0.0
    if grad_out is not None:
        go = clean(grad_out)
        table = torch.zeros(heads, 1, 1, dtype=D) if bias is None else torch.zeros_like(bias, dtype=D)
        r["grad_bias"], r["grad_bias_abs"] = table, table.clone()
    wh, ww = min(window[0], H), min(window[1], W)
    for n in range(N):
        for y0 in range(0, H, wh):
            for x0 in range(0, W, ww):
                h, w = min(wh, H - y0), min(ww, W - x0)
                L = h * w
                seen = ok[n, y0:y0 + h, x0:x0 + w].reshape(L)
                pair = seen[:, None] & seen[None, :]
                if bias is not None:
                    b, at = bias_of_window(bias.to(D), h, w, window, edges)
                for hd in range(heads):
                    kvh = hd // (heads // kv_heads)

                    def tokens(x, head):
                        return x[n, head * d:(head + 1) * d, y0:y0 + h, x0:x0 + w].reshape(d, L).T

                    def put(name, head, x):
                        r[name][n, head * d:(head + 1) * d, y0:y0 + h, x0:x0 + w] += x.T.reshape(d, h, w)

                    Q, K, V = tokens(q, hd), tokens(k, kvh), tokens(v, kvh)
                    s = Q @ K.T * scale + (b[hd] if bias is not None else 0.0)
                    sa = Q.abs() @ K.abs().T * scale + (torch.where(torch.isfinite(b[hd]), b[hd].abs(), torch.zeros((), dtype=D)) if bias is not None else 0.0)
                    if pair.any():
                        r["score_abs"] = max(r["score_abs"], float(torch.where(pair, sa, torch.zeros((), dtype=D)).max()))
                    s = torch.where(pair, s, torch.full((), -math.inf, dtype=D))
                    top = s.max(1, keepdim=True).values
                    e = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
                    total = e.sum(1, keepdim=True)
                    p = torch.where(total > 0, e / torch.where(total > 0, total, torch.ones_like(total)), torch.zeros_like(e))
                    put("out", hd, p @ V)
                    put("out_abs", hd, p @ V.abs())
                    if grad_out is None:
                        continue
                    G = tokens(go, hd)
                    dp = G @ V.T
                    delta = (p * dp).sum(1, keepdim=True)
                    ds = p * (dp - delta)
                    da = p * (G.abs() @ V.abs().T)
                    da = da + p * da.sum(1, keepdim=True)
                    put("grad_q", hd, ds @ K * scale)
                    put("grad_q_abs", hd, da @ K.abs() * scale)
                    put("grad_k", kvh, ds.T @ Q * scale)
                    put("grad_k_abs", kvh, da.T @ Q.abs() * scale)
                    put("grad_v", kvh, p.T @ G)
                    put("grad_v_abs", kvh, p.T @ G.abs())
                    if bias is not None:
                        r["grad_bias"][hd].view(-1).index_add_(0, at.reshape(-1), ds.reshape(-1))
                        r["grad_bias_abs"][hd].view(-1).index_add_(0, at.reshape(-1), da.reshape(-1))
    return r


def tolerance(r, name, dtype, d, tokens):
    """What fp32 arithmetic and the stated roundings can make of result `name`, element by element.

    fp32 part, in units of 2^-24: a score is off by at most d + 8 roundings of its terms' magnitudes S (products of three-term operands leave out
    up to eight units of each product, one on average); the exponent's argument by two roundings more of at most 2 S; an error of a score is a relative one of its
    exponential, counted twice (numerator and sum).  The sums over the keys and the queries, of 32 at a time, take at most tokens / 8 + 64
    roundings of the sum of magnitudes, and the gradients' delta as many again.
    bf16: results but the bias' gradient are rounded (half a step: 2^-8 of them); in the products the p of the result and of v's gradient are
    rounded once (2^-8 of each term), the ds of the gradients of q and k twice (2^-16)."""
    u = 2.0 ** -24
    rel = u * (2 * (2 * d + 16) * (r["score_abs"] + 1) + 2 * (tokens / 8 + 64))
    tol = rel * r[name + "_abs"]
    if dtype == torch.bfloat16 and name != "grad_bias":
        tol = tol + 2.0 ** (-8 if name in ("out", "grad_v") else -16) * r[name + "_abs"] + 2.0 ** -8 * r[name].abs()
    elif name != "grad_bias":
        tol = tol + u * r[name].abs()
    return tol + 1e-30


def assert_close(got, r, name, dtype, d, tokens, what=""):
    g = got.detach().cpu().to(D)
    tol = tolerance(r, name, dtype, d, tokens)
    off = (g - r[name]).abs()
    assert torch.isfinite(g).all(), (what, name, "not finite")
    worst = (off / tol).max().item()
    assert worst <= 1.0, (what, name, worst, off.max().item())
    norm = r[name].norm().item()
    # The library's own bars, over the norm - not where scores are so large that half a unit of their last place, counted in numerator and
    # sum, comes to the fp32 bar by itself (2 * 64 * 2^-24 = 8e-6; at 1000 it is 1.2e-4 of an exponential).
    if norm > 0 and r["score_abs"] <= 64:
        bar = 2e-2 if dtype == torch.bfloat16 and name != "grad_bias" else 1e-5
        # (where the terms cancel, what is left is small beside what rounding does to them)
        cancels = r[name + "_abs"].norm().item() / norm
        assert off.norm().item() <= bar * norm * max(1.0, cancels / 8), (what, name, off.norm().item() / norm, cancels)
    return worst


# ---- AdamW ----

BLOCK, CODE_MAX, TINY = 256, 448.0, 2.0 ** -100


def f32(x):
    return torch.tensor(x, dtype=D).to(torch.float32)


def held(x, up):
    """(codes, scales) of one tensor's state in 8 bits."""
    n = x.numel()
    blocks = -(-n // BLOCK)
    size = torch.where(torch.isfinite(x), x.abs(), torch.zeros(()))
    top = torch.nn.functional.pad(size, (0, blocks * BLOCK - n)).reshape(blocks, BLOCK).amax(1)
    full = top >= TINY
    scale = torch.where(full, top * f32(1 / CODE_MAX), torch.zeros(()))
    y = x * torch.where(full, CODE_MAX * (torch.ones(()) / top), torch.zeros(())).repeat_interleave(BLOCK)[:n]
    y = torch.where(torch.isfinite(y), y, torch.full((), math.nan))
    if up:
        y = torch.where((y > 0) & (y < 2.0 ** -9), torch.full((), 2.0 ** -9), y)
    return y.to(torch.float8_e4m3fn), scale


def adamw(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay, grad_scale, scales=None):
    """One step of one tensor; m and v are float32 tensors, or codes with scales = (m_scale, v_scale).  Returns p, m, v, m_scale, v_scale."""
    if scales is not None:
        each = torch.arange(p.numel()) // BLOCK
        m = m.to(torch.float32) * scales[0][each]
        root = v.to(torch.float32) * scales[1][each]
        v = root * root
    g = g.to(torch.float32) * f32(grad_scale)
    m = f32(beta1) * m + f32(1.0 - beta1) * g
    v = f32(beta2) * v + f32(1.0 - beta2) * (g * g)
    root = torch.sqrt(v.to(D)).to(torch.float32)  # (to the nearest; torch.sqrt on the CPU misses it by a unit in places)
    update = m / (root * f32(1.0 / math.sqrt(1.0 - beta2 ** t)) + f32(eps))
    # (the library takes a weight decay as float)
    p = p * f32(1.0 - lr * float(f32(weight_decay))) - f32(lr / (1.0 - beta1 ** t)) * update
    if scales is None:
        return p, m, v, None, None
    mc, ms = held(m, False)
    vc, vs = held(root, True)
    return p, mc, vc, ms, vs
