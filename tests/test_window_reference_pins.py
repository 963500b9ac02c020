"""The window attention reference against things it does not share: torch's own softmax attention, differences, closed forms."""
import math

import pytest
import torch

from tests import window_reference as ref

D = torch.float64


def inputs(seed, N, H, W, heads, kv, d, buckets):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(N, heads * d, H, W, generator=g, dtype=D)
    k, v = (torch.randn(N, kv * d, H, W, generator=g, dtype=D) for _ in range(2))
    return q, k, v, torch.randn(heads, *buckets, generator=g, dtype=D), torch.randn(N, heads * d, H, W, generator=g, dtype=D)


def test_one_window_is_plain_attention():
    q, k, v, bias, _ = inputs(1, 2, 3, 5, 2, 2, 4, (5, 9))
    r = ref.attention(q, k, v, 2, (3, 5), bias=bias)
    b, _ = ref.bias_of_window(bias, 3, 5, (3, 5), None)
    x = [t.reshape(2, 2, 4, 15).transpose(2, 3) for t in (q, k, v)]
    want = torch.nn.functional.scaled_dot_product_attention(*x, attn_mask=b[None].expand(2, -1, -1, -1))
    assert torch.allclose(r["out"].reshape(2, 2, 4, 15).transpose(2, 3), want, rtol=1e-12, atol=1e-12)


def test_buckets():
    assert [ref.bucket(o, 4, None) for o in (-3, 0, 3)] == [0, 3, 6]
    assert [ref.bucket(o, 99, [1, 2, 5]) for o in (-9, -5, -4, -2, -1, 0, 1, 2, 4, 5, 98)] == [0, 0, 1, 1, 2, 3, 4, 5, 5, 6, 6]


@pytest.mark.parametrize("edges,window", [(None, (2, 3)), ([1, 2], (3, 2)), (None, (1, 4))])
def test_gradients_against_differences(edges, window):
    n = 5 if edges else None
    buckets = (n, n) if edges else (2 * window[0] - 1, 2 * window[1] - 1)
    q, k, v, bias, go = inputs(3, 1, 4, 5, 2, 1, 3, buckets)
    mask = torch.ones(1, 4, 5, dtype=torch.uint8)
    mask[0, 1, 2] = mask[0, 3, 4] = 0
    kw = dict(edges=edges, mask=mask, kv_heads=1)
    r = ref.attention(q, k, v, 2, window, bias=bias, grad_out=go, **kw)
    live = go * mask[:, None]  # masked pixels have no result

    def loss(**change):
        x = dict(q=q, k=k, v=v, bias=bias)
        x.update(change)
        return (ref.attention(x["q"], x["k"], x["v"], 2, window, bias=x["bias"], **kw)["out"] * live).sum().item()

    eps = 1e-5
    for name, x in (("q", q), ("k", k), ("v", v), ("bias", bias)):
        flat = r["grad_" + name].reshape(-1)
        for i in range(0, x.numel(), max(1, x.numel() // 15)):
            a, b = x.clone(), x.clone()
            a.view(-1)[i] += eps
            b.view(-1)[i] -= eps
            assert abs((loss(**{name: a}) - loss(**{name: b})) / (2 * eps) - flat[i].item()) < 1e-8, (name, i)


def test_empty_rows_and_hidden_buckets():
    q, k, v, bias, go = inputs(4, 1, 2, 2, 1, 1, 2, (3, 3))
    r = ref.attention(q, k, v, 1, (2, 2), bias=torch.full_like(bias, -math.inf), grad_out=go)
    assert all((r[n] == 0).all() for n in ("out", "grad_q", "grad_k", "grad_v", "grad_bias"))
    only_self = torch.full_like(bias, -math.inf)
    only_self[0, 1, 1] = 0.3
    assert torch.equal(ref.attention(q, k, v, 1, (2, 2), bias=only_self)["out"], v)


def test_adamw_against_torch():
    g = torch.Generator().manual_seed(5)
    p = torch.randn(1000, generator=g)
    w = torch.nn.Parameter(p.to(D).clone())
    opt = torch.optim.AdamW([w], lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    m, v = torch.zeros(1000), torch.zeros(1000)
    for t in range(1, 6):
        grad = torch.randn(1000, generator=g)
        w.grad = grad.to(D)
        opt.step()
        p, m, v, _, _ = ref.adamw(p, grad, m, v, t, 1e-2, 0.9, 0.95, 1e-8, 0.1, 1.0)
        # five steps of a dozen roundings each, of values up to 4
        assert (p.to(D) - w.detach()).abs().max() < 5 * 12 * 4 * 2.0 ** -24


def test_states_in_8_bits():
    g = torch.Generator().manual_seed(6)
    x = torch.randn(700, generator=g) * torch.exp(4 * torch.randn(700, generator=g))
    codes, scale = ref.held(x, False)
    back = codes.to(torch.float32) * scale.repeat_interleave(256)[:700]
    # half a step of the format (2^-4 of a value; 2^-10 below its smallest normal one, 2^-6) and three fp32 roundings
    assert ((back - x).abs() <= (2.0 ** -4 * x.abs()).clamp(min=0) * (1 + 1e-6) + 2.0 ** -10 * scale.repeat_interleave(256)[:700]).all()
    codes, scale = ref.held(x.abs(), True)
    assert (codes.to(torch.float32) > 0).all()
    assert ref.held(torch.full((3,), 1e-32), True)[1].item() == 0
