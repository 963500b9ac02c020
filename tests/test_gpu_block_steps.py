"""A whole block as a network runs and trains it, all by the library's calls:

    y   = x + dropout( proj( window attention( qkv( norm(x) ) ) ) )
    out = y + second( gelu( first( norm(y) ) ) ) + stochastic depth

with all gradients and the AdamW step, against float64 autograd; the same from a graph; two blocks on two streams at once."""
import math

import pytest
import torch

from paper_2503_06671_amd import binding
from tests import block_reference as ref
from tests import window_reference

pytestmark = pytest.mark.gpu

N, HEADS, D, H, W, WINDOW, HIDDEN = 3, 2, 12, 13, 18, (6, 7), 40
C = HEADS * D
P, DEPTH, SEED, EPS = 0.2, 0.3, 1234567, 1e-5
HYPER = dict(beta1=0.8, beta2=0.9, eps=1.0, grad_scale=1.0 / (N * H * W))
LR, STEPS = 0.05, 3
NAMES = ("n1w", "n1b", "qkv", "bias", "proj", "projb", "n2w", "n2b", "first", "firstb", "second", "secondb")


def parameters(seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, scale=1.0: scale * torch.randn(*s, generator=g)  # noqa: E731
    return dict(n1w=1 + r(C, scale=0.2), n1b=r(C, scale=0.2), qkv=r(3 * C, C, scale=C ** -0.5), bias=r(HEADS, 11, 13, scale=0.5), proj=r(C, C, scale=C ** -0.5),
                projb=r(C, scale=0.1), n2w=1 + r(C, scale=0.2), n2b=r(C, scale=0.2), first=r(HIDDEN, C, scale=C ** -0.5), firstb=r(HIDDEN, scale=0.1),
                second=r(C, HIDDEN, scale=HIDDEN ** -0.5), secondb=r(C, scale=0.1))


def data(seed=1):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(N, C, H, W, generator=g), torch.randn(N, C, H, W, generator=g)


class Block:
    """One block with the buffers that a training program keeps."""

    def __init__(self, dtype=torch.float32):
        self.p = {n: t.cuda() for n, t in parameters().items()}
        self.g = {n: torch.empty_like(t) for n, t in self.p.items()}
        self.x, self.target = (t.cuda().to(dtype) for t in data())
        new = lambda c: torch.empty(N, c, H, W, device="cuda", dtype=dtype)  # noqa: E731
        self.n1, self.qkv, self.att, self.branch, self.y, self.n2, self.hidden, self.ffn, self.out = map(new, (C, 3 * C, C, C, C, C, HIDDEN, C, C))
        self.grad_out, self.g_ffn, self.g_hidden, self.g_n2, self.g_y, self.g_branch, self.g_att, self.g_qkv, self.g_n1, self.grad_x = \
            map(new, (C, C, HIDDEN, C, C, C, C, 3 * C, C, C))
        self.s1, self.s2 = (binding.new_layernorm_saved(N, H, W) for _ in range(2))
        self.nws = binding.new_layernorm_backward_workspace(N, C, H, W)
        self.saved = binding.new_window_attention_saved(N, HEADS, D, H, W, dtype)
        self.aws = binding.new_window_attention_backward_workspace(N, HEADS, D, H, W, WINDOW)
        self.pws = {n: binding.new_pointwise_backward_workspace(N, k, m, H, W, dtype, act=a)
                    for n, k, m, a in (("qkv", C, 3 * C, "none"), ("proj", C, C, "none"), ("first", C, HIDDEN, "gelu"), ("second", HIDDEN, C, "none"))}
        self.count = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.opt = binding.AdamW(list(self.p.values()), list(self.g.values()))

    def forward(self):
        p = self.p
        binding.layernorm_forward(self.x, p["n1w"], p["n1b"], EPS, out=self.n1, saved=self.s1)
        binding.pointwise_forward(self.n1, p["qkv"], out=self.qkv)
        q, k, v = self.qkv[:, :C], self.qkv[:, C:2 * C], self.qkv[:, 2 * C:]
        binding.window_attention_forward(q, k, v, HEADS, WINDOW, bias=p["bias"], out=self.att, saved=self.saved)
        binding.pointwise_forward(self.att, p["proj"], p["projb"], out=self.branch)
        binding.dropout_forward(self.branch, P, SEED, 0, offset_device=self.count, residual=self.x, out=self.y)
        binding.layernorm_forward(self.y, p["n2w"], p["n2b"], EPS, out=self.n2, saved=self.s2)
        binding.pointwise_forward(self.n2, p["first"], p["firstb"], "gelu", out=self.hidden)
        binding.pointwise_forward(self.hidden, p["second"], p["secondb"], out=self.ffn)
        binding.dropout_forward(self.ffn, DEPTH, SEED, 1, offset_device=self.count, over="image", residual=self.y, out=self.out)

    def backward(self):
        p, g = self.p, self.g
        binding.dropout_backward(self.grad_out, DEPTH, SEED, 1, offset_device=self.count, over="image", grad_x=self.g_ffn)
        binding.pointwise_backward(self.hidden, self.g_ffn, p["second"], self.pws["second"], p["secondb"],
                                   grads=dict(grad_x=self.g_hidden, grad_w=g["second"], grad_b=g["secondb"]))
        binding.pointwise_backward(self.n2, self.g_hidden, p["first"], self.pws["first"], p["firstb"], "gelu",
                                   grads=dict(grad_x=self.g_n2, grad_w=g["first"], grad_b=g["firstb"]))
        binding.layernorm_backward(self.y, self.g_n2, self.s2, self.nws, p["n2w"], p["n2b"], grad_skip=self.grad_out,
                                   grads=dict(grad_x=self.g_y, grad_weight=g["n2w"], grad_bias=g["n2b"]))
        binding.dropout_backward(self.g_y, P, SEED, 0, offset_device=self.count, grad_x=self.g_branch)
        binding.pointwise_backward(self.att, self.g_branch, p["proj"], self.pws["proj"], p["projb"],
                                   grads=dict(grad_x=self.g_att, grad_w=g["proj"], grad_b=g["projb"]))
        q, k, v = self.qkv[:, :C], self.qkv[:, C:2 * C], self.qkv[:, 2 * C:]
        binding.window_attention_backward(q, k, v, self.att, self.g_att, self.saved, HEADS, WINDOW, self.aws, bias=p["bias"],
                                          grads=dict(grad_q=self.g_qkv[:, :C], grad_k=self.g_qkv[:, C:2 * C], grad_v=self.g_qkv[:, 2 * C:], grad_bias=g["bias"]))
        binding.pointwise_backward(self.n1, self.g_qkv, p["qkv"], self.pws["qkv"], grads=dict(grad_x=self.g_n1, grad_w=g["qkv"]))
        binding.layernorm_backward(self.x, self.g_n1, self.s1, self.nws, p["n1w"], p["n1b"], grad_skip=self.g_y,
                                   grads=dict(grad_x=self.grad_x, grad_weight=g["n1w"], grad_bias=g["n1b"]))

    def step(self):
        self.forward()
        torch.sub(self.out, self.target, out=self.grad_out)
        self.backward()
        self.opt.step(LR, **HYPER)
        self.count.add_(2)


def kept(p, offset, over):
    return ref.kept((N, C, H, W), p, SEED, offset, over) * (65536 / (65536 - ref.dropped_of(p)))


def forward64(p, x, offset):
    """The block in float64, with autograd through everything."""
    def norm(t, w, b):
        return torch.nn.functional.layer_norm(t.permute(0, 2, 3, 1), (C,), w, b, EPS).permute(0, 3, 1, 2)

    def product(t, w, b=None):
        return torch.nn.functional.conv2d(t, w[:, :, None, None], b)

    qkv = product(norm(x, p["n1w"], p["n1b"]), p["qkv"])
    att = torch.zeros(N, C, H, W, dtype=torch.float64)
    pieces = []
    for y0 in range(0, H, WINDOW[0]):
        row = []
        for x0 in range(0, W, WINDOW[1]):
            t = qkv[:, :, y0:y0 + WINDOW[0], x0:x0 + WINDOW[1]]
            h, w = t.shape[2:]
            q, k, v = t.reshape(N, 3, HEADS, D, h * w).unbind(1)
            yy, xx = torch.arange(h).repeat_interleave(w), torch.arange(w).repeat(h)
            at = p["bias"][:, (yy[None] - yy[:, None] + WINDOW[0] - 1), (xx[None] - xx[:, None] + WINDOW[1] - 1)]
            s = torch.softmax(q.transpose(2, 3) @ k / math.sqrt(D) + at, -1)
            row.append((v @ s.transpose(2, 3)).reshape(N, C, h, w))
        pieces.append(torch.cat(row, 3))
    att = torch.cat(pieces, 2)
    y = x + kept(P, offset, "element") * product(att, p["proj"], p["projb"])
    hidden = torch.nn.functional.gelu(product(norm(y, p["n2w"], p["n2b"]), p["first"], p["firstb"]))
    return y + kept(DEPTH, offset + 1, "image") * product(hidden, p["second"], p["secondb"])


def test_the_reference_attends_as_the_other_one():
    # (the block above against the window attention tests' own float64 form)
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(N, C, H, W, generator=g) for _ in range(3))
    bias = torch.randn(HEADS, 11, 13, generator=g)
    want = window_reference.attention(q, k, v, HEADS, WINDOW, bias=bias)["out"]
    saved = binding.new_window_attention_saved(N, HEADS, D, H, W, torch.float32)
    got = binding.window_attention_forward(q.cuda(), k.cuda(), v.cuda(), HEADS, WINDOW, bias=bias.cuda(), saved=saved)
    assert (got.cpu() - want).abs().max() < 1e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gradients_of_the_block(dtype):
    block = Block(dtype)
    block.forward()
    torch.sub(block.out, block.target, out=block.grad_out)
    block.backward()
    p = {n: t.double().requires_grad_() for n, t in parameters().items()}
    x, target = (t.to(dtype).double() for t in data())
    x.requires_grad_()
    out = forward64(p, x, 0)
    (0.5 * (out - target).square().sum()).backward()
    # fp32: the library's bar for sums over all pixels, 5e-5 of the largest.  bf16: every tensor on the way is off by 2^-9 of itself on average (2^-8 at
    # most), in some twenty steps there and back, independent of one another: 20^(1/2) 2^-9 = 0.009, and of single elements up to four times that
    bar = 5e-5 if dtype == torch.float32 else 4 * 20 ** 0.5 * 2.0 ** -9
    for name, got, want in [("out", block.out, out.detach()), ("x", block.grad_x, x.grad)] + [(n, block.g[n], p[n].grad) for n in NAMES]:
        off = (got.cpu().double() - want).abs().max().item()
        assert off <= bar * want.abs().max().item(), (name, off, want.abs().max().item())


def test_steps_follow_float64():
    block = Block()
    start = {n: t.clone() for n, t in block.p.items()}
    for _ in range(STEPS):
        block.step()
    p = {n: t.double() for n, t in parameters().items()}
    states = {n: (torch.zeros_like(t), torch.zeros_like(t)) for n, t in p.items()}
    x, target = (t.double() for t in data())
    largest = {n: 0.0 for n in p}
    for step in range(1, STEPS + 1):
        p = {n: t.detach().requires_grad_() for n, t in p.items()}
        (0.5 * (forward64(p, x, 2 * (step - 1)) - target).square().sum()).backward()
        with torch.no_grad():
            for n in NAMES:
                g = p[n].grad * HYPER["grad_scale"]
                largest[n] = max(largest[n], g.abs().max().item())
                m, v = states[n]
                m.mul_(HYPER["beta1"]).add_(g, alpha=1 - HYPER["beta1"])
                v.mul_(HYPER["beta2"]).add_(g * g, alpha=1 - HYPER["beta2"])
                update = m / (1 - HYPER["beta1"] ** step) / (torch.sqrt(v / (1 - HYPER["beta2"] ** step)) + HYPER["eps"])
                p[n] = p[n] - LR * update
    for n in NAMES:
        # with eps = 1 an error e of a gradient moves a step by at most 2 lr e; gradients are within 5e-5 of the largest, and what earlier steps moved
        # comes on top (twice), and a half unit of a parameter's last place a step
        off = (block.p[n].cpu().double() - p[n]).abs().max().item()
        assert off <= STEPS * (2 * 2 * LR * 5e-5 * largest[n] + 2.0 ** -24 * p[n].abs().max().item() * 2), (n, off)
        moved = (block.p[n] - start[n]).abs().max().item()
        assert moved > 100 * off, (n, moved, off)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_replayed_steps_equal_eager_ones(dtype):
    eager, replayed = Block(dtype), Block(dtype)
    eager.step()
    replayed.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.step()
    masks = []
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        eager.step()
        for n in ("n1", "qkv", "att", "y", "out", "grad_x"):
            assert torch.equal(getattr(eager, n), getattr(replayed, n)), (k, n)
        for n in NAMES:
            assert torch.equal(eager.p[n], replayed.p[n]) and torch.equal(eager.g[n], replayed.g[n]), (k, n)
        masks.append(eager.g_branch == 0)
    assert not torch.equal(masks[0], masks[1]) and eager.count.item() == 10


def test_two_streams_at_once():
    blocks = [Block() for _ in range(3)]
    torch.cuda.synchronize()

    def work(block):
        for _ in range(STEPS):
            block.step()

    work(blocks[0])
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for s, block in zip(streams, blocks[1:]):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            work(block)
    torch.cuda.synchronize()
    for block in blocks[1:]:
        assert torch.equal(blocks[0].out, block.out) and torch.equal(blocks[0].grad_x, block.grad_x)
        for n in NAMES:
            assert torch.equal(blocks[0].p[n], block.p[n]), n
