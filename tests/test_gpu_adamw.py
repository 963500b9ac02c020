"""The AdamW step over many tensors, states in 32 and in 8 bits, against the same fp32 operations done one by one on the CPU."""
import math

import pytest
import torch

from paper_2503_06671_amd import binding
from tests import window_reference as ref

pytestmark = pytest.mark.gpu

SIZES = [1, 3, 4, 255, 256, 257, 1023, 4096, 4097, 0, 70001, 2, 9 * 16 * 8]


class Net:
    """Seeded parameters, gradients and states; `shift` puts each tensor off its natural alignment by that many elements."""

    def __init__(self, states, grads=torch.float32, sizes=SIZES, shift=0, seed=0, step=4):
        g = torch.Generator().manual_seed(seed)

        def device(x):
            room = torch.empty(x.numel() + 16, dtype=x.dtype, device="cuda") if x.dtype != torch.float8_e4m3fn else \
                torch.empty(x.numel() + 16, dtype=torch.uint8, device="cuda").view(x.dtype)
            t = room[shift:shift + x.numel()]
            t.view(torch.uint8).copy_(x.view(torch.uint8)) if x.dtype == torch.float8_e4m3fn else t.copy_(x)
            return t

        self.states, self.step = states, step
        self.p = [0.1 * torch.randn(n, generator=g) for n in sizes]
        self.g = [(torch.randn(n, generator=g) * torch.exp(2 * torch.randn(n, generator=g))).to(grads) for n in sizes]
        m = [0.3 * torch.randn(n, generator=g) for n in sizes]
        v = [torch.randn(n, generator=g).square() * torch.exp(3 * torch.randn(n, generator=g)) for n in sizes]
        self.scales = [None] * len(sizes)
        if states == "8bit":
            hm, hv = [ref.held(x, False) for x in m], [ref.held(torch.sqrt(x), True) for x in v]
            m, v = [c for c, _ in hm], [c for c, _ in hv]
            self.scales = [(a, b) for (_, a), (_, b) in zip(hm, hv)]
        self.m, self.v = m, v
        self.decay = [0.1 if i % 2 else 0.0 for i in range(len(sizes))]
        self.dp, self.dg = [device(x) for x in self.p], [device(x) for x in self.g]
        self.dm, self.dv = [device(x) for x in m], [device(x) for x in v]
        kw = {}
        if states == "8bit":
            self.ms, self.vs = [s[0].cuda() for s in self.scales], [s[1].cuda() for s in self.scales]
            kw = dict(m_scale=self.ms, v_scale=self.vs)
        self.opt = binding.AdamW(self.dp, self.dg, states=states, weight_decay=self.decay, step=step, m=self.dm, v=self.dv, **kw)

    def reference_step(self, lr, beta1, beta2, eps, grad_scale):
        self.step += 1
        for i in range(len(self.p)):
            if self.p[i].numel() == 0:
                continue
            self.p[i], self.m[i], self.v[i], ms, vs = ref.adamw(self.p[i], self.g[i], self.m[i], self.v[i], self.step, lr, beta1, beta2, eps,
                                                                self.decay[i], grad_scale, self.scales[i])
            self.scales[i] = None if ms is None else (ms, vs)

    def check(self):
        for i in range(len(self.p)):
            for name, a, b in (("p", self.dp[i], self.p[i]), ("m", self.dm[i], self.m[i]), ("v", self.dv[i], self.v[i])):
                a, b = a.cpu().to(torch.float32), b.to(torch.float32)
                assert torch.equal(torch.isnan(a), torch.isnan(b)), (i, name)
                assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)), (i, name, (a - b).abs().max())
            if self.states == "8bit" and self.p[i].numel():
                assert torch.equal(self.ms[i].cpu(), self.scales[i][0]) and torch.equal(self.vs[i].cpu(), self.scales[i][1]), i


@pytest.mark.parametrize("shift", [0, 1, 2])
@pytest.mark.parametrize("grads", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_steps_equal_the_operations_one_by_one(states, grads, shift):
    net = Net(states, grads, shift=shift, seed=shift)
    for k, h in enumerate([dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=1.0), dict(lr=5e-4, beta1=0.8, beta2=0.999, eps=1e-3, grad_scale=0.37),
                           dict(lr=0.0, beta1=0.0, beta2=0.0, eps=0.0, grad_scale=-2.0)]):
        h = dict(h)
        net.opt.step(h.pop("lr"), **h) if k else net.opt.step(**h)
        net.reference_step([1e-2, 5e-4, 0.0][k], *(h[n] for n in ("beta1", "beta2", "eps", "grad_scale")))
        net.check()
    assert net.opt.steps == 7


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_from_nothing_and_neighbours(states):
    # new states, zero gradients in part, values beside the tensors untouched
    room = torch.full((64 + 1000,), 7.0, device="cuda")
    p = room[32:32 + 1000]
    g = torch.randn(1000, device="cuda")
    g[300:700] = 0
    opt = binding.AdamW([p], [g], states=states)
    start = p.clone()
    opt.step(1e-3)
    # the first step moves by lr in the gradient's direction, where there is one
    want = start - 1e-3 * g / (g.abs() + 1e-8)
    # (beside 7, one unit of the last place of the result and the correction's rounding)
    assert (p - want).abs().max() <= 2 * 7 * 2.0 ** -23
    assert (room[:32] == 7).all() and (room[-32:] == 7).all()
    assert opt.steps == 1 and torch.isfinite(opt.m[0].to(torch.float32)).all()


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_values_that_are_not_finite_stay_by_themselves(states):
    net = Net(states, sizes=[1000], seed=3)
    bad = torch.zeros(1000, dtype=torch.bool)
    for i, x in ((5, math.nan), (300, math.inf), (301, -math.inf), (999, math.nan)):
        net.g[0][i] = x
        net.dg[0][i] = x
        bad[i] = True
    h = (1e-2, 0.9, 0.99, 1e-8, 1.0)
    for _ in range(2):
        net.opt.step(*h)
        net.reference_step(*h)
    got = net.dp[0].cpu()
    assert torch.equal(torch.isfinite(got), ~bad)
    assert torch.equal(got[~bad], net.p[0][~bad])
    for t in (net.dm[0], net.dv[0]):
        x = t.cpu().to(torch.float32)
        assert torch.isfinite(x[~bad]).all() and not torch.isfinite(x[bad]).any()


def test_tiny_and_huge_gradients_in_8_bits():
    # blocks whose states underflow hold zeros; large ones keep their range
    sizes = [256, 256, 512]
    net = Net("8bit", sizes=sizes, seed=4)
    for i, f in enumerate((1e-38, 1e15, 1e-6)):
        net.g[i] *= f
        net.dg[i] *= f
    for _ in range(30):
        net.opt.step(1e-3, beta1=0.5, beta2=0.5)
        net.reference_step(1e-3, 0.5, 0.5, 1e-8, 1.0)
    net.check()


def test_many_tensors_and_a_large_one():
    g = torch.Generator().manual_seed(9)
    sizes = [int(x) for x in torch.randint(1, 3000, (700,), generator=g)] + [9_000_011]   # more chunks than blocks
    net = Net("8bit", torch.bfloat16, sizes=sizes, seed=5)
    h = (1e-3, 0.9, 0.99, 1e-8, 1.0)
    for _ in range(2):
        net.opt.step(*h)
        net.reference_step(*h)
    net.check()
    assert net.opt.steps == 6


def test_replayed_steps_count_and_follow_the_learning_rate():
    net, same = Net("f32", seed=6), Net("f32", seed=6)
    lr = torch.zeros(1, device="cuda")
    net.opt.step(lr)          # (lr 0: only the states move)
    same.opt.step(0.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.opt.step(lr, beta2=0.99)
    for x in (0.5, 0.25, 1e-3):
        lr.fill_(x)
        graph.replay()
        torch.cuda.synchronize()
        same.opt.step(lr.item(), beta2=0.99)  # (the value as float32 holds it)
        for a, b in zip(net.dp + net.dm + net.dv, same.dp + same.dm + same.dv):
            assert torch.equal(a, b)
    assert net.opt.steps == same.opt.steps == 8


def test_on_a_side_stream():
    net = Net("8bit", seed=7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h = (1e-3, 0.9, 0.99, 1e-8, 1.0)
    net.opt.step(*h, stream=side)
    side.synchronize()
    net.reference_step(*h)
    net.check()


def test_only_empty_tensors():
    net = Net("f32", sizes=[0, 0], seed=8)
    net.opt.step(1e-3)
    assert net.opt.steps == 5


def test_short_tensors_step_after_step():
    # blocks whose first wavefront has little to do beside others that have nothing: each step's count is that of all of them
    net = Net("8bit", sizes=[1] * 40, seed=9)
    for k in range(20):
        h = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, grad_scale=1.0)
        net.opt.step(**h)
        net.reference_step(**h)
    net.check()
    assert net.opt.steps == 24


@pytest.mark.parametrize("replayed", [False, True])
def test_steps_waits_for_every_stream(replayed):
    net = Net("f32", seed=10)
    net.opt.step(1e-3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.opt.step(1e-3)
    x = torch.randn(4096, 4096, device="cuda")
    x @ x
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(20):  # (some milliseconds of work in front of the step)
            x @ x
        graph.replay() if replayed else net.opt.step(1e-3)
    assert net.opt.steps == 6


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_laid_out_on_a_side_stream(states):
    # the states' zeros and the plan come in front of a step on the same stream, whatever the current one is busy with
    p, g = torch.randn(70001, device="cuda"), torch.randn(70001, device="cuda")
    same = p.clone()
    want = binding.AdamW([same], [g], states=states)
    want.step(1e-2)
    x = torch.randn(4096, 4096, device="cuda")
    x @ x
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        x @ x
    opt = binding.AdamW([p], [g], states=states, stream=side)
    opt.step(1e-2, stream=side)
    assert opt.steps == 1
    assert torch.equal(p, same)
    for a, b in ((opt.m[0], want.m[0]), (opt.v[0], want.v[0])):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
