"""Window attention with a learned relative position bias, and its gradients, against the float64 reference, at the sizes, masks and
layouts where it can go wrong."""
import math

import pytest
import torch

from paper_2503_06671_amd import binding
from tests import window_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
NAMES = ("out", "grad_q", "grad_k", "grad_v", "grad_bias")


class Case:
    """Seeded inputs on the device, q, k and v as slices of one tensor unless `apart`."""

    def __init__(self, dtype, N, H, W, heads, d, window, kv=None, edges=None, mask=None, bias=0.5, apart=False, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.heads, self.kv, self.d, self.window, self.edges = dtype, heads, kv or heads, d, window, edges
        self.N, self.H, self.W = N, H, W
        C, Ckv = heads * d, self.kv * d
        qkv = torch.randn(N, C + 2 * Ckv, H, W, generator=g).to(dtype)
        self.go = torch.randn(N, C, H, W, generator=g).to(dtype).cuda()
        n = (2 * len(edges) + 1,) * 2 if edges else (2 * window[0] - 1, 2 * window[1] - 1)
        self.bias = None if bias is None else (bias * torch.randn(heads, *n, generator=g)).cuda()
        self.mask = None
        if mask is not None:
            m = mask(N, H, W, g)
            qkv = torch.where(m[:, None], qkv, torch.full((), math.nan, dtype=dtype))
            self.mask = m.to(torch.uint8).cuda()
        qkv = qkv.cuda()
        parts = qkv[:, :C], qkv[:, C:C + Ckv], qkv[:, C + Ckv:]
        self.q, self.k, self.v = (p.contiguous() for p in parts) if apart else parts
        self.kw = dict(bias=self.bias, edges=edges, mask=self.mask, kv_heads=self.kv)
        self.tokens = min(window[0], H) * min(window[1], W)

    def buffers(self):
        return (binding.new_window_attention_saved(self.N, self.heads, self.d, self.H, self.W, self.dtype),
                binding.new_window_attention_backward_workspace(self.N, self.heads, self.d, self.H, self.W, self.window))

    def forward(self, **kw):
        return binding.window_attention_forward(self.q, self.k, self.v, self.heads, self.window, **{**self.kw, **kw})

    def train(self, buffers=None, **kw):
        saved, ws = buffers or self.buffers()
        out = self.forward(saved=saved)
        grads = binding.window_attention_backward(self.q, self.k, self.v, out, self.go, saved, self.heads, self.window, ws,
                                                  **{**self.kw, **kw})
        return dict(grads, out=out)

    def reference(self):
        cpu = [None if t is None else t.cpu() for t in (self.q, self.k, self.v, self.bias, self.mask, self.go)]
        return ref.attention(*cpu[:3], self.heads, self.window, bias=cpu[3], edges=self.edges, mask=cpu[4], kv_heads=self.kv, grad_out=cpu[5])

    def check(self, got, r, what=""):
        for n in NAMES:
            if n in got:
                # a key and value head is summed over its group's queries
                tokens = self.tokens * (self.heads // self.kv if n in ("grad_k", "grad_v") else 1)
                if n == "grad_bias":
                    tokens *= self.N * math.ceil(self.H / self.window[0]) * math.ceil(self.W / self.window[1])
                ref.assert_close(got[n], r, n, self.dtype, self.d, tokens, what)


def whole_images_and_holes(N, H, W, g):
    m = torch.rand(N, H, W, generator=g) > 0.15
    m[:, int(H * 0.7):] = False
    m[0, :, W // 2:] = False
    if N > 1:
        m[-1] = False
    return m


CASES = [
    # N, H, W, heads, d, window, keywords
    (1, 1, 1, 1, 1, (1, 1), {}),                                       # one pixel
    (2, 3, 2, 2, 5, (4, 4), {}),                                       # a window larger than the map
    (1, 7, 9, 1, 16, (1, 1), {}),                                      # windows of one pixel
    (1, 40, 5, 2, 8, (16, 1), {}),                                     # columns
    (1, 2, 333, 2, 12, (1, 128), {}),                                  # rows, the last shorter
    (1, 16, 16, 4, 16, (8, 8), {}),                                    # whole vectors
    (2, 33, 35, 2, 16, (8, 8), {}),                                    # windows cut at both edges
    (1, 20, 28, 3, 24, (7, 7), {}),                                    # rows that are no whole vectors
    (1, 45, 50, 2, 33, (13, 17), {"kv": 1}),                           # odd everything, shared keys
    (1, 32, 32, 2, 16, (32, 32), {}),                                  # 1024 pixels
    (1, 64, 33, 1, 16, (32, 32), {}),                                  # a window of one column beside whole ones
    (1, 48, 48, 1, 32, (48, 48), {}),
    (1, 24, 31, 6, 64, (12, 12), {"kv": 2}),                           # widest heads, groups of three
    (1, 64, 64, 1, 64, (64, 64), {}),                                  # the largest square window with the widest head
    (1, 1, 2500, 2, 16, (1, 4096), {"kv": 1, "edges": [1, 2, 3, 5, 9, 17, 33, 65, 129, 257]}),  # a sequence with buckets
    (2, 21, 26, 2, 16, (10, 10), {"edges": [1, 3]}),
    (3, 21, 26, 4, 8, (10, 10), {"kv": 2, "mask": whole_images_and_holes}),
    (2, 32, 40, 2, 16, (16, 16), {"mask": whole_images_and_holes, "edges": [2, 4, 8]}),
    (2, 17, 19, 2, 16, (8, 8), {"bias": None}),
    (2, 12, 16, 2, 20, (8, 8), {"apart": True}),
    (3, 5, 7, 1, 3, (3, 3), {"kv": 1}),                                # planes, images and tensors at odd elements
    (2, 1, 9, 37, 1, (1, 5), {"kv": 1}),                               # one channel a head, 37 heads share a key
    (40, 1, 2, 2, 16, (1, 2), {}),                                     # two tokens: nothing averages what rounding does
    (9, 6, 5, 4, 24, (2, 3), {"kv": 2, "edges": [1, 2], "mask": whole_images_and_holes}),
    (5, 33, 37, 3, 8, (4, 4), {"kv": 1}),                              # hundreds of windows, not a whole number of runs
    (2, 23, 163, 2, 33, (5, 9), {"kv": 1, "mask": whole_images_and_holes}),  # rows that end in a window of one column
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_and_gradients(case, dtype):
    N, H, W, heads, d, window, more = CASES[case]
    print(f"[case] {CASES[case]} {dtype}", flush=True)
    c = Case(dtype, N, H, W, heads, d, window, seed=100 + case, **more)
    r = c.reference()
    got = c.train()
    c.check(got, r, CASES[case])
    # without `saved` the same but for what the backward pass needs
    alone = c.forward()
    ref.assert_close(alone, r, "out", dtype, d, c.tokens)
    if c.mask is not None:
        hidden = (c.mask == 0)[:, None]
        for n in ("out", "grad_q", "grad_k", "grad_v"):
            assert (torch.where(hidden, got[n], torch.zeros_like(got[n])) == 0).all(), n
    if dtype == F32:
        assert torch.equal(alone, got["out"])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_equal_calls_give_equal_bits(dtype):
    c = Case(dtype, 3, 70, 61, 4, 16, (20, 20), kv=2, seed=7)
    a, b = c.train(), c.train()
    for n in NAMES:
        assert torch.equal(a[n], b[n]), n


def test_a_batch_reproduces_its_images():
    c = Case(BF16, 3, 40, 24, 2, 16, (16, 16), seed=8)
    whole = c.train()
    for n in range(3):
        one = binding.window_attention_forward(c.q[n:n + 1], c.k[n:n + 1], c.v[n:n + 1], 2, (16, 16), **c.kw,
                                               saved=binding.new_window_attention_saved(1, 2, 16, 40, 24, BF16))
        assert torch.equal(one, whole["out"][n:n + 1])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_biases_that_hide(dtype):
    # -infinity beyond a distance, in a whole head, and the type's lowest value everywhere (which leaves the scores' order)
    c = Case(dtype, 1, 20, 24, 3, 16, (10, 12), seed=9)
    y, x = torch.arange(-9, 10)[:, None], torch.arange(-11, 12)[None]
    c.bias[0][((y.abs() > 3) | (x.abs() > 2)).cuda()] = -math.inf
    c.bias[1] = -math.inf
    r = c.reference()
    got = c.train()
    c.check(got, r)
    assert (got["out"][:, 16:32] == 0).all() and (got["grad_bias"][1] == 0).all()
    c.bias[:] = torch.finfo(F32).min
    got = c.train()
    want = torch.nn.functional.avg_pool2d(c.v.double(), (10, 12)).repeat_interleave(10, 2).repeat_interleave(12, 3)
    # scores vanish beside the lowest value: equal weights
    assert (got["out"].double() - want).abs().max() < (2.0 ** -7 if dtype == BF16 else 1e-5)


def test_scores_far_apart_and_large():
    # scores up to hundreds: the running maximum decides; a row that keeps one key only
    c = Case(F32, 1, 32, 32, 1, 16, (32, 32), seed=10)
    c.q *= 8
    c.k *= 8
    r = c.reference()
    c.check(c.train(), r)
    # and scores beyond 2^24, where rounding is coarser than an exponential: one key a row is left, and nothing overflows
    c.q *= 2.0 ** 50
    got = c.train()
    assert all(torch.isfinite(got[n]).all() for n in NAMES)
    # (rows whose two largest scores are nearer than 2^-20 of them may take either)
    q, k, v = (x.double().reshape(16, 1024).T for x in (c.q, c.k, c.v))
    two = (q @ k.T).topk(2, dim=1)
    clear = two.values[:, 0] - two.values[:, 1] > 2.0 ** -20 * two.values.abs().amax(1)
    assert clear.sum() > 900
    assert torch.equal(got["out"].reshape(16, 1024).T[clear].double(), v[two.indices[clear, 0]])
    if clear.all():  # each key's gradient is the sum over the rows that took it
        want = torch.zeros(1024, 16, device="cuda", dtype=torch.float64).index_add_(0, two.indices[:, 0], c.go.double().reshape(16, 1024).T)
        assert (got["grad_v"].reshape(16, 1024).T.double() - want).abs().max() <= 1024 * 2.0 ** -24 * want.abs().max()


def test_nan_reaches_its_own_window_and_head_alone():
    c = Case(F32, 1, 16, 16, 2, 16, (8, 8), seed=11)
    want = c.forward()
    c.v[0, 3, 2, 5] = math.nan   # head 0, first window, channel 3
    got = c.forward()
    bad = torch.zeros_like(want, dtype=torch.bool)
    bad[0, 3, :8, :8] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])


def test_accumulate_and_buffers():
    c = Case(F32, 2, 24, 20, 2, 16, (8, 8), seed=12)
    plain = c.train()
    start = torch.randn_like(c.bias)
    room = torch.full((2, 3 * 32, 24, 20), math.nan, device="cuda")   # one tensor for all three gradients
    grads = {"grad_q": room[:, :32], "grad_k": room[:, 32:64], "grad_v": room[:, 64:], "grad_bias": start.clone()}
    got = c.train(accumulate=True, grads=grads)
    assert torch.equal(got["grad_bias"], start + plain["grad_bias"])
    for n in ("grad_q", "grad_k", "grad_v"):
        assert got[n] is grads[n] and torch.equal(got[n], plain[n]), n


def test_one_tensor_as_query_key_and_value():
    # attention without projections
    c = Case(BF16, 1, 32, 32, 4, 16, (16, 16), seed=13)
    x = c.q
    out = binding.window_attention_forward(x, x, x, 4, (16, 16), bias=c.bias)
    r = ref.attention(x.cpu(), x.cpu(), x.cpu(), 4, (16, 16), bias=c.bias.cpu())
    ref.assert_close(out, r, "out", BF16, 16, 256)


def test_neighbours_of_out_stay():
    c = Case(BF16, 1, 9, 11, 2, 7, (4, 4), seed=14)
    room = torch.full((c.q.numel() + 64,), 3.0, device="cuda", dtype=BF16)
    out = room[32:32 + c.q.numel()].view(c.q.shape)
    c.forward(out=out)
    assert (room[:32] == 3).all() and (room[-32:] == 3).all()


def test_images_more_than_32_bits_apart():
    c = Case(BF16, 2, 16, 16, 1, 16, (16, 16), apart=True, seed=15)
    want = c.train()
    step = 2 ** 31 + 24
    room = torch.empty(step + 3 * 16 * 256, device="cuda", dtype=BF16)
    q, k, v = (room.as_strided((2, 16, 16, 16), (step, 256, 16, 1), i * 16 * 256) for i in range(3))
    for to, x in ((q, c.q), (k, c.k), (v, c.v)):
        to.copy_(x)
    c.q, c.k, c.v = q, k, v
    grads = {n: torch.empty(1, device="cuda", dtype=BF16) for n in ()}
    got = c.train(grads=grads)
    for n in NAMES:
        assert torch.equal(got[n], want[n]), n


def test_stream_and_replayed_graph():
    c = Case(BF16, 2, 40, 48, 2, 16, (16, 16), seed=16)
    want = c.train()
    buffers = c.buffers()
    room = {n: torch.empty_like(want[n]) for n in NAMES}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def work():
        binding.window_attention_forward(c.q, c.k, c.v, 2, (16, 16), **c.kw, out=room["out"], saved=buffers[0])
        binding.window_attention_backward(c.q, c.k, c.v, room["out"], c.go, buffers[0], 2, (16, 16), buffers[1], **c.kw,
                                          grads={n: room[n] for n in NAMES[1:]})

    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    for n in NAMES:
        assert torch.equal(room[n], want[n]), n
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for seed in range(3):
        x = Case(BF16, 2, 40, 48, 2, 16, (16, 16), seed=50 + seed)
        for a, b in ((c.q, x.q), (c.k, x.k), (c.v, x.v), (c.go, x.go), (c.bias, x.bias)):
            a.copy_(b)
        eager = c.train()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in NAMES:
            assert torch.equal(room[n], eager[n]), (seed, n)


def test_accumulate_without_a_buffer_on_a_side_stream():
    c = Case(F32, 2, 24, 20, 2, 16, (8, 8), seed=17)
    want = c.train()
    saved, ws = c.buffers()
    out = c.forward(saved=saved)
    x = torch.randn(4096, 4096, device="cuda")
    x @ x
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):  # (the current stream is busy meanwhile)
        x @ x
    got = binding.window_attention_backward(c.q, c.k, c.v, out, c.go, saved, c.heads, c.window, ws, **c.kw, accumulate=True, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for n in NAMES[1:]:
        assert torch.equal(got[n], want[n]), n
