"""Layer norm, products and dropout captured into graphs, one of each kernel's kind: replays with other inputs equal the eager calls, with eager work and
synchronisations between them, of two graphs in turn."""
import pytest
import torch

from paper_2503_06671_amd import binding

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# dtype, N, K, M, H, W, act: input channels in registers (few and most, with and without the joint backward kernel), streamed, by addresses, few pixels, many splits and few
PRODUCTS = [(F32, 1, 64, 65, 64, 64, "gelu"), (F32, 3, 40, 20, 150, 301, "silu"), (F32, 1, 155, 40, 64, 64, "none"), (BF16, 1, 190, 100, 100, 130, "gelu"), (BF16, 3, 60, 100, 150, 301, "gelu"),
            (BF16, 1, 260, 210, 180, 320, "silu"), (F32, 2, 210, 130, 100, 131, "gelu"), (BF16, 300, 24, 40, 3, 5, "silu"), (F32, 1, 640, 32, 5, 9, "gelu"), (BF16, 1, 700, 1000, 33, 31, "none")]
NORMS = [(F32, 2, 64, 33, 31), (BF16, 4, 700, 9, 9), (F32, 1, 1100, 12, 13), (BF16, 70, 16, 1, 1)]
DROPOUTS = [(F32, 2, 7, 9, 11, "plane"), (BF16, 3, 5, 40, 40, "plane"), (F32, 4, 6, 8, 8, "image"), (BF16, 2, 3, 33, 7, "element")]


def product(dtype, N, K, M, H, W, act, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    inputs = [r(N, K, H, W).to(dtype), r(M, K) * K ** -0.5, r(M), r(N, M, H, W).to(dtype), r(N, M, H, W).to(dtype)]
    ws = binding.new_pointwise_backward_workspace(N, K, M, H, W, dtype, act=act)

    def run(x, w, b, res, go):
        out = binding.pointwise_forward(x, w, b, act, res)
        return [out, *binding.pointwise_backward(x, go, w, ws, b, act).values(), *binding.pointwise_backward(x, go, w, ws, b, act, need=("grad_w",)).values()]
    return inputs, run


def norm(dtype, N, C, H, W, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    inputs = [r(N, C, H, W).to(dtype), r(C), r(C), r(N, C, H, W).to(dtype), r(N, C, H, W).to(dtype)]
    saved, ws = binding.new_layernorm_saved(N, H, W), binding.new_layernorm_backward_workspace(N, C, H, W)

    def run(x, w, b, skip, go):
        out = binding.layernorm_forward(x, w, b, saved=saved)
        return [out, *binding.layernorm_backward(x, go, saved, ws, w, b, grad_skip=skip).values()]
    return inputs, run


def dropout(dtype, N, C, H, W, over, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g).to(dtype)  # noqa: E731
    inputs = [r(N, C, H, W), r(N, C, H, W), r(N, C, H, W), torch.tensor([seed], device="cuda")]

    def run(x, res, go, count):
        return [binding.dropout_forward(x, 0.4, 11, 3, offset_device=count, over=over, residual=res), binding.dropout_backward(go, 0.4, 11, 3, offset_device=count, over=over)]
    return inputs, run


@pytest.mark.parametrize("make, case", [(f, c) for f, cases in ((product, PRODUCTS), (norm, NORMS), (dropout, DROPOUTS)) for c in cases], ids=lambda v: v.__name__ if callable(v) else "-".join(map(str, v)))
def test_replays_equal_eager_calls(make, case):
    pairs = []
    for seed in (1, 2):   # two graphs, each with its own buffers
        inputs, run = make(*case, seed)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(*inputs)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results = run(*inputs)
        pairs.append((inputs, run, graph, results))
    for turn in range(3):
        for k, (inputs, run, graph, results) in enumerate(pairs):
            for t, new in zip(inputs, make(*case, 10 * turn + k)[0]):
                t.copy_(new)
            graph.replay()
            if turn % 2:
                torch.cuda.synchronize()
            want = [t.clone() for t in results]
            eager = run(*inputs)
            assert all(torch.equal(a, b) for a, b in zip(want, eager)), (turn, k)
            assert all(torch.equal(a, b) for a, b in zip(results, want)), (turn, k)
