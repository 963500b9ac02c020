"""The point-wise product's results in all, in every kernel: fp32 ones hold fp32 accuracy (no term of a factor is missing), bf16 ones are the nearest of the
definition's but for a few."""
import pytest
import torch

from paper_2503_06671_amd import binding
from tests import block_reference as ref
from tests import product_accuracy as pa

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", pa.CASES, ids=lambda c: "-".join([pa.NAMES[c[0]], *map(str, c[1:])]))
def test_results_are_as_accurate_as_their_terms(case):
    dt, N, K, M, H, W, act = case
    dtype = torch.float32 if dt == pa.F32 else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(17)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, w, b, go, res = r(N, K, H, W).to(dtype), r(M, K) * K ** -0.5, r(M), r(N, M, H, W).to(dtype), r(N, M, H, W).to(dtype)
    want = {n: v for n, (v, _) in ref.product(x, w, b, act, None, go).items()}
    ws = binding.new_pointwise_backward_workspace(N, K, M, H, W, dtype, act=act)
    results = [("out", binding.pointwise_forward(x, w, b, act), want["out"]),
               ("out", binding.pointwise_forward(x, w, b, act, res), want["out"] + res.double())]
    for need in (None, ("grad_w", "grad_b")):
        results += [(n, t, want[n]) for n, t in binding.pointwise_backward(x, go, w, ws, b, act, need=need).items()]
    bars = pa.bars(case)
    for name, got, true in results:
        if got.dtype == torch.float32:
            assert pa.off(got, true) < bars[name], (name, pa.off(got, true), bars[name])
        else:
            others = (got != true.bfloat16()).double().mean().item()
            assert others < pa.OTHERS, (name, others)


@pytest.mark.parametrize("dt, act", [(pa.F32, "none"), (pa.F32, "silu"), (pa.BF16, "silu")])
@pytest.mark.parametrize("K, M", [(31, 3), (100, 70)])
def test_long_sums_lean_to_neither_side(K, M, dt, act):
    # roundings of either sign: over n independent sums the mean of what they are off by is within five sqrt(1/n) of its root mean square
    dtype = torch.float32 if dt == pa.F32 else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(18)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x, w, b, go = r(1, K, 1024, 1024).to(dtype), r(M, K) * K ** -0.5, r(M), r(1, M, 1024, 1024).to(dtype)
    ws = binding.new_pointwise_backward_workspace(1, K, M, 1024, 1024, dtype, act=act)
    got = binding.pointwise_backward(x, go, w, ws, b, act, need=("grad_w",))["grad_w"]
    want = sum(ref.product(x[:, :, y:y + 64], w, b, act, None, go[:, :, y:y + 64])["grad_w"][0] for y in range(0, 1024, 64))
    d = got.double() - want
    assert d.mean().abs() < 5 * (d.numel() ** -0.5) * d.square().mean().sqrt(), (d.mean().item(), d.square().mean().sqrt().item())
