"""Window attention where fewer bits than the result's type holds would show, against the float64 reference."""
import pytest
import torch

from tests import window_reference as ref
from tests.test_gpu_window_attention import BF16, Case, whole_images_and_holes

pytestmark = pytest.mark.gpu

# windows of few pixels: nothing averages what rounding does to single terms
SMALL = [
    # N, H, W, heads, d, window, keywords
    (6, 12, 20, 2, 16, (1, 2), {}),
    (4, 15, 18, 4, 8, (2, 3), {"kv": 2}),
    (3, 16, 20, 3, 32, (4, 4), {"mask": whole_images_and_holes}),
    (2, 24, 23, 2, 64, (5, 3), {"edges": [1, 2]}),
    (2, 33, 40, 2, 16, (8, 8), {}),
    (1, 64, 40, 2, 24, (20, 20), {}),
]


def assert_rounded_once(got, r, name, d, tokens, terms, what):
    """`got` is r[name] rounded to bf16 from a value that is off by e: e is what fp32 arithmetic does (ref.tolerance of fp32 results) and `terms`
    of the sum of magnitudes.  A value's distance from the nearest bf16 one changes by no more than the value, so the rounded value is at
    most 2 e farther off than the exact one rounded."""
    exact = r[name]
    rounding = (exact.to(BF16).to(ref.D) - exact).abs()
    e = ref.tolerance(r, name, torch.float32, d, tokens) + terms * r[name + "_abs"]
    off = (got.detach().cpu().to(ref.D) - exact).abs()
    assert torch.isfinite(off).all(), (what, name)
    worst = (off / (rounding + 2 * e)).max().item()
    assert worst <= 1.0, (what, name, worst)


@pytest.mark.parametrize("case", range(len(SMALL)))
def test_probabilities_in_bf16_results(case):
    # two bf16 terms at least: 2^-8 of what is left after the first, 2^-16 of a probability
    N, H, W, heads, d, window, more = SMALL[case]
    print(f"[case] {SMALL[case]}", flush=True)
    c = Case(BF16, N, H, W, heads, d, window, seed=300 + case, **more)
    r = c.reference()
    assert_rounded_once(c.forward(), r, "out", d, c.tokens, 2.0 ** -16, SMALL[case])
    assert_rounded_once(c.train()["out"], r, "out", d, c.tokens, 2.0 ** -16, SMALL[case])


@pytest.mark.parametrize("case", range(len(SMALL)))
def test_terms_of_the_gradients(case):
    # p and the scores' gradients in two bf16 terms at least
    N, H, W, heads, d, window, more = SMALL[case]
    print(f"[case] {SMALL[case]}", flush=True)
    c = Case(BF16, N, H, W, heads, d, window, seed=330 + case, **more)
    r, got = c.reference(), c.train()
    group = c.heads // c.kv
    for name, tokens in (("grad_q", c.tokens), ("grad_k", c.tokens * group), ("grad_v", c.tokens * group)):
        assert_rounded_once(got[name], r, name, d, tokens, 2.0 ** -16, SMALL[case])


def exact_scores(dtype, base, N, heads, seed, grads=True):
    """A case whose scores are whole numbers, `base` and some tens around it, which fp32 holds as they are: whatever the results are off is the
    softmax's own doing.  Biases that rise for half of a tile's queries only make its running maxima move together by anything between nothing and
    tens."""
    c = Case(dtype, N, 16, 16, heads, 16, (16, 16), seed=seed)
    g = torch.Generator().manual_seed(seed + 1)
    for t in (c.q, c.k):
        t.copy_(torch.randint(-1, 2, t.shape, generator=g).to(dtype))
    c.bias.copy_(base + torch.randint(0, 4, c.bias.shape, generator=g))
    for i, oy in enumerate(range(-12, 13, 4)):
        c.bias[:, 15 + oy, 15 + 8] += 8 * i
    c.kw["scale"] = 1.0
    cpu = [t.cpu() for t in (c.q, c.k, c.v, c.bias)]
    r = ref.attention(*cpu[:3], heads, c.window, bias=cpu[3], scale=1.0, grad_out=c.go.cpu() if grads else None)
    assert r["score_abs"] < 2 ** 24
    # what may round are differences of scores from the largest, the largest being exact
    r["score_abs"] = 3.0 + 48.0 + 2 * 16.0
    return c, r


# (exponentials are worked out in different ways below and beyond shifts of 2^8 and of 2^20)
BASES = [0, 2 ** 10, 2 ** 16, 2 ** 19, -2 ** 19, 2 ** 21, -2 ** 21]


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("base", BASES)
def test_gradients_of_large_scores(base, dtype):
    c, r = exact_scores(dtype, base, 2, 2, seed=400)
    got = c.train()
    for name in ("grad_q", "grad_k", "grad_v", "grad_bias"):
        ref.assert_close(got[name], r, name, dtype, c.d, c.tokens * (c.N if name == "grad_bias" else 1), base)


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,heads", [(2, 2), (70, 4), (140, 4)])   # keys shared by wavefronts, one tile a wavefront, two
@pytest.mark.parametrize("base", BASES)
def test_sums_keep_step_with_a_rising_maximum(base, N, heads, dtype):
    c, r = exact_scores(dtype, base, N, heads, seed=430, grads=False)
    for saved in (None, c.buffers()[0]):
        out = c.forward(saved=saved)
        if dtype == BF16:
            assert_rounded_once(out, r, "out", c.d, c.tokens, 2.0 ** -16, base)
        else:
            ref.assert_close(out, r, "out", dtype, c.d, c.tokens, base)


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,heads", [(2, 2), (70, 4)])
def test_rows_of_very_different_scores_beside_each_other(N, heads, dtype):
    # rows whose scores reach 2^4 to 2^21, in turn within each tile: each way of working out exponentials in each tile
    c, _ = exact_scores(dtype, 0, N, heads, seed=460, grads=False)
    factor = 2.0 ** torch.tensor([0, 5, 12, 17, 0, 3, 9])[torch.arange(256) % 7].reshape(16, 16)
    c.q.mul_(factor.to("cuda", dtype))
    cpu = [t.cpu() for t in (c.q, c.k, c.v, c.bias)]
    r = ref.attention(*cpu[:3], heads, c.window, bias=cpu[3], scale=1.0, grad_out=c.go.cpu())
    assert 2 ** 20 < r["score_abs"] < 2 ** 24
    r["score_abs"] = 3.0 + 48.0 + 2 * 16.0  # (scores farther than that below the largest weigh nothing)
    got = c.train()
    for name in ("grad_q", "grad_k", "grad_v", "grad_bias"):
        ref.assert_close(got[name], r, name, dtype, c.d, c.tokens * (N if name == "grad_bias" else 1), N)
    if dtype == BF16:
        assert_rounded_once(got["out"], r, "out", c.d, c.tokens, 2.0 ** -16, N)
    else:
        ref.assert_close(got["out"], r, "out", dtype, c.d, c.tokens, N)
