"""Layer norm, the point-wise product and their gradients at sizes near the limits of a launch and of 32-bit offsets."""
import math

import pytest
import torch

from paper_2503_06671_amd import binding
from tests import block_reference as ref
from tests import product_limits

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def filled(*shape, dtype=BF16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty(*shape, device="cuda", dtype=dtype)
    for part in t.view(-1).split(2 ** 28):
        part.normal_(generator=g)
    return t


# images of one pixel: 2^24 tiles of blocks that have a tile each, or four; a few more, so that a second launch is there and small
@pytest.mark.parametrize("N, C", [(2 ** 24 + 301, 49), (2 ** 26 + 70, 3)])
def test_layer_norm_of_more_blocks_than_a_launch_has(N, C):
    x, w, b = filled(N, C, 1, 1), filled(C, dtype=torch.float32, seed=1), filled(C, dtype=torch.float32, seed=2)
    print(f"[case] layer norm of {N} images of one pixel, {C} channels", flush=True)
    out = torch.full_like(x, float("nan"))
    binding.layernorm_forward(x, w, b, out=out)
    # a pixel's result depends on nothing else: the same from calls of fewer images
    for first in range(0, N, 2 ** 23):
        part = slice(first, min(first + 2 ** 23, N))
        assert torch.equal(out[part], binding.layernorm_forward(x[part], w, b)), first
    for part in (slice(0, 500), slice(2 ** 24 - 200, 2 ** 24 + 300), slice(N - 500, N)):
        ref.check(out[part], ref.norm(x[part], w, b)["out"], "out")


# planes of 2^30 pixels, by addresses of 64 bits; images of 96 pixels that have a block each, in the kernels that keep the input channels in registers
@pytest.mark.parametrize("N, H, W, K, M, act", [(2, 2 ** 15, 2 ** 15, 2, 3, "none"), (2 ** 24 + 130, 96, 1, 2, 1, "none"), (2 ** 24 + 130, 96, 1, 1, 2, "gelu")])
def test_products_of_more_blocks_than_a_launch_has(N, H, W, K, M, act):
    x, go = filled(N, K, H, W), filled(N, M, H, W, seed=1)
    w, b = filled(M, K, dtype=torch.float32, seed=2), filled(M, dtype=torch.float32, seed=3)
    print(f"[case] product of {N} x {H} x {W} pixels, {K} to {M} channels, {act}", flush=True)
    out, gx = torch.full_like(go, float("nan")), torch.full_like(x, float("nan"))
    binding.pointwise_forward(x, w, b, act, out=out)
    ws = binding.new_pointwise_backward_workspace(N, K, M, H, W, BF16, act=act)
    got = binding.pointwise_backward(x, go, w, ws, b, act, grads=dict(grad_x=gx))
    del ws
    assert torch.isfinite(got["grad_w"]).all()
    each = max(1, N // 4)
    for first in range(0, N, each):
        part = slice(first, min(first + each, N))
        n = part.stop - part.start
        assert torch.equal(out[part], binding.pointwise_forward(x[part], w, b, act)), first
        ws = binding.new_pointwise_backward_workspace(n, K, M, H, W, BF16, act=act)
        assert torch.equal(gx[part], binding.pointwise_backward(x[part], go[part], w, ws, b, act, need=("grad_x",))["grad_x"]), first
    # some rows of the first and last images, and of those on either side of the 2^24th block's, against float64
    for n in {0, min(N - 1, 2 ** 24 - 1), min(N - 1, 2 ** 24), N - 1}:
        for y in (0, H // 2 - 1, H - 2):
            at = (slice(n, n + 1), slice(None), slice(y, y + 2))
            want = ref.product(x[at], w, b, act, None, go[at])
            ref.check(out[at], want["out"], "out")
            ref.check(gx[at], want["grad_x"], "grad_x")
    # the weights' gradients: a share (of 512) adds its pixels up in sixteens, then come the shares' sums: off by 2^-24 each time at most of the magnitudes
    sums = torch.zeros(M, K, dtype=torch.float64, device="cuda")
    size, off = sums.clone(), sums.clone()
    for first in range(0, N, max(1, N // 64)):
        part = slice(first, min(first + max(1, N // 64), N))
        for y in range(0, H, 4096):
            xs, gs = x[part, :, y:y + 4096].double(), go[part, :, y:y + 4096].double()
            gp = gs
            if act != "none":
                parts = [w[:, k].double().view(1, -1, 1, 1) * xs[:, k:k + 1] for k in range(K)] + [ref.each(b)]
                gp = gs * ref.slope(act, sum(parts))
                # (as ref.product has it: the slope within 1e-6, |act''| <= 0.8, its argument's terms and sums)
                e = gs.abs() * (0.8 * (2.0 ** -21 + (K + 16) * 2.0 ** -23) * sum(t.abs() for t in parts) + 1e-6)
            for m in range(M):
                for k in range(K):
                    p = gp[:, m] * xs[:, k]
                    sums[m, k] += p.sum()
                    size[m, k] += p.abs().sum()
                    if act != "none":
                        off[m, k] += (e[:, m] * xs[:, k].abs()).sum()
    depth = (N * H * W / 512 / 16 + 64) * 2.0 ** -23
    assert ((got["grad_w"].double() - sums).abs() <= off + (2.0 ** -21 + depth) * size).all()


@pytest.mark.parametrize("case", product_limits.CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_products_on_either_side_of_32_bit_offsets(case):
    dt, K, M, H, W, act, _, _ = case
    dtype = torch.float32 if dt == product_limits.F32 else BF16
    x, go, res = filled(1, K, H, W, dtype=dtype), filled(1, M, H, W, dtype=dtype, seed=1), filled(1, M, H, W, dtype=dtype, seed=2)
    w, b = filled(M, K, dtype=torch.float32, seed=3) * K ** -0.5, filled(M, dtype=torch.float32, seed=4)
    print(f"[case] product of {H} x {W} pixels, {K} to {M} channels, {act}, {dtype}", flush=True)
    # (guards: nothing is written in front of a result or behind it)
    room = {n: torch.full((c * H * W + 2048,), 7.0, device="cuda", dtype=dtype) for n, c in (("out", M), ("grad_x", K))}
    out, gx = room["out"][1024:-1024].view(1, M, H, W), room["grad_x"][1024:-1024].view(1, K, H, W)
    out.fill_(math.nan), gx.fill_(math.nan)
    binding.pointwise_forward(x, w, b, act, res, out=out)
    ws = binding.new_pointwise_backward_workspace(1, K, M, H, W, dtype, act=act)
    got = binding.pointwise_backward(x, go, w, ws, b, act, grads=dict(grad_x=gx))
    for n in room:
        assert (room[n][:1024] == 7).all() and (room[n][-1024:] == 7).all() and torch.isfinite(room[n]).all(), n
    for y in (0, H // 3, H // 2, H - 2):
        rows = (slice(None), slice(None), slice(y, y + 2))
        want = ref.product(x[rows], w, b, act, res[rows], go[rows])
        ref.check(out[rows], want["out"], "out")
        ref.check(gx[rows], want["grad_x"], "grad_x")
    # the weights' gradients, by their 2-norm: terms and slope 2^-20, a share's additions (128 shares at least, six products of terms
    # for sixteen pixels) and the shares'
    sums = {"grad_w": 0.0, "grad_b": 0.0}
    for y in range(0, H, 256):
        xs, gp = x[0, :, y:y + 256].double().flatten(1), go[0, :, y:y + 256].double().flatten(1)
        if act != "none":
            gp = gp * ref.slope(act, w.double() @ xs + b.double()[:, None])
        sums = {"grad_w": sums["grad_w"] + torch.stack([(gp * row).sum(1) for row in xs], 1), "grad_b": sums["grad_b"] + gp.sum(1)}
    bar = 2.0 ** -20 + 2.0 ** -23 * math.sqrt(6 * H * W / 16 / 128 + 32)
    for n, true in sums.items():
        assert ((got[n].double() - true).norm() / true.norm()).item() < bar, n
