"""The point-wise product with bias, activation and residual, and its gradients: equal to whole numbers where all sums are exact, within derived
bounds of float64 elsewhere."""
import math

import pytest
import torch

from paper_2503_06671_amd import binding
from tests import block_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
# N, K, M, H, W
SHAPES = [(1, 1, 1, 1, 1), (1, 3, 5, 1, 1), (67, 9, 4, 1, 1), (1, 16, 32, 1, 2), (3, 17, 33, 1, 3), (2, 64, 64, 7, 9), (1, 64, 192, 16, 16), (2, 33, 65, 5, 27),
          (9, 48, 40, 3, 5), (1, 129, 70, 11, 13), (2, 200, 96, 8, 31), (1, 15, 257, 4, 130), (1, 640, 130, 5, 8), (5, 7, 300, 2, 2), (1, 500, 8, 33, 1),
          (1, 64, 128, 64, 64), (40, 24, 24, 6, 7), (1, 1300, 20, 3, 3), (2, 201, 33, 1, 7), (5, 131, 40, 1, 1),
          (1, 322, 30, 90, 900), (3, 196, 29, 150, 301), (2, 270, 66, 130, 255), (300, 35, 40, 3, 11)]

# many pixels: two a lane, wide tiles, and the backward pass in one launch (up to 128 channels, 64 with fp32); every number of channels that has code of its own
LARGE = [(2, 30, 40, 301, 255), (2, 50, 100, 301, 255), (3, 64, 33, 150, 301), (2, 120, 70, 301, 255), (2, 155, 20, 301, 255), (2, 190, 100, 301, 255),
         (2, 24, 300, 301, 255), (1, 24, 300, 130, 257), (2, 210, 260, 301, 255), (1, 300, 60, 130, 200), (2, 300, 60, 301, 255), (2, 260, 129, 160, 161),
         (70, 100, 90, 31, 33), (45, 60, 130, 31, 33), (300, 140, 300, 8, 8)]


def inputs(shape, dtype, seed=0, whole=False):
    N, K, M, H, W = shape
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s, scale=1.0):
        if whole:
            return torch.randint(-4, 5, s, device="cuda", generator=g).float()
        return torch.randn(*s, device="cuda", generator=g) * scale

    return dict(x=normal(N, K, H, W).to(dtype), w=normal(M, K, scale=K ** -0.5), b=normal(M), residual=normal(N, M, H, W).to(dtype),
                grad_out=normal(N, M, H, W).to(dtype))


def workspace(shape, dtype, act="none"):
    return binding.new_pointwise_backward_workspace(*shape, dtype, act=act)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES + LARGE, ids=str)
def test_whole_numbers_are_exact(shape, dtype):
    # sums of products up to 16 stay below 2^24: every result is a whole number (rounded where its type is bf16)
    i = inputs(shape, dtype, whole=True)
    x, w, go = i["x"].double(), i["w"].double(), i["grad_out"].double()
    pre = torch.einsum("mk,nkhw->nmhw", w, x) + ref.each(i["b"])
    assert torch.equal(binding.pointwise_forward(i["x"], i["w"], i["b"]), pre.to(dtype))
    assert torch.equal(binding.pointwise_forward(i["x"], i["w"], i["b"], residual=i["residual"]), (pre + i["residual"].double()).to(dtype))
    assert torch.equal(binding.pointwise_forward(i["x"], i["w"]), (pre - ref.each(i["b"])).to(dtype))
    got = binding.pointwise_backward(i["x"], i["grad_out"], i["w"], workspace(shape, dtype), i["b"])
    assert torch.equal(got["grad_x"], torch.einsum("mk,nmhw->nkhw", w, go).to(dtype))
    assert torch.equal(got["grad_w"], torch.einsum("nmhw,nkhw->mk", go, x).float())
    assert torch.equal(got["grad_b"], go.sum((0, 2, 3)).float())


@pytest.mark.parametrize("shape, act", [(s, a) for s in SHAPES for a in ("none", "gelu", "silu")] + [(s, "gelu") for s in LARGE], ids=str)
@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_against_float64(shape, dtype, act):
    i = inputs(shape, dtype, 1)
    want = ref.product(i["x"], i["w"], i["b"], act, i["residual"], i["grad_out"])
    out = binding.pointwise_forward(i["x"], i["w"], i["b"], act, i["residual"])
    ref.check(out, want["out"], "out")
    ws = workspace(shape, dtype, act)
    got = binding.pointwise_backward(i["x"], i["grad_out"], i["w"], ws, i["b"], act)
    assert set(got) == {"grad_x", "grad_w", "grad_b"}
    for n in got:
        ref.check(got[n], want[n], n)
    again = binding.pointwise_backward(i["x"], i["grad_out"], i["w"], ws, i["b"], act)
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_fp32_results_hold_fp32_accuracy(act, dtype):
    # over the whole result: terms left out (2^-21 of a product at most, of either sign) and roundings (2^-24 of a partial sum each, some dozens)
    # are independent of one another, so they stay below 2^-20 of the 2-norm; a term of a value that went missing is 2^-15 of it
    shape = (2, 192, 130, 40, 43)
    i = inputs(shape, dtype, 2)
    want = ref.product(i["x"], i["w"], i["b"], act, None, i["grad_out"])
    got = binding.pointwise_backward(i["x"], i["grad_out"], i["w"], workspace(shape, dtype, act), i["b"], act)
    got["out"] = binding.pointwise_forward(i["x"], i["w"], i["b"], act)
    for n in ("grad_w", "grad_b", "out", "grad_x"):
        if got[n].dtype == torch.float32:
            off = ((got[n].double() - want[n][0]).norm() / want[n][0].norm()).item()
            assert off < 2.0 ** -20, (n, off)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 20, 12, 5, 9), (2, 70, 130, 16, 9), (30, 5, 6, 1, 3)], ids=str)
def test_slices_of_larger_tensors(shape, dtype, act):
    N, K, M, H, W = shape
    i = inputs(shape, dtype, 3)
    ws = workspace(shape, dtype, act)
    want = binding.pointwise_forward(i["x"], i["w"], i["b"], act, i["residual"])
    back = binding.pointwise_backward(i["x"], i["grad_out"], i["w"], ws, i["b"], act)

    def inside(t):
        room = torch.full((N, t.shape[1] + 3, H, W), 7.0, device="cuda", dtype=dtype)
        room[:, 1:-2] = t
        return room, room[:, 1:-2]

    x, res, go = (inside(i[n])[1] for n in ("x", "residual", "grad_out"))
    (oroom, out), (groom, gx) = inside(torch.zeros_like(i["grad_out"])), inside(torch.zeros_like(i["x"]))
    assert binding.pointwise_forward(x, i["w"], i["b"], act, res, out=out) is out
    got = binding.pointwise_backward(x, go, i["w"], ws, i["b"], act, grads=dict(grad_x=gx))
    assert torch.equal(out, want) and got["grad_x"] is gx and all(torch.equal(got[n], back[n]) for n in back)
    for room in (oroom, groom):
        assert (room[:, :1] == 7).all() and (room[:, -2:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 64, 40, 9, 17), (2, 60, 100, 301, 255), (1, 256, 72, 130, 257), (1, 512, 40, 3, 5), (1, 40, 256, 130, 257)], ids=str)
def test_weights_at_odd_addresses(shape, dtype):
    N, K, M, H, W = shape
    i = inputs(shape, dtype, 11)
    room, bias = torch.empty(M * K + 1, device="cuda"), torch.empty(M + 1, device="cuda")
    w, b, gw, gb = room[1:].view(M, K), bias[1:], torch.empty(M * K + 3, device="cuda")[3:].view(M, K), torch.empty(M + 1, device="cuda")[1:]
    w.copy_(i["w"]), b.copy_(i["b"])
    ws = workspace(shape, dtype, "gelu")
    assert torch.equal(binding.pointwise_forward(i["x"], w, b, "silu"), binding.pointwise_forward(i["x"], i["w"], i["b"], "silu"))
    want = binding.pointwise_backward(i["x"], i["grad_out"], i["w"], ws, i["b"], "gelu")
    got = binding.pointwise_backward(i["x"], i["grad_out"], w, ws, b, "gelu", grads=dict(grad_w=gw, grad_b=gb), need=(n for n in ("grad_x", "grad_w", "grad_b")))
    assert got["grad_w"] is gw and got["grad_b"] is gb and all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_single_gradients_accumulation_and_buffers_full_of_nan(dtype):
    shape = (2, 40, 24, 13, 7)
    i = inputs(shape, dtype, 4)
    ws = workspace(shape, dtype, "gelu")
    args = (i["x"], i["grad_out"], i["w"], ws, i["b"], "gelu")
    all_of = binding.pointwise_backward(*args)
    for name in all_of:
        ws.view(torch.float32).fill_(math.nan)
        one = binding.pointwise_backward(*args, need=[name], grads={name: torch.full_like(all_of[name], math.nan)})
        assert torch.equal(one[name], all_of[name]) and set(one) == {name}
    mine = {n: torch.randn_like(all_of[n]) for n in ("grad_w", "grad_b")}
    start = {n: t.clone() for n, t in mine.items()}
    got = binding.pointwise_backward(*args, accumulate=True, grads=mine)
    for n in mine:
        assert got[n] is mine[n] and torch.equal(mine[n], start[n] + all_of[n])
    assert torch.equal(binding.pointwise_backward(*args, accumulate=True)["grad_w"], all_of["grad_w"])
    with pytest.raises(ValueError):
        binding.pointwise_backward(*args, accumulate=True, grads=dict(grad_w=mine["grad_w"]))
    assert set(binding.pointwise_backward(*args[:4], act="gelu")) == {"grad_x", "grad_w"}


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 20, 9, 6, 11), (1, 40, 70, 9, 129), (20, 33, 5, 1, 3)], ids=str)
def test_values_that_are_not_finite_reach_their_own_pixels_only(shape, dtype):
    N, K, M, H, W = shape
    i = inputs(shape, dtype, 5)
    bad = torch.zeros(N, H, W, dtype=torch.bool, device="cuda")
    for n, k, y, x, v in ((0, 2, 0, 1, math.nan), (N - 1, K - 1, H - 1, W - 1, math.inf), (0, 0, H - 1, 0, -math.inf)):
        i["x"][n, k, y, x] = v
        bad[n, y, x] = True
    out = binding.pointwise_forward(i["x"], i["w"], i["b"], residual=i["residual"])
    assert not torch.isfinite(out).any(1)[bad].any() and torch.isfinite(out).all(1)[~bad].all()
    # a row of w, and a pixel of grad_out
    i = inputs(shape, dtype, 6)
    i["w"][M - 1, 1] = math.nan
    out = binding.pointwise_forward(i["x"], i["w"], i["b"])
    assert torch.isnan(out[:, M - 1]).all() and torch.isfinite(out[:, :M - 1]).all()
    i = inputs(shape, dtype, 7)
    i["grad_out"][0, 1, 0, 0] = math.inf
    got = binding.pointwise_backward(i["x"], i["grad_out"], i["w"], workspace(shape, dtype), i["b"])
    assert not torch.isfinite(got["grad_x"][0, :, 0, 0]).any() and torch.isfinite(got["grad_x"]).sum() == got["grad_x"].numel() - K
    rows = torch.arange(M, device="cuda") == 1
    assert not torch.isfinite(got["grad_w"][rows]).any() and torch.isfinite(got["grad_w"][~rows]).all()
    assert not torch.isfinite(got["grad_b"][rows]).any() and torch.isfinite(got["grad_b"][~rows]).all()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_activations_over_their_whole_range(act):
    # one channel, weight one: out = act(x)
    v = torch.cat([torch.linspace(-12, 12, 4000), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 80.0, -80.0, 3e4, -3e4, 1e30, -1e30])]).cuda()
    x = v.view(1, 1, 1, -1)
    one, go = torch.ones(1, 1, device="cuda"), torch.ones_like(x)
    want = ref.product(x, one, None, act, None, go)
    ref.check(binding.pointwise_forward(x, one, act=act), want["out"], act)
    got = binding.pointwise_backward(x, go, one, workspace((1, 1, 1, 1, x.shape[3]), torch.float32, act), act=act, need=("grad_x",))["grad_x"]
    ref.check(got, want["grad_x"], act)


def test_small_and_large_values():
    # three terms are exact from 2^-110 on; nothing rounds up to an infinity
    for scale, top in ((2.0 ** -60, 1.0), (2.0 ** 60, 1.0), (1.0, 2.0 ** 127)):
        shape = (1, 20, 6, 5, 9)
        i = inputs(shape, torch.float32, 8)
        x = i["x"] * scale
        w = i["w"]
        if top != 1.0:
            x = torch.full_like(x, 3.4e38)
            w = torch.zeros_like(w)
            w[:, 3] = 0.5
        ref.check(binding.pointwise_forward(x, w), ref.product(x, w)["out"], scale)


@pytest.mark.parametrize("act", ["none", "gelu"])
def test_images_far_apart(act):
    # more than 2^32 elements from image to image
    shape = (2, 48, 40, 16, 9)
    i = inputs(shape, torch.bfloat16, 9)
    room = torch.empty(2 ** 32 + 2 ** 20, device="cuda", dtype=torch.bfloat16)
    x = torch.as_strided(room, (2, 48, 16, 9), (2 ** 32 + 64, 144, 9, 1))
    x.copy_(i["x"])
    want = ref.product(i["x"], i["w"], i["b"], act, None, i["grad_out"])
    ref.check(binding.pointwise_forward(x, i["w"], i["b"], act), want["out"], "out")
    got = binding.pointwise_backward(x, i["grad_out"], i["w"], workspace(shape, torch.bfloat16, act), i["b"], act)
    for n in got:
        ref.check(got[n], want[n], n)


def test_an_image_beyond_32_bits():
    K, M, H, W = 40, 34, 8192, 8200
    x = torch.empty(1, K, H, W, device="cuda", dtype=torch.bfloat16)
    for k in range(K):
        x[0, k].normal_()
    w = torch.randn(M, K, device="cuda")
    out = binding.pointwise_forward(x, w)
    for y, rows in ((0, 3), (4100, 2), (H - 2, 2)):
        ref.check(out[:, :, y:y + rows], ref.product(x[:, :, y:y + rows], w)["out"], "out")
    # The gradients, of signs and zeros.  A share of the pixels (one of 512) has a whole sum far below 2^24, exact; shares are added 16 in a row and
    # then in five halvings.  Where out follows x the shares' sums have one sign, up to 67 million in all: beyond 2^24 each of those 21 additions is off by
    # 2^-24 of what it adds up at most; sums below 2^23 stay exact (their partial sums too, which have the same sign or are the few thousands of chance).
    x.copy_(torch.sign(x) * (x.abs() > 0.4))
    go = torch.sign(out) * (out.abs() > 0.5)
    del out
    got = binding.pointwise_backward(x, go, w, workspace((1, K, M, H, W), torch.bfloat16))
    want = sum(go[0, :, y:y + 1024].reshape(M, -1).double() @ x[0, :, y:y + 1024].reshape(K, -1).double().t().contiguous() for y in range(0, H, 1024))
    off, small = (got["grad_w"].double() - want).abs(), want.abs() < 2 ** 23
    assert small.sum() > 300 and (off[small] == 0).all() and (off <= 21 * 2.0 ** -24 * H * W).all()
    for y, rows in ((0, 3), (4100, 2), (H - 2, 2)):
        part = ref.product(x[:, :, y:y + rows], w, None, "none", None, go[:, :, y:y + rows])
        ref.check(got["grad_x"][:, :, y:y + rows], part["grad_x"], "grad_x")


def test_streams_and_two_at_once():
    shapes = [(2, 64, 128, 31, 30), (3, 30, 64, 33, 9)]
    i = [inputs(s, torch.float32, 10 + k) for k, s in enumerate(shapes)]
    ws = [workspace(s, torch.float32, "gelu") for s in shapes]

    def work(k):
        a = i[k]
        got = binding.pointwise_backward(a["x"], a["grad_out"], a["w"], ws[k], a["b"], "gelu")
        return [binding.pointwise_forward(a["x"], a["w"], a["b"], "gelu", a["residual"]), *got.values()]

    want = [work(0), work(1)]
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = [None, None]
    for _ in range(3):
        for k, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got[k] = work(k)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k in (0, 1) for a, b in zip(want[k], got[k]))


def test_binding_refuses():
    shape = (2, 6, 5, 4, 4)
    i = inputs(shape, torch.float32)
    ws = workspace(shape, torch.float32)
    x, w, b, go = i["x"], i["w"], i["b"], i["grad_out"]
    for error, call in [
        (TypeError, lambda: binding.pointwise_forward(x.half(), w)),
        (TypeError, lambda: binding.pointwise_forward(x.transpose(2, 3), w)),
        (TypeError, lambda: binding.pointwise_forward(x, w.bfloat16())),
        (TypeError, lambda: binding.pointwise_forward(x, w.cpu())),
        (TypeError, lambda: binding.pointwise_forward(x, w.t())),
        (ValueError, lambda: binding.pointwise_forward(x, w[:, :5].contiguous())),
        (ValueError, lambda: binding.pointwise_forward(x, w, b[:4].contiguous())),
        (ValueError, lambda: binding.pointwise_forward(x, w, b, "tanh")),
        (ValueError, lambda: binding.pointwise_forward(x, w, residual=x)),
        (TypeError, lambda: binding.pointwise_forward(x, w, residual=go.bfloat16())),
        (ValueError, lambda: binding.pointwise_forward(x, w, out=torch.empty_like(x))),
        (binding.EscError, lambda: binding.pointwise_forward(x, torch.randn(6, 6, device="cuda"), out=x)),
        (binding.EscError, lambda: binding.pointwise_forward(x, w, residual=go, out=go)),
        (ValueError, lambda: binding.pointwise_backward(x, x, w, ws)),
        (binding.EscError, lambda: binding.pointwise_backward(x, go, w, ws[:128])),
        (binding.EscError, lambda: binding.pointwise_backward(x, go, w, ws, act="gelu")),  # (a workspace for none is too small)
        (binding.EscError, lambda: binding.pointwise_backward(x, go, w, ws, need=())),
        (ValueError, lambda: binding.pointwise_backward(x, go, w, ws, need=("grad_y",))),
        (ValueError, lambda: binding.pointwise_backward(x, go, w, ws, need="grad_x")),
        (ValueError, lambda: binding.pointwise_backward(x, go, w, ws, grads=dict(grad_w=b))),
        (TypeError, lambda: binding.pointwise_backward(x, go, w, ws, grads=dict(grad_w=w.double()))),
    ]:
        with pytest.raises(error):
            call()
