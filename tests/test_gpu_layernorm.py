"""Layer norm over the channels of each pixel and its gradients against float64, within what fp32 sums and the roundings may be off by."""
import math

import pytest
import torch

from paper_2503_06671_amd import binding
from tests import block_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
# N, C, H, W: one token; few; rows that are no whole lanes; many channels; large and small images
SHAPES = [(1, 1, 1, 1), (1, 3, 1, 1), (70, 5, 1, 1), (2, 7, 3, 5), (1, 64, 16, 16), (3, 64, 9, 31), (2, 45, 33, 17), (1, 192, 20, 36), (5, 193, 3, 3),
          (1, 256, 1, 63), (1, 257, 8, 8), (2, 640, 5, 13), (1, 1025, 4, 4), (2, 2500, 1, 3), (1, 16, 130, 129), (33, 12, 7, 1), (1, 100, 1, 4097)]

# enough pixels for four of a lane (or two): every number of channels that has code of its own
LARGE = [(2, C, 93, 91) for C in (15, 32, 47, 64, 94, 128, 190, 256, 380, 512, 700, 1000)] + [(1, 1100, 128, 130)]


def inputs(shape, dtype, seed=0, mean=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    N, C, H, W = shape

    def normal(*s):
        return torch.randn(*s, device="cuda", generator=g)

    size = torch.exp(0.5 * normal(C, 1, 1))
    return dict(x=((normal(*shape) + mean * normal(C, 1, 1)) * size).to(dtype), weight=1 + 0.3 * normal(C), bias=normal(C), grad_out=normal(*shape).to(dtype),
                skip=normal(*shape).to(dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES + LARGE + [(3, C, 5, 7) for _, C, _, _ in LARGE], ids=str)
def test_against_float64(shape, dtype):
    i = inputs(shape, dtype)
    N, C, H, W = shape
    saved, ws = binding.new_layernorm_saved(N, H, W), binding.new_layernorm_backward_workspace(N, C, H, W)
    want = ref.norm(i["x"], i["weight"], i["bias"], 1e-4, i["grad_out"], i["skip"])
    out = binding.layernorm_forward(i["x"], i["weight"], i["bias"], 1e-4, saved=saved)
    ref.check(out, want["out"], "out")
    assert torch.equal(out, binding.layernorm_forward(i["x"], i["weight"], i["bias"], 1e-4))
    got = binding.layernorm_backward(i["x"], i["grad_out"], saved, ws, i["weight"], i["bias"], grad_skip=i["skip"])
    assert set(got) == {"grad_x", "grad_weight", "grad_bias"}
    for n in got:
        ref.check(got[n], want[n], n)
    again = binding.layernorm_backward(i["x"], i["grad_out"], saved, ws, i["weight"], i["bias"], grad_skip=i["skip"])
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 64, 6, 11), (1, 300, 5, 5), (4, 2000, 2, 3)], ids=str)
def test_without_weight_or_bias_or_skip_and_single_gradients(shape, dtype):
    i = inputs(shape, dtype, 1)
    N, C, H, W = shape
    saved, ws = binding.new_layernorm_saved(N, H, W), binding.new_layernorm_backward_workspace(N, C, H, W)
    for weight, bias in ((None, None), (i["weight"], None), (None, i["bias"])):
        want = ref.norm(i["x"], weight, bias, grad_out=i["grad_out"])
        ref.check(binding.layernorm_forward(i["x"], weight, bias, saved=saved), want["out"], "out")
        got = binding.layernorm_backward(i["x"], i["grad_out"], saved, ws, weight, bias)
        assert set(got) == {"grad_x"} | ({"grad_weight"} if weight is not None else set()) | ({"grad_bias"} if bias is not None else set())
        for n in got:
            ref.check(got[n], want[n], n)
    both = binding.layernorm_backward(i["x"], i["grad_out"], saved, ws, i["weight"], i["bias"])
    for name in both:
        one = binding.layernorm_backward(i["x"], i["grad_out"], saved, ws, i["weight"], i["bias"], need=(name,))
        assert set(one) == {name} and torch.equal(one[name], both[name])


def test_accumulate_and_given_buffers():
    shape = (2, 40, 7, 9)
    i = inputs(shape, torch.float32, 2)
    saved, ws = binding.new_layernorm_saved(2, 7, 9), binding.new_layernorm_backward_workspace(*shape)
    binding.layernorm_forward(i["x"], i["weight"], i["bias"], saved=saved)
    args = (i["x"], i["grad_out"], saved, ws, i["weight"], i["bias"])
    plain = binding.layernorm_backward(*args)
    mine = {n: torch.randn_like(t) for n, t in plain.items()}
    start = {n: t.clone() for n, t in mine.items()}
    got = binding.layernorm_backward(*args, accumulate=True, grads=mine)
    assert all(got[n] is mine[n] for n in got) and torch.equal(got["grad_x"], plain["grad_x"])
    for n in ("grad_weight", "grad_bias"):
        assert torch.equal(got[n], start[n] + plain[n])
    assert torch.equal(binding.layernorm_backward(*args, accumulate=True)["grad_bias"], plain["grad_bias"])  # (nothing there to add to)
    with pytest.raises(ValueError):
        binding.layernorm_backward(*args, accumulate=True, grads=dict(grad_bias=mine["grad_bias"]))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("C", [5, 64, 190, 400])
def test_slices_of_larger_tensors(C, dtype):
    # images apart from one another, at odd addresses; nothing beside them is touched
    i = inputs((3, C, 5, 9), dtype, 3)
    saved, ws = binding.new_layernorm_saved(3, 5, 9), binding.new_layernorm_backward_workspace(3, C, 5, 9)

    def inside(t):
        room = torch.full((3, C + 3, 5, 9), 7.0, device="cuda", dtype=dtype)
        room[:, 1:1 + C] = t
        return room, room[:, 1:1 + C]

    want = binding.layernorm_forward(i["x"], i["weight"], i["bias"], saved=saved)
    back = binding.layernorm_backward(i["x"], i["grad_out"], saved, ws, i["weight"], i["bias"], grad_skip=i["skip"])
    x, go, skip = (inside(i[n])[1] for n in ("x", "grad_out", "skip"))
    (oroom, out), (groom, gx) = inside(torch.zeros_like(i["x"])), inside(torch.zeros_like(i["x"]))
    assert binding.layernorm_forward(x, i["weight"], i["bias"], saved=saved, out=out) is out
    got = binding.layernorm_backward(x, go, saved, ws, i["weight"], i["bias"], grad_skip=skip, grads=dict(grad_x=gx))
    assert torch.equal(out, want) and all(torch.equal(got[n], back[n]) for n in back)
    for room in (oroom, groom):
        assert (room[:, :1] == 7).all() and (room[:, 1 + C:] == 7).all()


@pytest.mark.parametrize("C", [6, 64, 200, 500])
def test_values_that_are_not_finite_stay_in_their_pixel(C):
    i = inputs((2, C, 7, 11), torch.float32, 4)
    i["x"][0, 3, 2, 5], i["x"][1, 0, 6, 10], i["x"][1, C - 1, 0, 0] = math.nan, math.inf, -math.inf
    bad = torch.zeros(2, 7, 11, dtype=torch.bool, device="cuda")
    bad[0, 2, 5] = bad[1, 6, 10] = bad[1, 0, 0] = True
    saved, ws = binding.new_layernorm_saved(2, 7, 11), binding.new_layernorm_backward_workspace(2, C, 7, 11)
    out = binding.layernorm_forward(i["x"], i["weight"], i["bias"], saved=saved)
    gx = binding.layernorm_backward(i["x"], i["grad_out"], saved, ws, i["weight"], i["bias"], need=("grad_x",))["grad_x"]
    clean = torch.where(bad[:, None], torch.ones_like(i["x"]), i["x"])
    want = ref.norm(clean, i["weight"], i["bias"], grad_out=i["grad_out"])
    for got, name in ((out, "out"), (gx, "grad_x")):
        assert torch.isnan(got).any(1)[bad].all() and torch.isfinite(got).all(1)[~bad].all()
        ref.check(torch.where(bad[:, None], want[name][0].float(), got), want[name], name)


@pytest.mark.parametrize("scale", [1e-18, 1e-3, 1e15])
def test_small_and_large_values(scale):
    # (squares of differences stay in fp32's range)
    i = inputs((1, 70, 9, 9), torch.float32, 5)
    x = i["x"] * scale
    saved = binding.new_layernorm_saved(1, 9, 9)
    ref.check(binding.layernorm_forward(x, i["weight"], i["bias"], 1e-12, saved=saved), ref.norm(x, i["weight"], i["bias"], 1e-12)["out"], "out")


def test_a_mean_far_from_zero():
    # differences, not squares: the error is what the mean's rounding makes it, not the square of that
    i = inputs((1, 64, 12, 12), torch.float32, 6)
    x = i["x"] + 4096.0
    saved, ws = binding.new_layernorm_saved(1, 12, 12), binding.new_layernorm_backward_workspace(1, 64, 12, 12)
    want = ref.norm(x, i["weight"], i["bias"], grad_out=i["grad_out"])
    ref.check(binding.layernorm_forward(x, i["weight"], i["bias"], saved=saved), want["out"], "out")
    got = binding.layernorm_backward(x, i["grad_out"], saved, ws, i["weight"], i["bias"])
    for n in got:
        ref.check(got[n], want[n], n)


@pytest.mark.parametrize("C", [48, 700])
def test_images_and_channels_far_apart(C):
    # images more than 2^32 elements apart; with 48 channels also planes beyond 2^32 bytes of an image
    room = torch.empty(2 ** 32 + 2 ** 20 * 1, device="cuda", dtype=torch.bfloat16)
    x = torch.as_strided(room, (2, C, 16, 9), (2 ** 32 + 64, 144, 9, 1))
    i = inputs((2, C, 16, 9), torch.bfloat16, 7)
    x.copy_(i["x"])
    saved, ws = binding.new_layernorm_saved(2, 16, 9), binding.new_layernorm_backward_workspace(2, C, 16, 9)
    want = ref.norm(i["x"], i["weight"], i["bias"], grad_out=i["grad_out"])
    ref.check(binding.layernorm_forward(x, i["weight"], i["bias"], saved=saved), want["out"], "out")
    got = binding.layernorm_backward(x, i["grad_out"], saved, ws, i["weight"], i["bias"])
    for n in got:
        ref.check(got[n], want[n], n)


def test_an_image_beyond_32_bits():
    C, H, W = 40, 8192, 8200
    x = torch.empty(1, C, H, W, device="cuda", dtype=torch.bfloat16)
    for c in range(C):
        x[0, c].normal_(mean=0.1 * c)
    saved = binding.new_layernorm_saved(1, H, W)
    out = binding.layernorm_forward(x, saved=saved)
    go = x.flip(1)
    gx = binding.layernorm_backward(x, go, saved, binding.new_layernorm_backward_workspace(1, C, H, W), need=("grad_x",))["grad_x"]
    for y, rows in ((0, 3), (4100, 2), (H - 2, 2)):
        want = ref.norm(x[:, :, y:y + rows], grad_out=go[:, :, y:y + rows])
        ref.check(out[:, :, y:y + rows], want["out"], "out")
        ref.check(gx[:, :, y:y + rows], want["grad_x"], "grad_x")


def test_streams():
    # no stream given: the current one, behind what it still has to do; a stream given: that one
    later = inputs((2, 64, 30, 31), torch.float32, 8)
    want = binding.layernorm_forward(later["x"], later["weight"], later["bias"])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for given in (False, True):
        x, big = torch.zeros_like(later["x"]), torch.randn(4096, 4096, device="cuda")
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(10):
                big = big @ big * 1e-4
            x.copy_(later["x"])
            if not given:
                got = binding.layernorm_forward(x, later["weight"], later["bias"])
        if given:
            got = torch.empty_like(x)
            s.wait_stream(torch.cuda.current_stream())
            binding.layernorm_forward(x, later["weight"], later["bias"], out=got, stream=s)
        s.synchronize()
        assert torch.equal(got, want)


def test_binding_refuses():
    i = inputs((2, 6, 4, 4), torch.float32)
    saved, ws = binding.new_layernorm_saved(2, 4, 4), binding.new_layernorm_backward_workspace(2, 6, 4, 4)
    x, go, w = i["x"], i["grad_out"], i["weight"]
    for error, call in [
        (TypeError, lambda: binding.layernorm_forward(x.half())),
        (TypeError, lambda: binding.layernorm_forward(x.transpose(2, 3))),
        (TypeError, lambda: binding.layernorm_forward(x[0])),
        (TypeError, lambda: binding.layernorm_forward(x, w.double())),
        (ValueError, lambda: binding.layernorm_forward(x, w[:5].contiguous())),
        (ValueError, lambda: binding.layernorm_forward(x, out=torch.empty(2, 6, 4, 5, device="cuda"))),
        (TypeError, lambda: binding.layernorm_forward(x, out=torch.empty_like(x, dtype=torch.bfloat16))),
        (TypeError, lambda: binding.layernorm_forward(x, saved=saved.cpu())),
        (binding.EscError, lambda: binding.layernorm_forward(x, out=x)),
        (binding.EscError, lambda: binding.layernorm_forward(x, eps=0)),
        (binding.EscError, lambda: binding.layernorm_forward(x, saved=saved[:64])),
        (ValueError, lambda: binding.layernorm_backward(x, go[:1], saved, ws)),
        (TypeError, lambda: binding.layernorm_backward(x, go.bfloat16(), saved, ws)),
        (binding.EscError, lambda: binding.layernorm_backward(x, go, saved, ws[:0])),
        (binding.EscError, lambda: binding.layernorm_backward(x, go, saved, ws, need=())),
        (ValueError, lambda: binding.layernorm_backward(x, go, saved, ws, need=("grad_y",))),
        (ValueError, lambda: binding.layernorm_backward(x, go, saved, ws, need="grad_x")),
        (binding.EscError, lambda: binding.layernorm_backward(x, go, saved, ws, grads=dict(grad_x=go))),
    ]:
        with pytest.raises(error):
            call()
