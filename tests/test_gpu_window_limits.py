"""Window attention at the ends of what its calls accept."""
import pytest
import torch

from paper_2503_06671_amd import binding
from tests.test_gpu_window_attention import BF16, NAMES, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [(4200, 4100), (8192, 3), (1, 8192)])
def test_windows_far_larger_than_the_map(window):
    # all but the few buckets of the map's own offsets are empty; those are what a window of the map's size gives
    N, H, W, heads = 2, 9, 7, 2
    if window[0] == 1:
        H = 1
    c = Case(torch.float32, N, H, W, heads, 16, window, seed=500)
    h, w = min(H, window[0]), min(W, window[1])
    middle = slice(None), slice(window[0] - h, window[0] + h - 1), slice(window[1] - w, window[1] + w - 1)
    same = Case(torch.float32, N, H, W, heads, 16, (h, w), seed=500)
    for a, b in ((same.q, c.q), (same.k, c.k), (same.v, c.v), (same.go, c.go)):
        a.copy_(b)
    same.bias.copy_(c.bias[middle])
    got, want = c.train(), same.train()
    for n in NAMES[:4]:
        assert torch.equal(got[n], want[n]), n
    rest = got["grad_bias"].clone()
    assert torch.equal(rest[middle], want["grad_bias"]) and (want["grad_bias"] != 0).any()
    rest[middle] = 0
    assert (rest == 0).all()
    again = c.train(accumulate=True, grads={"grad_bias": got["grad_bias"]})["grad_bias"]
    assert torch.equal(again[middle], 2 * want["grad_bias"])


def test_gradients_of_images_more_than_32_bits_apart():
    c = Case(BF16, 2, 16, 16, 1, 16, (16, 16), seed=510)
    want = c.train()
    step, image = 2 ** 31 + 24, 16 * 256
    room = torch.full((step + 3 * image,), 3.0, device="cuda", dtype=BF16)
    grads = {n: room.as_strided((2, 16, 16, 16), (step, 256, 16, 1), i * image) for i, n in enumerate(NAMES[1:4])}
    got = c.train(grads=grads)
    for n in NAMES[1:]:
        assert torch.equal(got[n], want[n]), n
        assert n == "grad_bias" or got[n] is grads[n]
    between = room[3 * image:step]
    assert between.amin() == 3 and between.amax() == 3
