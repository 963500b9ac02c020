"""The float64 forms that the GPU tests compare with, pinned by something other than themselves."""
import math

import pytest
import torch

from tests import block_reference as ref


def test_philox_against_published_numbers():
    # the known answers that the generator's authors publish with it (ten rounds)
    assert ref.philox(0, 0, 0) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 2 ** 64 - 1
    assert ref.philox(ones, ones, ones) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert ref.philox(0x85A308D3243F6A88, 0x0370734413198A2E, 0x299F31D0A4093822) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_draws_are_even():
    d = ref.draws(40000, seed=5, offset=9).double()
    # mean and share below a quarter of uniform draws, within five standard deviations
    assert abs(d.mean().item() / 65535 - 0.5) < 5 * math.sqrt(1 / 12 / 40000)
    assert abs((d < 16384).double().mean().item() - 0.25) < 5 * math.sqrt(0.25 * 0.75 / 40000)
    assert not torch.equal(ref.draws(64, 5, 10), ref.draws(64, 5, 9)) and not torch.equal(ref.draws(64, 6, 9), ref.draws(64, 5, 9))
    assert torch.equal(ref.draws(20, 5, 9, first=13), ref.draws(40, 5, 9)[13:33])


@pytest.mark.parametrize("affine", [False, True])
def test_norm_is_the_library_routine_and_its_gradients(affine):
    g = torch.Generator().manual_seed(0)
    x = torch.randn(2, 7, 3, 4, generator=g, dtype=torch.float64).float().requires_grad_()
    w, b = (torch.randn(7, generator=g).requires_grad_() if affine else None for _ in range(2))
    go, skip = torch.randn(2, 7, 3, 4, generator=g), torch.randn(2, 7, 3, 4, generator=g)
    x64 = x.double()
    y = torch.nn.functional.layer_norm(x64.permute(0, 2, 3, 1), (7,), None if w is None else w.double(), None if b is None else b.double(), 1e-3)
    y = y.permute(0, 3, 1, 2)
    (y * go).sum().backward()
    got = ref.norm(x.detach(), None if w is None else w.detach(), None if b is None else b.detach(), 1e-3, go, skip)
    assert (got["out"][0] - y).abs().max() < 1e-12
    assert (got["grad_x"][0] - skip - x.grad).abs().max() < 1e-5
    if affine:
        assert (got["grad_weight"][0] - w.grad).abs().max() < 1e-5 and (got["grad_bias"][0] - b.grad).abs().max() < 1e-5


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_product_is_the_library_convolution_and_differences(act):
    g = torch.Generator().manual_seed(1)
    x, w, b, go = torch.randn(2, 5, 3, 4, generator=g), torch.randn(6, 5, generator=g), torch.randn(6, generator=g), torch.randn(2, 6, 3, 4, generator=g)
    res = torch.randn(2, 6, 3, 4, generator=g)
    f = {"none": lambda v: v, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[act]

    def forward(x, w, b):
        return f(torch.nn.functional.conv2d(x, w[:, :, None, None], b)) + res.double()

    t = [v.double() for v in (x, w, b)]
    got = ref.product(x, w, b, act, res, go)
    assert (got["out"][0] - forward(*t)).abs().max() < 1e-12
    for i, name in enumerate(("grad_x", "grad_w", "grad_b")):
        d = torch.randn(t[i].shape, generator=g, dtype=torch.float64)
        h = 1e-6
        up, down = ([v + s * h * d if j == i else v for j, v in enumerate(t)] for s in (1, -1))
        difference = ((forward(*up) - forward(*down)) * go).sum() / (2 * h)
        assert abs((got[name][0] * d).sum() - difference) < 1e-6, name
