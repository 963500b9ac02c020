"""Dropout from the counter-based generator: equal to the same operations one by one, with the generator's words in whole numbers of Python."""
import math

import pytest
import torch

from paper_2503_06671_amd import binding
from tests import block_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
SHAPES = [(1, 1, 1, 1), (1, 1, 1, 7), (3, 5, 1, 1), (2, 3, 5, 7), (1, 4, 16, 16), (4, 9, 23, 25), (2, 3, 24, 25), (1, 2, 67, 65)]


def inputs(shape, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(*shape, generator=g).to(dtype) for _ in range(3)]


@pytest.mark.parametrize("over", ["element", "plane", "image"])
@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_equal_to_the_definition(shape, dtype, over):
    x, res, go = inputs(shape, dtype)
    seed, offset = 0xFEDCBA9876543210, 2 ** 40 + 3
    for p in (0.0, 0.3, 0.5, 0.9):
        kw = dict(p=p, seed=seed, offset=offset, over=over)
        assert torch.equal(binding.dropout_forward(x.cuda(), residual=res.cuda(), **kw).cpu(), ref.dropout(x, p, seed, offset, over, res)), p
        assert torch.equal(binding.dropout_forward(x.cuda(), **kw).cpu(), ref.dropout(x, p, seed, offset, over)), p
        assert torch.equal(binding.dropout_backward(go.cuda(), **kw).cpu(), ref.dropout(go, p, seed, offset, over)), p


@pytest.mark.parametrize("over", ["element", "plane", "image"])
@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 5, 3, 7), (4, 2, 30, 31), (5, 1, 1, 3), (3, 5, 63, 45), (2, 45, 15, 15)], ids=str)
def test_masks_do_not_depend_on_strides(shape, dtype, over):
    x, res, go = inputs(shape, dtype, 1)
    N, C, H, W = shape
    kw = dict(p=0.4, seed=7, offset=1, over=over)

    def inside(t):
        room = torch.full((N, C + 3, H, W), 7.0, device="cuda", dtype=dtype)
        room[:, 1:1 + C] = t.cuda()
        return room, room[:, 1:1 + C]

    (room, out), (groom, gx) = inside(torch.zeros_like(x)), inside(torch.zeros_like(x))
    assert binding.dropout_forward(inside(x)[1], residual=inside(res)[1], out=out, **kw) is out
    assert binding.dropout_backward(inside(go)[1], grad_x=gx, **kw) is gx
    assert torch.equal(out.cpu(), ref.dropout(x, 0.4, 7, 1, over, res)) and torch.equal(gx.cpu(), ref.dropout(go, 0.4, 7, 1, over))
    for r in (room, groom):
        assert (r[:, :1] == 7).all() and (r[:, 1 + C:] == 7).all()
    # one side contiguous, the other not
    assert torch.equal(binding.dropout_forward(inside(x)[1], residual=res.cuda(), **kw), out)


def test_dropped_values_count_as_zero_whatever_they_are():
    x = torch.full((1, 8, 8, 8), math.nan)
    keep = ref.kept(x.shape, 0.5, 3, 4, "element")
    x[keep] = 1.5
    for over in ("element",):
        out = binding.dropout_forward(x.cuda(), 0.5, 3, 4, over=over).cpu()
        assert torch.equal(out, torch.where(keep, torch.tensor(3.0), torch.tensor(0.0)))
    x = torch.full((6, 2, 25, 25), math.inf)
    keep = ref.kept(x.shape, 0.5, 3, 4, "image")
    assert keep.any() and not keep.all()
    x[keep] = 1.0
    assert torch.equal(binding.dropout_forward(x.cuda(), 0.5, 3, 4, over="image", residual=torch.ones_like(x).cuda()).cpu(), 1 + 2 * keep.float())


@pytest.mark.parametrize("over", ["element", "plane"])
def test_offsets_on_the_device_and_in_replayed_graphs(over):
    shape = (3, 6, 9, 11)
    x, res, go = inputs(shape, torch.float32, 2)
    dx, dres, dgo, out, gx = x.cuda(), res.cuda(), go.cuda(), torch.empty(shape, device="cuda"), torch.empty(shape, device="cuda")
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    kw = dict(p=0.25, seed=11, offset=2 ** 32 - 2, offset_device=count, over=over)

    def step():
        binding.dropout_forward(dx, residual=dres, out=out, **kw)
        binding.dropout_backward(dgo, grad_x=gx, **kw)
        count.add_(2)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    seen = [out.clone()]
    for k in range(1, 5):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), ref.dropout(x, 0.25, 11, 2 ** 32 - 2 + 2 * k, over, res))
        assert torch.equal(gx.cpu(), ref.dropout(go, 0.25, 11, 2 ** 32 - 2 + 2 * k, over))
        assert not any(torch.equal(out, o) for o in seen)
        seen.append(out.clone())
    assert count.item() == 10


def test_offsets_count_modulo_64_bits():
    x, _, _ = inputs((1, 2, 5, 5), torch.float32, 3)
    count = torch.tensor([-1], device="cuda")
    out = binding.dropout_forward(x.cuda(), 0.5, 1, 2 ** 64 - 1, offset_device=count)
    assert torch.equal(out.cpu(), ref.dropout(x, 0.5, 1, 2 ** 64 - 2, "element"))


def test_elements_beyond_32_bits():
    N, C, H, W = 3, 20, 8192, 8200
    x = torch.ones(N, C, H, W, device="cuda", dtype=torch.bfloat16)
    out = binding.dropout_forward(x, 0.5, 5, 6)
    flat = out.view(-1)
    for first in (0, 2 ** 31 - 40, 2 ** 32 - 40, flat.numel() - 333):
        n = min(400, flat.numel() - first)
        keep = ref.draws(n, 5, 6, first=first) >= 32768
        assert torch.equal(flat[first:first + n].cpu(), torch.where(keep, 2.0, 0.0).bfloat16())
    share = sum((out[n, c] == 0).sum().item() for n in range(N) for c in range(C)) / out.numel()
    assert abs(share - 0.5) < 5 * 0.5 / math.sqrt(out.numel())
    del out, flat
    # images more than 2^32 elements apart
    y, _, _ = inputs((2, 5, 7, 9), torch.bfloat16, 4)
    room = x.view(-1)
    far = torch.as_strided(room, (2, 5, 7, 9), (2 ** 31 + 2 ** 30 + 64, 63, 9, 1))
    far.copy_(y)
    for over in ("element", "plane", "image"):
        assert torch.equal(binding.dropout_forward(far, 0.4, 5, 6, over=over).cpu(), ref.dropout(y, 0.4, 5, 6, over))


def test_binding_refuses():
    x = torch.randn(2, 6, 4, 4, device="cuda")
    one = torch.zeros(1, dtype=torch.int64, device="cuda")
    for error, call in [
        (TypeError, lambda: binding.dropout_forward(x.half(), 0.5, 1)),
        (TypeError, lambda: binding.dropout_forward(x.transpose(2, 3), 0.5, 1)),
        (TypeError, lambda: binding.dropout_forward(x, "half", 1)),
        (TypeError, lambda: binding.dropout_forward(x, 0.5, 1.5)),
        (ValueError, lambda: binding.dropout_forward(x, 0.5, -1)),
        (ValueError, lambda: binding.dropout_forward(x, 0.5, 1, 2 ** 64)),
        (ValueError, lambda: binding.dropout_forward(x, 0.5, 1, over="row")),
        (TypeError, lambda: binding.dropout_forward(x, 0.5, 1, offset_device=one.int())),
        (TypeError, lambda: binding.dropout_forward(x, 0.5, 1, offset_device=one.cpu())),
        (ValueError, lambda: binding.dropout_forward(x, 0.5, 1, residual=x[:1])),
        (TypeError, lambda: binding.dropout_forward(x, 0.5, 1, residual=x.bfloat16())),
        (binding.EscError, lambda: binding.dropout_forward(x, 0.5, 1, out=x)),
        (binding.EscError, lambda: binding.dropout_forward(x, 1.0, 1)),
        (binding.EscError, lambda: binding.dropout_backward(x, -0.1, 1)),
    ]:
        with pytest.raises(error):
            call()
