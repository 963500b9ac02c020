"""Launches of layer norm, the point-wise product and dropout at sizes up to the documented limits: a launch has fewer than 2^32 threads a dimension."""
import re

import pytest

from tests import launches, product_limits
from tests.test_abi_host import kernel_notes, lib  # noqa: F401

OK, SHAPE, UNSUPPORTED = 0, 2, 4


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    p = launches.build(tmp_path_factory.mktemp("launches"))
    if p is None:
        pytest.skip("no hipcc")
    return p


# N, H, W: the fewest and the most blocks by images, by planes, and by both
EXTENTS = [(1, 1, 1), (1 << 24, 1, 1), (1 << 26, 1, 1), ((1 << 31) - 1, 1, 1), (1 << 22, 1, 1), (1 << 27, 1, 3), (1 << 24, 9, 9), (1 << 24, 96, 1), (1 << 20, 1000, 1), (2, 1 << 15, 1 << 15),
           (1 << 15, 256, 256), (1 << 8, 4096, 4096), (1 << 8, 4096, 4097), (1, 46341, 46339), (64, 46341, 46339), (500, 46341, 46339)]


@pytest.mark.parametrize("extent", EXTENTS, ids=str)
def test_no_launch_has_more_threads_than_there_may_be(program, extent):
    N, H, W = extent
    calls = [(name, dt, N, K, M, H, W, act, flag)
             for name in launches.CALLS for dt in (0, 1) for K, M in ((1, 1), (3, 3), (16, 40), (17, 300), (100, 20), (300, 129), (1000, 1), (8191, 65536), (65536, 2))
             for act in ((0, 1) if "pointwise" in name else (0, 1, 2) if "dropout" in name else (0,)) for flag in ((0, 1) if name in ("pointwise_forward", "dropout_forward") else (0,))]
    for call, (status, made) in zip(calls, launches.ask(program, calls)):
        far = N > 1 and max(call[3], call[4]) * H * W > 2 ** 46  # (images further apart than they may be)
        assert status == OK and made or status in ((SHAPE, UNSUPPORTED) if far else (UNSUPPORTED,)) and not made, (call, status, made)
        for l in made:
            assert 0 < l.gx * l.block < 2 ** 32 and 0 < l.gy < 2 ** 16 and l.gz == 1, (call, l)


def test_every_built_kernel_is_launched_at_some_size(program, lib):  # noqa: F811
    built = {k[0] for k in kernel_notes() if re.search("(product|strip|norm|dropout|parts)_(thin_|weights_|back_|any_)*kernel", k[0])}
    assert len(built) > 230
    extents = [(1, 3, 3), (1, 30, 30), (1, 64, 64), (1, 100, 130), (1, 130, 257), (2, 301, 255), (3, 150, 301), (5, 50, 61), (20, 31, 33), (700, 8, 8), (3000, 1, 2)]
    channels = [8, 16, 17, 30, 33, 49, 60, 70, 100, 129, 160, 190, 193, 260, 300, 385, 520, 770, 1100]
    calls = [(name, dt, N, K, 1, H, W, 0, 0) for name in ("layernorm_forward", "layernorm_backward") for dt in (0, 1) for N, H, W in extents for K in channels]
    calls += [("dropout_forward", dt, N, K, 1, H, W, over, flag) for dt in (0, 1) for N, H, W in extents for K in (5, 64) for over in (0, 1, 2) for flag in (0, 1)]
    calls += [(name, dt, N, K, M, H, W, act, flag) for name in ("pointwise_forward", "pointwise_backward") for dt in (0, 1) for N, H, W in extents
              for K in channels[:-4] for M in (8, 20, 33, 65, 130, 210, 300) for act in (0, 1) for flag in (0, 1)]
    reached = {l.kernel for _, made in launches.ask(program, calls) for l in made}
    assert built == reached, (built - reached, reached - built)


def test_what_fits_a_card_is_taken(program):
    # (288 GB, bf16)
    calls = [(name, 1, N, K, M, H, W, 0, 0) for name in launches.CALLS for N, H, W in EXTENTS for K, M in ((1, 1), (3, 3), (16, 40), (17, 300), (1000, 1), (1, 65536))
             if N * H * W * (K + (M if "pointwise" in name else K)) * 2 < 288e9]
    assert len(calls) > 200
    for call, (status, _) in zip(calls, launches.ask(program, calls)):
        assert status == OK, call


def test_sizes_beyond_32_bit_offsets_go_by_addresses(program):
    acts = {"none": 0, "gelu": 1, "silu": 2}
    for dt, K, M, H, W, act, forward, backward in product_limits.CASES:
        made = launches.ask(program, [(f"pointwise_{d}", dt, 1, K, M, H, W, acts[act], 0) for d in ("forward", "backward")])
        for (status, all_of), kernels in zip(made, (forward, backward)):
            names = [l.kernel for l in all_of if "weights" not in l.kernel and "parts" not in l.kernel]
            assert status == OK and names and all(re.search(kernels, n) for n in names), (dt, K, M, H, W, act, names)
