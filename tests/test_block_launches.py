"""Launches of layer norm, the point-wise product and dropout at sizes up to the documented limits: a launch has fewer than 2^32 threads a dimension."""
import pytest

from tests import launches

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


def test_what_fits_a_card_is_taken(program):
    # (288 GB, bf16)
    calls = [(name, 1, N, K, M, H, W, 0, 0) for name in launches.CALLS for N, H, W in EXTENTS for K, M in ((1, 1), (3, 3), (16, 40), (17, 300), (1000, 1), (1, 65536))
             if N * H * W * (K + (M if "pointwise" in name else K)) * 2 < 288e9]
    assert len(calls) > 200
    for call, (status, _) in zip(calls, launches.ask(program, calls)):
        assert status == OK, call
