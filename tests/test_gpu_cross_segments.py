"""Cross attention of many segments, and larger calls outside the wide tiles of states; element by element against the formulas in 64 bits with the
bounds of test_gpu_cross.py."""
import numpy as np
import pytest
import torch

from paper_2508_21058_amd import binding as mb
from tests.test_gpu_cross import check, ran_wide

pytestmark = pytest.mark.gpu


def kernels_of(**call):
    """Kernels that the call's passes ran, its results having been checked."""
    mb.prof_enable(True)
    try:
        check(**call)
        return mb.prof_read()
    finally:
        mb.prof_enable(False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("S,other", [(65, ()), (128, ()), (100, range(60, 62)), (128, range(63, 65)), (128, range(64, 66)), (90, (0, 63, 64, 89))])
def test_short_segments_joined_across_a_wave(S, other, d, dtype):
    """Segments of zero to 23 queries with the range of their neighbours, but for a few; runs go across segments 63 and 64, or end there."""
    g = np.random.default_rng(S)
    offs = np.concatenate(([0], np.cumsum(g.integers(0, 24, S)))).tolist()
    ranges = [[(30, 75) if s in other else (0, 81) for s in range(S)], [(5, 5) if s in other else (3, 40) for s in range(S)]]
    check(2, 2, 1, offs[-1], 81, d, dtype, ranges=ranges, offs=offs)


@pytest.mark.parametrize("kind", ["distinct", "mixed", "equal"])
def test_wide_tiles_of_128_segments(kind):
    """All words of segments and more cuts than a workgroup has threads."""
    S, N, M, B = 128, 40_000, 1500, 2
    g = np.random.default_rng(5)
    offs = [0] + sorted(g.integers(0, N + 1, S - 1).tolist()) + [N]
    if kind == "distinct":
        one = lambda b, s: (11 * s + b, 11 * s + b + 11)
    elif kind == "equal":
        one = lambda b, s: (7, 1400 - 300 * b)
    else:       # wide, narrow, empty, reversed and past the states
        one = lambda b, s: [(8 * s, 8 * s + 400), (1500 - 10 * s, 1500), (s, s), (900, 20 * b), (-4, 5 + s), (700, 1 << 30)][(s + b) % 6]
    ranges = [[one(b, s) for s in range(S)] for b in range(B)]
    ran_wide(lambda: check(B, 12, 4, N, M, 128, torch.bfloat16, ranges=ranges, offs=offs))


SMALL_TILES = {
    "fp32, 128 features": dict(B=1, H=6, Hk=2, N=4100, M=333, d=128, dtype=torch.float32, offs=[0, 700, 701, 2900, 4100], ranges=[[(0, 333), (40, 41), (17, 300), (100, 100)]]),
    "fp32, 64 features": dict(B=3, H=4, Hk=4, N=3333, M=500, d=64, dtype=torch.float32, offs=[0, 1500, 3333], ranges=[[(0, 500), (0, 300)], [(0, 0), (499, 500)], [(33, 470), (33, 470)]]),
    "fp32, one segment": dict(B=2, H=12, Hk=4, N=2047, M=129, d=128, dtype=torch.float32, ranges=[[(0, 129)], [(0, 97)]]),
    "bf16, 64 features": dict(B=2, H=8, Hk=4, N=9001, M=700, d=64, dtype=torch.bfloat16, offs=[0, 31, 4000, 4032, 8999, 9001],
                              ranges=[[(0, 700), (5, 140), (0, 0), (139, 650), (699, 700)], [(0, 64)] * 5]),
    "bf16, 64 features, one segment": dict(B=1, H=6, Hk=6, N=12_345, M=257, d=64, dtype=torch.bfloat16),
    "bf16, 128 features, few states": dict(B=2, H=6, Hk=3, N=7001, M=50, d=128, dtype=torch.bfloat16, offs=[0, 1111, 3500, 7001],
                                           ranges=[[(0, 50), (3, 33), (40, 41)], [(0, 1), (0, 0), (31, 50)]]),
}


@pytest.mark.parametrize("name", SMALL_TILES)
def test_larger_calls_in_small_tiles(name):
    """Thousands of queries, in parts, of several segments."""
    ran = kernels_of(**SMALL_TILES[name])
    assert "cross_dkdv" in ran and "cross_sum" in ran and "cross_dkdv_wide" not in ran, ran
