"""Host-only checks of how the products with a few tokens are cut: the refusals of the hook that tells, and that the sizes of the GPU
tests reach the ways that they are there for, so that a change of the estimate which hides one is seen."""
import ctypes

import pytest

from paper_2609_39223_b200 import api
from test_gpu_matvec_paths import KINDS, grouped_size, plain_size

SHAPE, FORMAT, NULL = 2, 4, 1


def test_refusals():
    f, out = api.lib().qf_selftest_matvec_cut, (ctypes.c_int * 9)()
    for bad in ((0, 8, 256, 0), (1, 0, 256, 0), (1, 8, 0, 0), (1, 8, 250, 0), (1, 8, 256, -1), (1, 8, 256, 1025), (1 << 31, 8, 256, 0), (1, 1 << 31, 256, 0)):
        assert f(api.FMT_NVFP4, *bad, out) == SHAPE, bad
    assert f(api.FMT_NONE, 1, 8, 256, 0, out) == FORMAT and f(api.FMT_NVFP4, 1, 8, 256, 0, None) == NULL
    assert f(api.FMT_NVFP4, 1, 8, 256, 0, out) == 0


@pytest.mark.parametrize("M,N,K,experts", [(1, 1, 256, 0), (1, 128256, 4096, 0), (16, 300, 1 << 20, 0), (200, 5000, 256, 0), (8, 1536, 2048, 128), (3000, 768, 2048, 16)])
@pytest.mark.parametrize("fmt", [api.FMT_NVFP4, api.FMT_MXFP4, api.FMT_Q4_K])
def test_a_cut_covers_the_product(fmt, M, N, K, experts):
    c = api.qf_selftest_matvec_cut(fmt, M, N, K, experts)
    rows = c.warps // c.kw * 16
    assert c.warps in (4, 8, 16) and c.kw * rows == 16 * c.warps and (c.blocks - 1) * rows < N <= c.blocks * rows
    assert 1 <= c.grid_x <= c.blocks and (c.nz - 1) * c.kz < K <= c.nz * c.kz and c.kz % 256 == 0 and 0 < c.kc <= c.kz and c.kc % 256 == 0


@pytest.mark.parametrize("kind,loose", KINDS)
def test_the_gpu_tests_reach_the_ways(kind, loose):
    for tiles in (1, 2):
        for wanted in (("whole", "several", "at once"), ("warps", "several", "at once"), ("cluster", "several", "at once"), ("cluster", "one", "pieces"),
                       ("whole", "one", "pieces")):
            assert plain_size(kind, loose, tiles, wanted), (tiles, wanted)
    for tiles, listed in ((1, "by pair"), (1, "by expert"), (2, "by expert")):
        for wanted in (("whole", "several", "at once"), ("warps", "several", "at once"), ("cluster", "one", "pieces"), ("warps", "one", "pieces")):
            assert grouped_size(kind, loose, tiles, listed, wanted), (tiles, listed, wanted)
    assert grouped_size(kind, loose, 2, "by expert", ("cluster", "several", "at once"))
