"""Host-only checks of how attention over the 4-bit cache is cut: the refusals of the hook that tells, that a cut fits the call, and that the
sizes of the GPU tests reach the ways that they are there for, so that a change of the rules which hides one is seen."""
import ctypes

import pytest

from paper_2609_39223_b200 import api
from test_gpu_kv_ranges import WAYS
from test_gpu_kv_shares import BY_CTA

NULL, SHAPE, FORMAT = 1, 2, 4
FMTS = pytest.mark.parametrize("fmt", [api.FMT_NVFP4, api.FMT_MXFP4], ids=["nvfp4", "mxfp4"])


def test_refusals():
    f, out = api.lib().qf_selftest_kv_attention_cut, (ctypes.c_int * 5)()

    def go(batch=3, q_len=2, q_heads=32, max_pages=10, to=out, **kw):
        cache = api._KvCacheStruct(**dict(dict(fmt=api.FMT_NVFP4, kv_heads=8, head_dim=128, page_size=64, pages=100), **kw))
        return f(ctypes.addressof(cache), batch, q_len, q_heads, max_pages, to)

    assert go() == 0 and f(None, 1, 1, 8, 1, out) == NULL and go(to=None) == NULL and go(fmt=api.FMT_Q4_K) == FORMAT
    for kw in (dict(batch=0), dict(q_len=0), dict(batch=-1), dict(q_heads=0), dict(q_heads=12), dict(max_pages=-1), dict(max_pages=1 << 25),
               dict(batch=(1 << 20) + 1), dict(head_dim=96), dict(page_size=8), dict(batch=1 << 20, q_len=1 << 12)):
        assert go(**kw) == SHAPE, kw


@FMTS
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("q_len,group", [(1, 1), (1, 4), (5, 4), (17, 3)])
def test_a_cut_fits_the_call(fmt, dim, q_len, group):
    for batch in (1, 2, 7, 40, 150, 600, 5000):
        for heads in (1, 8, 37):
            for most in (0, 1, 2, 30, 80, 250, 4000):
                c = api.qf_selftest_kv_attention_cut(fmt, batch, q_len, heads * group, heads, dim, 64, most)
                eights = -(-q_len * group // 8)
                segments = batch * heads * -(-eights // c.row_tiles)
                assert 1 <= c.row_tiles <= min(eights, {64: 4, 128: 3, 256: 2}[dim]) and c.ctas >= 1
                if c.split > 0:
                    assert c.split in (1, 2, 4, 8) and c.ctas == segments * c.split and c.tasks == 0
                elif c.split == 0:
                    assert c.ctas == -(-segments // 4) and c.tasks == 0
                else:
                    assert c.ctas <= 148 * 4 and c.by_segment == (segments <= c.ctas) and c.tasks == (segments if c.by_segment else c.ctas)


@FMTS
def test_the_gpu_tests_reach_the_ways(fmt):
    for dim, q_len, group, batch, heads, most in BY_CTA:
        c = api.qf_selftest_kv_attention_cut(fmt, batch, q_len, heads * group, heads, dim, 16, most // 16)
        assert c.split == -1 and not c.by_segment and c.tasks == c.ctas, (dim, c)
    tiles = {(dim, api.qf_selftest_kv_attention_cut(fmt, b, n, h * g, h, dim, 16, m // 16).row_tiles) for dim, n, g, b, h, m in BY_CTA}
    assert tiles >= {(64, 1), (64, 2), (64, 4), (128, 1), (128, 3), (256, 1), (256, 2)}
    wanted = {"warps": lambda c: c.split == 0, "CTAs": lambda c: c.split == 1, "small clusters": lambda c: c.split in (2, 4), "clusters": lambda c: c.split == 8,
              "shares": lambda c: c.split == -1 and c.by_segment, "shares by CTA": lambda c: c.split == -1 and not c.by_segment}
    for name, (batch, heads, n) in WAYS.items():
        for dim in (64, 128, 256):
            c = api.qf_selftest_kv_attention_cut(fmt, batch, 2, heads * 2, heads, dim, 16, -(-n // 16))
            assert wanted[name](c), (name, dim, c)
