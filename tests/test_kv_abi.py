"""Host-only checks of the 4-bit key/value cache calls: refusal of bad arguments with the documented codes before anything touches
CUDA, and of tensors on other devices."""
import ctypes

import pytest
import torch

from paper_2609_39223_b200 import api
from test_binding_devices import Called, Stand

P = 0x10000            # a fake, 16-byte aligned, never dereferenced device address
NULL, SHAPE, ALIGN, FORMAT, WORKSPACE, CUDA, DTYPE = 1, 2, 3, 4, 5, 6, 9
HERE = CUDA if not torch.cuda.is_available() else None          # what a valid call says without a device
CACHE = dict(fmt=api.FMT_NVFP4, kv_heads=8, head_dim=128, page_size=64, pages=100, k_codes=P, k_scales=P, v_codes=P, v_scales=P, k_tscale=P, v_tscale=P)


def _call(f, names, base):
    def go(cache=None, **kw):
        c = api._KvCacheStruct(**dict(CACHE, **(cache or {})))
        args = dict(base, **kw)
        return f(None if kw.get("none") else ctypes.addressof(c), *[args[n] for n in names], None)
    return go


def calls():
    L = api.lib()
    append = _call(L.qf_kv_append, "k ks v vs tokens slots dt flags".split(), dict(k=P, ks=1024, v=P, vs=1024, tokens=5, slots=P, dt=api.DT_I32, flags=0))
    read = _call(L.qf_kv_read, "slots dt rows k v".split(), dict(slots=P, dt=api.DT_I64, rows=5, k=P, v=P))
    ws = api.qf_workspace_bytes(api.OP_KV_ATTENTION, 6, 32, 128, 8)
    attend = _call(L.qf_kv_attention, "q qs batch q_len q_heads table max_pages lens scale out lse ws wsb".split(),
                   dict(q=P, qs=4096, batch=3, q_len=2, q_heads=32, table=P, max_pages=10, lens=P, scale=1.0, out=P, lse=P, ws=P, wsb=ws))
    return append, read, attend


@pytest.mark.parametrize("which", range(3), ids=["append", "read", "attention"])
def test_caches_that_are_refused(which):
    f = calls()[which]
    assert f(none=True) == NULL
    for fmt in (api.FMT_NONE, api.FMT_Q4_K, 9):
        assert f(dict(fmt=fmt)) == FORMAT
    for kw in (dict(kv_heads=0), dict(kv_heads=65536), dict(head_dim=96), dict(head_dim=32), dict(head_dim=512), dict(page_size=0), dict(page_size=24),
               dict(page_size=(1 << 20) + 16), dict(pages=-1), dict(pages=1 << 31), dict(pages=(1 << 31) - 1, page_size=64)):
        assert f(kw) == SHAPE, kw
    for n in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert f({n: P + 8}) == ALIGN and f({n: None}) == NULL, n
    for n in ("k_tscale", "v_tscale"):
        assert f({n: P + 2}) == ALIGN and f({n: None}) == NULL, n
        if HERE:
            assert f({"fmt": api.FMT_MXFP4, n: None}) == HERE
        if which > 0:                                              # a cache without pages is read as nothing, but its scales are looked at
            assert f({"pages": 0, n: None}) == NULL
    if HERE:
        assert f() == HERE and f(dict(pages=0, k_codes=None, v_scales=None)) == HERE


def test_append_refusals():
    f = calls()[0]
    for kw in (dict(tokens=-1), dict(tokens=1 << 31), dict(ks=1016), dict(vs=1020), dict(ks=1028), dict(vs=1 << 31)):
        assert f(**kw) == SHAPE, kw
    assert f(dict(kv_heads=65535, head_dim=256), ks=65535 * 256, vs=65535 * 256, tokens=1 << 20) == SHAPE       # more CTAs than there are numbers
    for kw in (dict(dt=api.DT_BF16), dict(dt=7)):
        assert f(**kw) == DTYPE, kw
    for n in ("k", "v", "slots"):
        assert f(**{n: None}) == NULL, n
    for kw in (dict(k=P + 8), dict(v=P + 2), dict(slots=P + 2), dict(slots=P + 4, dt=api.DT_I64)):
        assert f(**kw) == ALIGN, kw
    if HERE:
        assert f(slots=P + 4) == HERE and f(tokens=0, k=None, v=None, slots=None) == HERE and f(dict(pages=0, k_codes=None)) == HERE


def test_read_refusals():
    f = calls()[1]
    assert f(rows=-1) == SHAPE and f(rows=1 << 31) == SHAPE and f(dt=api.DT_F32) == DTYPE
    assert f(slots=None) == NULL and f(k=None, v=None) == NULL
    assert f(k=P + 8) == ALIGN and f(v=P + 4) == ALIGN and f(slots=P + 4) == ALIGN
    if HERE:
        assert f(k=None) == HERE and f(v=None) == HERE and f(rows=0, slots=None, k=None, v=None) == HERE


def test_attention_refusals():
    f = calls()[2]
    for kw in (dict(batch=-1), dict(q_len=-1), dict(q_heads=0), dict(q_heads=12), dict(max_pages=-1), dict(max_pages=1 << 25), dict(qs=4088), dict(qs=4100),
               dict(batch=(1 << 20) + 1), dict(batch=1 << 20, q_len=1 << 12), dict(q_heads=1 << 21, qs=1 << 28)):
        assert f(**kw) == SHAPE, kw
    for kw in (dict(ws=None), dict(wsb=255), dict(wsb=api.qf_workspace_bytes(api.OP_KV_ATTENTION, 6, 32, 128, 8) - 1)):
        assert f(**kw) == WORKSPACE, kw
    for n in ("q", "out", "lens", "table"):
        assert f(**{n: None}) == NULL, n
    for kw in (dict(q=P + 8), dict(out=P + 8), dict(ws=P + 8), dict(table=P + 2), dict(lens=P + 1), dict(lse=P + 2)):
        assert f(**kw) == ALIGN, kw
    if HERE:
        assert f(lse=None) == HERE and f(batch=0, q=None, out=None) == HERE and f(q_len=0, q=None) == HERE and f(max_pages=0, table=None) == HERE


def test_workspace_does_not_grow_with_the_batch_without_end():
    f = lambda rows, heads: api.qf_workspace_bytes(api.OP_KV_ATTENTION, rows, heads, 128, 8)
    assert f(1, 32) >= 256 and f(1, 32) % 256 == 0
    assert f(1 << 20, 32) == f(1 << 16, 32) < 1 << 28


def test_every_tensor_has_to_be_on_the_current_device(monkeypatch):
    class Lib:
        def __getattr__(self, name):
            def called(*args):
                raise Called(name)
            return called
    monkeypatch.setattr(api, "lib", lambda: Lib())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0)
    monkeypatch.setattr(Stand, "dim", lambda self: len(self.shape), raising=False)
    BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
    cache = dict(k_codes=(U8, 4, 2, 16, 32), k_scales=(U8, 4, 2, 16, 4), v_codes=(U8, 4, 2, 16, 32), v_scales=(U8, 4, 2, 16, 4), k_tscale=(F32, 1),
                 v_tscale=(F32, 1))
    made = lambda t: api.KvCache(api.FMT_NVFP4, *[t[n] for n in cache])
    rows = dict(k=(BF, 5, 2, 64), v=(BF, 5, 2, 64), slots=(I32, 5))
    attend = dict(q=(BF, 3, 1, 4, 64), table=(I32, 3, 2), lens=(I32, 3), out=(BF, 3, 1, 4, 64), lse=(F32, 3, 1, 4), ws=(U8, 1 << 20))
    for kinds, go in (({**cache, **rows}, lambda t: api.qf_kv_append(made(t), t["k"], t["v"], t["slots"])),
                      ({**cache, **rows}, lambda t: api.qf_kv_read(made(t), t["slots"], k=t["k"], v=t["v"])),
                      ({**cache, **attend}, lambda t: api.qf_kv_attention(made(t), t["q"], t["table"], t["lens"], out=t["out"], lse=t["lse"], ws=t["ws"]))):
        make = lambda other=None, device=1: {n: Stand(*k, device=device if n == other else 0) for n, k in kinds.items()}
        with pytest.raises(Called):
            go(make())
        for name in kinds:
            with pytest.raises(ValueError, match="cuda:"):
                go(make(name))
            with pytest.raises(TypeError):
                go(make(name, device=-1))
        with pytest.raises(ValueError, match="cuda:"):             # all on one device, which is not the current one
            go({n: Stand(*k, device=1) for n, k in kinds.items()})
