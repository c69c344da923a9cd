"""Host-only checks of the mixture-of-experts routing calls and of the products with a few tokens: sizes, and the refusal
of bad arguments with the documented codes before anything touches CUDA."""
import pytest
import torch

from paper_2609_39223_b200 import api

P = 0x10000            # a fake, 16-byte aligned, never dereferenced device address
BF, F32, I32, I64 = api.DT_BF16, api.DT_F32, api.DT_I32, api.DT_I64
NULL, SHAPE, ALIGN, FORMAT, CUDA, DTYPE = 1, 2, 3, 4, 6, 9
HERE = CUDA if not torch.cuda.is_available() else None          # what a valid call says without a device


@pytest.mark.parametrize("tokens,top_k,experts,rows", [(0, 8, 128, 0), (1, 1, 1, 128), (1, 8, 128, 1024), (7, 8, 128, 56 * 128),
                                                       (16384, 8, 128, 147328), (129, 1, 1, 256), (128, 1, 1, 128)])
def test_rows_bound(tokens, top_k, experts, rows):
    assert api.qf_moe_rows_bound(tokens, top_k, experts) == rows


def test_rows_bound_holds_every_split_of_a_few_pairs():
    """Every way to give P pairs to G experts needs at most the bound, and one way needs all of it."""
    def splits(pairs, groups):
        if groups == 1:
            yield (pairs,)
            return
        for c in range(pairs + 1):
            for rest in splits(pairs - c, groups - 1):
                yield (c, *rest)
    for pairs, groups in ((1, 3), (5, 3), (130, 2), (257, 2)):
        need = max(sum((c + 127) // 128 * 128 for c in s) for s in splits(pairs, groups))
        assert api.qf_moe_rows_bound(pairs, 1, groups) == need


def test_rows_bound_refusals():
    for bad in ((-1, 8, 4), (4, 0, 4), (4, 2, 0), (4, 2, api.MOE_MAX_EXPERTS + 1), (1 << 31, 1, 4), (1 << 29, 8, 4)):
        with pytest.raises(api.QfError):
            api.qf_moe_rows_bound(*bad)


def _call(f, names, base):
    def go(**kw):
        args = dict(base, **kw)
        return f(*[args[n] for n in names], None)
    return go


def test_sort_refusals():
    f = _call(api.lib().qf_moe_sort, "ids dt tokens k G rows row_of offs counts".split(),
              dict(ids=P, dt=I32, tokens=10, k=2, G=4, rows=512, row_of=P, offs=P, counts=P))
    for kw in (dict(tokens=-1), dict(k=0), dict(G=0), dict(G=1025), dict(rows=100), dict(rows=-128), dict(rows=1 << 31), dict(tokens=1 << 31)):
        assert f(**kw) == SHAPE, kw
    for kw in (dict(dt=BF), dict(dt=F32), dict(dt=9)):
        assert f(**kw) == DTYPE, kw
    for kw in (dict(ids=None), dict(row_of=None), dict(offs=None), dict(counts=None)):
        assert f(**kw) == NULL, kw
    for kw in (dict(ids=P + 4), dict(row_of=P + 4), dict(offs=P + 8), dict(counts=P + 4)):
        assert f(**kw) == ALIGN, kw
    if HERE:
        assert f() == HERE and f(tokens=0, ids=None, row_of=None) == HERE


def test_dispatch_refusals():
    f = _call(api.lib().qf_moe_dispatch, "x tokens k H row_of offs counts G rows xs".split(),
              dict(x=P, tokens=10, k=2, H=64, row_of=P, offs=P, counts=P, G=4, rows=512, xs=P))
    for kw in (dict(tokens=-1), dict(k=0), dict(H=-8), dict(H=12), dict(H=1 << 29), dict(tokens=1 << 24, k=1, H=1 << 20), dict(G=0), dict(G=2000), dict(rows=130), dict(rows=-128)):
        assert f(**kw) == SHAPE, kw
    for name in ("x", "row_of", "offs", "counts", "xs"):
        assert f(**{name: None}) == NULL, name
        assert f(**{name: P + 2}) == ALIGN, name
    if HERE:
        assert f() == HERE


def test_dispatch_gradient_refusals():
    f = _call(api.lib().qf_moe_dispatch_bwd, "dxs dt tokens k H row_of rows dx odt".split(),
              dict(dxs=P, dt=BF, tokens=10, k=2, H=64, row_of=P, rows=512, dx=P, odt=BF))
    for kw in (dict(tokens=-1), dict(k=0), dict(H=12), dict(rows=130)):
        assert f(**kw) == SHAPE, kw
    for kw in (dict(dt=I32), dict(odt=I64), dict(dt=7)):
        assert f(**kw) == DTYPE, kw
    for name in ("dxs", "row_of", "dx"):
        assert f(**{name: None}) == NULL, name
        assert f(**{name: P + 8}) == ALIGN, name
    if HERE:
        assert f() == HERE


def test_combine_refusals():
    f = _call(api.lib().qf_moe_combine, "ys dt w tokens k H row_of rows out odt".split(),
              dict(ys=P, dt=BF, w=P, tokens=10, k=2, H=64, row_of=P, rows=512, out=P, odt=BF))
    for kw in (dict(tokens=-1), dict(k=0), dict(H=12), dict(rows=130), dict(row_of=None, rows=19)):
        assert f(**kw) == SHAPE, kw
    for kw in (dict(dt=I32), dict(odt=I64)):
        assert f(**kw) == DTYPE, kw
    for name in ("ys", "w", "out"):
        assert f(**{name: None}) == NULL, name
    for name in ("ys", "w", "row_of", "out"):
        assert f(**{name: P + 4}) == ALIGN, name
    if HERE:
        assert f() == HERE and f(row_of=None, rows=20) == HERE


def test_combine_gradient_refusals():
    f = _call(api.lib().qf_moe_combine_bwd, "dout dt ys ydt w tokens k H row_of offs counts G rows dys dw".split(),
              dict(dout=P, dt=BF, ys=P, ydt=BF, w=P, tokens=10, k=2, H=64, row_of=P, offs=P, counts=P, G=4, rows=512, dys=P, dw=P))
    for kw in (dict(tokens=-1), dict(k=0), dict(H=12), dict(G=0), dict(G=1025), dict(rows=130)):
        assert f(**kw) == SHAPE, kw
    for kw in (dict(dt=I32), dict(ydt=I64)):
        assert f(**kw) == DTYPE, kw
    for name in ("dout", "ys", "w", "row_of", "offs", "counts", "dys"):
        assert f(**{name: None}) == NULL, name
    for name in ("dout", "ys", "w", "row_of", "offs", "counts", "dys", "dw"):
        assert f(**{name: P + 4}) == ALIGN, name
    if HERE:
        assert f() == HERE and f(dw=None, ys=None) == HERE


def test_matvec_refusals():
    f = _call(api.lib().qf_fq_matvec, "fmt X M codes scales ts N K Y dt".split(),
              dict(fmt=api.FMT_NVFP4, X=P, M=3, codes=P, scales=P, ts=P, N=10, K=512, Y=P, dt=BF))
    for kw in (dict(M=-1), dict(N=-1), dict(K=-16), dict(K=500), dict(fmt=api.FMT_MXFP4, K=528), dict(fmt=api.FMT_Q4_K, K=384), dict(N=1 << 31), dict(K=(1 << 26) + 256),
               dict(M=1 << 31)):
        assert f(**kw) == SHAPE, kw
    for fmt in (api.FMT_NONE, 4, -1):
        assert f(fmt=fmt) == FORMAT
    assert f(dt=I32) == DTYPE
    for name in ("X", "codes", "scales", "ts", "Y"):
        assert f(**{name: None}) == NULL, name
        assert f(**{name: P + 2}) == ALIGN, name
    if HERE:
        assert f() == HERE and f(fmt=api.FMT_MXFP4, ts=None) == HERE and f(M=0) == HERE



def test_matvec_row_numbers_fit_32_bits():
    """Rows are walked 1024 at a time with 32-bit numbers: the last step must not pass 2^31 - 1."""
    f = _call(api.lib().qf_fq_matvec, "fmt X M codes scales ts N K Y dt".split(),
              dict(fmt=api.FMT_NVFP4, X=P, M=1, codes=P, scales=P, ts=P, N=1, K=16, Y=P, dt=BF))
    for name in ("M", "N"):
        for most in ((1 << 31) - 1024, (1 << 31) - 257, (1 << 31) - 1):
            assert f(**{name: most}) == SHAPE, (name, most)
        if HERE:
            assert f(**{name: (1 << 31) - 1025}) == HERE, name


def test_grouped_matvec_refusals():
    f = _call(api.lib().qf_fq_grouped_matvec, "fmt X xr ids idt pairs G codes scales ts N K Y dt".split(),
              dict(fmt=api.FMT_MXFP4, X=P, xr=3, ids=P, idt=I32, pairs=24, G=16, codes=P, scales=P, ts=None, N=10, K=512, Y=P, dt=BF))
    for kw in (dict(pairs=-1), dict(xr=0), dict(xr=5), dict(xr=48), dict(G=0), dict(G=1025), dict(K=40), dict(N=-1)):
        assert f(**kw) == SHAPE, kw
    assert f(idt=BF) == DTYPE and f(dt=I64) == DTYPE and f(fmt=7) == FORMAT
    for name in ("X", "ids", "codes", "scales", "Y"):
        assert f(**{name: None}) == NULL, name
        assert f(**{name: P + 2}) == ALIGN, name
    assert f(fmt=api.FMT_NVFP4) == NULL                       # one tensor scale per expert is needed
    if HERE:
        assert f() == HERE


def test_binding_refuses_host_tensors_and_wrong_shapes():
    ids = torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(TypeError):
        api.qf_moe_sort(ids, 4)
    with pytest.raises(TypeError):
        api.qf_fq_matvec(api.FMT_MXFP4, torch.zeros((1, 64), dtype=torch.bfloat16), torch.zeros((4, 32), dtype=torch.uint8),
                         torch.zeros((4, 2), dtype=torch.uint8))
    with pytest.raises(api.QfError):
        api.qf_fq_matvec(api.FMT_NONE, torch.zeros((1, 64), dtype=torch.bfloat16), torch.zeros((4, 32), dtype=torch.uint8),
                         torch.zeros((4, 2), dtype=torch.uint8))
