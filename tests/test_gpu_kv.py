"""The 4-bit key/value cache on the GPU: writes bit for bit the oracle's quantizer, reads the oracle's dequantizer, attention within
derived bounds of the 64-bit form."""
import math

import numpy as np
import pytest
import torch

import oracle
from kv_reference import check_attention
from paper_2609_39223_b200 import api
from util import bits_to_torch, torch_to_bits

pytestmark = pytest.mark.gpu
FMTS = {"nvfp4": api.FMT_NVFP4, "mxfp4": api.FMT_MXFP4}
fmts = pytest.mark.parametrize("fmt", FMTS.values(), ids=FMTS.keys())
BF = torch.bfloat16


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def tscales(fmt, k=30.0 / 2688, v=6.0 / 2688):
    return (torch.tensor([k], device="cuda"), torch.tensor([v], device="cuda")) if fmt == api.FMT_NVFP4 else (None, None)


def filled(fmt, pages, page_size, heads, dim, byte=0xA5, **kw):
    c = api.KvCache.empty(fmt, pages, page_size, heads, dim, *tscales(fmt, **kw))
    for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales):
        t.fill_(byte)
    return c


def random_cache(fmt, pages, page_size, heads, dim, seed=0, scale_bytes=None):
    """Random codes with the block scales of about N(0, 1) data."""
    g = gen(seed)
    c = api.KvCache.empty(fmt, pages, page_size, heads, dim, *tscales(fmt, 1 / 256, 1 / 512))
    for t in (c.k_codes, c.v_codes):
        t.copy_(torch.randint(0, 256, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    low, high = scale_bytes or ((0x60, 0x7F) if fmt == api.FMT_NVFP4 else (123, 128))
    for t in (c.k_scales, c.v_scales):
        t.copy_(torch.randint(low, high, t.shape, generator=g, device="cuda", dtype=torch.uint8))
    return c


def paged(lens, page_size, max_pages=None, spare=2, seed=0, unused=-7):
    """A page table of shuffled pages for the given lengths; entries that no key needs hold `unused`."""
    need = [-(-n // page_size) for n in lens]
    most = max([1, *need]) if max_pages is None else max_pages
    total = sum(need) + spare
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((len(lens), most), unused, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), total


def quantized(fmt, x, ts, noclip=False):
    """Oracle codes, scales and values of BF16 rows [..., dim]."""
    rows = x.reshape(-1, x.shape[-1])
    r = oracle.qdq(fmt, torch_to_bits(rows), None if ts is None else float(ts), noclip)
    return (torch.from_numpy(r["codes"]).view(*x.shape[:-1], -1), torch.from_numpy(r["scales"]).view(*x.shape[:-1], -1), bits_to_torch(r["out"]).view(x.shape))


# ---- writes and reads --------------------------------------------------------------------------------------------------------

@fmts
@pytest.mark.parametrize("tokens,heads,dim,page,dtype", [(1, 1, 64, 16, torch.int32), (33, 8, 128, 64, torch.int64), (257, 3, 256, 48, torch.int32),
                                                         (1000, 5, 64, 16, torch.int64)])
def test_rows_are_the_oracles_and_nothing_else_changes(fmt, tokens, heads, dim, page, dtype):
    g = gen(tokens)
    pages = tokens // page + 3
    c = filled(fmt, pages, page, heads, dim)
    k = (torch.randn((tokens, heads, dim), generator=g, device="cuda") * torch.exp2(torch.randint(-12, 4, (tokens, heads, 1), generator=g, device="cuda"))).to(BF)
    v = torch.randn((tokens, heads, dim), generator=g, device="cuda").to(BF)
    v[0, :, :32] = 0
    v[-1, 0, :40] = -0.0
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens].to(dtype)
    drop = torch.rand(tokens, generator=g, device="cuda") < 0.2
    drop[0] = False
    bad = torch.tensor([-1, pages * page, -pages * page, 2 ** 31 - 1], device="cuda")[torch.arange(tokens, device="cuda") % 4].to(dtype)
    slots = torch.where(drop, bad, slots)
    api.qf_kv_append(c, k, v, slots)
    kept = ~drop.cpu()
    at = slots.cpu().long()[kept]
    for x, codes, scales, ts in ((k, c.k_codes, c.k_scales, c.k_tscale), (v, c.v_codes, c.v_scales, c.v_tscale)):
        rc, rs, _ = quantized(fmt, x.cpu()[kept], ts)
        for got, want in ((codes, rc), (scales, rs)):
            expect = torch.full_like(got, 0xA5).cpu()
            expect[at // page, :, at % page] = want
            assert torch.equal(got.cpu(), expect)
    rk, rv = api.qf_kv_read(c, slots)
    for got, x, ts in ((rk, k, c.k_tscale), (rv, v, c.v_tscale)):
        want = torch.zeros(x.shape, dtype=BF)
        want[kept] = quantized(fmt, x.cpu()[kept], ts)[2]
        assert np.array_equal(torch_to_bits(got), torch_to_bits(want))
    only_k, none = api.qf_kv_read(c, slots, want_v=False)
    none2, only_v = api.qf_kv_read(c, slots, want_k=False)
    assert none is None and none2 is None and torch.equal(only_k, rk) and torch.equal(only_v, rv)


@fmts
@pytest.mark.parametrize("tokens,heads,dim,page,dtype", [(61, 14, 256, 16, torch.int64), (700, 33, 128, 32, torch.int32), (6001, 7, 128, 64, torch.int64),
                                                         (20011, 1, 64, 16, torch.int32), (5, 70, 256, 16, torch.int64)])
def test_rows_that_need_several_CTAs_and_CTAs_of_several_rows(fmt, tokens, heads, dim, page, dtype):
    test_rows_are_the_oracles_and_nothing_else_changes(fmt, tokens, heads, dim, page, dtype)


@fmts
@pytest.mark.parametrize("noclip", [False, True])
def test_every_magnitude(fmt, noclip):
    """Raw BF16 patterns over the whole finite range, with the tensor scale far from them as well."""
    r = np.random.default_rng(5)
    bits = r.integers(0, 1 << 16, (64, 2, 128), dtype=np.uint16)
    bits = np.where((bits & 0x7F80) == 0x7F80, bits & 0xBFFF, bits).astype(np.uint16)
    if noclip:          # blocks above 3.5 * 2^126 overflow under that rule
        bits = np.where((bits & 0x7F80) > 0x7E00, bits & 0xBFFF, bits).astype(np.uint16)
    x = bits_to_torch(bits)
    for k, v in ((1.0, 2.0 ** -30), (2.0 ** 40, 2.0 ** -60)):
        c = filled(fmt, 5, 16, 2, 128, k=k, v=v)
        slots = torch.arange(3, 67, device="cuda")
        api.qf_kv_append(c, x.cuda(), x.cuda(), slots, flags=api.MXFP4_NO_CLIP if noclip else 0)
        for got, codes, scales, ts in zip(api.qf_kv_read(c, slots), (c.k_codes, c.v_codes), (c.k_scales, c.v_scales), (c.k_tscale, c.v_tscale)):
            rc, rs, out = quantized(fmt, x, ts, noclip and fmt == api.FMT_MXFP4)
            at = slots.cpu()
            assert torch.equal(codes.cpu()[at // 16, :, at % 16], rc) and torch.equal(scales.cpu()[at // 16, :, at % 16], rs)
            assert np.array_equal(torch_to_bits(got), torch_to_bits(out))


@fmts
def test_slices_of_a_fused_projection_and_repeated_reads(fmt):
    g = gen(9)
    T, H, D = 37, 2, 64
    qkv = torch.randn((T, (6 + 2 * H) * D), generator=g, device="cuda").to(BF)
    k, v = qkv[:, 6 * D:(6 + H) * D].view(T, H, D), qkv[:, (6 + H) * D:].view(T, H, D)
    a, b = filled(fmt, 4, 16, H, D), filled(fmt, 4, 16, H, D)
    slots = torch.arange(T, device="cuda")
    api.qf_kv_append(a, k, v, slots)
    api.qf_kv_append(b, k.contiguous(), v.contiguous(), slots)
    for n in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert torch.equal(getattr(a, n), getattr(b, n))
    again = slots[torch.randint(0, T, (500,), generator=g, device="cuda")]
    rk, rv = api.qf_kv_read(a, again)
    full = api.qf_kv_read(a, slots)
    assert torch.equal(rk, full[0][again]) and torch.equal(rv, full[1][again])


@fmts
def test_nothing_to_write_or_read(fmt):
    c = filled(fmt, 2, 16, 2, 64)
    none = torch.empty((0,), dtype=torch.int64, device="cuda")
    api.qf_kv_append(c, torch.empty((0, 2, 64), dtype=BF, device="cuda"), torch.empty((0, 2, 64), dtype=BF, device="cuda"), none)
    k, v = api.qf_kv_read(c, none)
    assert k.shape == v.shape == (0, 2, 64)
    z = api.KvCache.empty(fmt, 0, 16, 2, 64, *tscales(fmt))
    x = torch.ones((3, 2, 64), dtype=BF, device="cuda")
    api.qf_kv_append(z, x, x, torch.arange(3, device="cuda"))
    k, v = api.qf_kv_read(z, torch.arange(3, device="cuda"))
    assert (k == 0).all() and (v == 0).all()
    table = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    out, lse = api.qf_kv_attention(z, torch.ones((2, 1, 4, 64), dtype=BF, device="cuda"), table, torch.tensor([5, 0], dtype=torch.int32, device="cuda"), want_lse=True)
    assert (out == 0).all() and torch.isinf(lse).all()
    assert api.qf_kv_attention(c, torch.empty((0, 1, 4, 64), dtype=BF, device="cuda"), table[:0], table[:0, 0]).shape == (0, 1, 4, 64)


# ---- attention ---------------------------------------------------------------------------------------------------------------

def attend(fmt, lens, page, heads, group, dim, q_len=1, seed=0, scale=None, cache=None, **kw):
    table, n, pages = paged(lens, page, seed=seed, **kw)
    c = random_cache(fmt, pages, page, heads, dim, seed) if cache is None else cache(pages)
    q = torch.randn((len(lens), q_len, heads * group, dim), generator=gen(seed + 1), device="cuda").to(BF)
    out, lse = api.qf_kv_attention(c, q, table, n, softmax_scale=scale, want_lse=True)
    check_attention(c, q, table, lens, dim ** -0.5 if scale is None else scale, out, lse)
    assert torch.equal(out, api.qf_kv_attention(c, q, table, n, softmax_scale=scale))        # the same bits every time, and without lse
    return c, q, table, n, out, lse


@fmts
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group", [(1, 1), (8, 4), (3, 7), (2, 8), (1, 16), (5, 2), (2, 24)])
def test_head_layouts(fmt, dim, heads, group):
    attend(fmt, [1, 47, 200, 16], 16, heads, group, dim)


@fmts
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 48, 64, 1024])
def test_lengths_around_every_border(fmt, dim, page):
    attend(fmt, [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 0, 255, 257, 511, 513], page, 2, 4, dim)


@fmts
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("q_len,group", [(2, 4), (3, 1), (5, 4), (7, 5), (16, 1), (17, 2), (40, 3)])
def test_several_new_tokens_see_up_to_themselves(fmt, dim, q_len, group):
    """Sequences shorter than q_len leave rows without keys."""
    attend(fmt, [q_len, 0, 1, q_len - 1, q_len + 1, 100, 333], 32, 2, group, dim, q_len=q_len)


@fmts
@pytest.mark.parametrize("batch,heads,group,dim,length", [(1, 8, 4, 128, 20000), (1, 1, 1, 64, 70001), (1, 1, 12, 256, 9000), (2, 1, 8, 128, 33333), (3, 4, 3, 64, 12345)])
def test_long_sequences(fmt, batch, heads, group, dim, length):
    attend(fmt, [length - 77 * b for b in range(batch)], 64, heads, group, dim)


@fmts
def test_a_large_ragged_batch(fmt):
    r = np.random.default_rng(3)
    lens = [int(x) for x in np.exp(r.uniform(0, math.log(2000), 200))]
    lens[::17] = [0] * len(lens[::17])
    attend(fmt, lens, 16, 2, 4, 128)


@fmts
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("q_len,group", [(1, 4), (5, 4), (3, 8)])
def test_short_sequences_in_a_wide_page_table(fmt, dim, q_len, group):
    """A table for 20000 keys: how the work is cut goes by what the table can hold, the lengths are short, empty and in between."""
    attend(fmt, [1, 0, 31, 32, 33, 100, 383, 384, 385, 416, 0, 700, 1500, 7], 16, 3, group, dim, q_len=q_len, max_pages=1250)
    attend(fmt, [300], 32, 1, group, dim, q_len=q_len, max_pages=625)
    attend(fmt, [20, 0, 0], 32, 1, group, dim, q_len=q_len, max_pages=625)


@fmts
@pytest.mark.parametrize("dim,q_len,group", [(64, 1, 12), (64, 5, 4), (64, 4, 8), (64, 3, 11), (128, 3, 4), (128, 3, 8), (128, 5, 8), (256, 1, 12), (256, 2, 8), (256, 3, 8)])
@pytest.mark.parametrize("batch,heads,most", [(20, 3, 1536), (50, 4, 700), (8, 3, 10000)])
def test_every_tile_of_query_rows_with_every_cut(fmt, dim, q_len, group, batch, heads, most):
    """Tables large enough for the larger tiles, in clusters, with a CTA a sequence, and in shares; few of the sequences fill them."""
    r = np.random.default_rng(dim + group)
    lens = [int(x) for x in r.integers(0, 150, batch)]
    lens[1], lens[2], lens[-1] = min(most, 1100), 0, min(most, 700)
    attend(fmt, lens, 16, heads, group, dim, q_len=q_len, max_pages=-(-most // 16))


@fmts
@pytest.mark.parametrize("dim,q_len,group", [(64, 1, 1), (64, 3, 4), (64, 3, 8), (64, 4, 8), (64, 9, 4), (128, 1, 8), (128, 3, 4), (128, 3, 8), (128, 5, 8), (256, 1, 4), (256, 3, 4), (256, 3, 8)])
@pytest.mark.parametrize("most", [1, 130])
def test_a_warp_a_sequence(fmt, dim, q_len, group, most):
    """More (sequence, head) pairs than CTAs, not a multiple of a CTA's warps, of empty to short sequences."""
    r = np.random.default_rng(dim + group)
    lens = [int(x) for x in r.integers(0, most + 1, 701)]
    lens[0], lens[-1] = most, 0
    attend(fmt, lens, 16, 3, group, dim, q_len=q_len)


@fmts
def test_the_same_rows_whatever_the_table_can_hold(fmt):
    """Two ways to cut the work give the same rows up to FP32 sums and weights."""
    lens, page = [700, 3, 0, 260, 129], 16
    table, n, pages = paged(lens, page)
    wide, _, _ = paged(lens, page, max_pages=2000)
    c = random_cache(fmt, pages, page, 2, 128, 3)
    q = torch.randn((5, 1, 8, 128), generator=gen(4), device="cuda").to(BF)
    (a, la), (b, lb) = (api.qf_kv_attention(c, q, x, n, want_lse=True) for x in (table, wide))
    check_attention(c, q, table, lens, 128 ** -0.5, a, la)
    check_attention(c, q, wide, lens, 128 ** -0.5, b, lb)


@fmts
@pytest.mark.parametrize("batch,most,page", [(130, 400, 16), (700, 70, 32), (3000, 20, 16), (40, 385, 64)])
def test_many_short_sequences(fmt, batch, most, page):
    """More sequences than threads look at, than CTAs, and of the length from which on sequences are cut."""
    r = np.random.default_rng(batch)
    lens = [int(x) for x in r.integers(0, most + 1, batch)]
    lens[0] = most
    attend(fmt, lens, page, 1, 3, 64)


@fmts
def test_a_batch_without_keys(fmt):
    c = random_cache(fmt, 2, 16, 2, 128)
    q = torch.randn((300, 3, 8, 128), generator=gen(0), device="cuda").to(BF)
    out, lse = torch.full_like(q, 7.0), torch.zeros((300, 3, 8), device="cuda")
    api.qf_kv_attention(c, q, torch.full((300, 4), -1, dtype=torch.int32, device="cuda"), torch.zeros(300, dtype=torch.int32, device="cuda"), out=out, lse=lse)
    assert (out == 0).all() and torch.isinf(lse).all() and (lse < 0).all()


@fmts
@pytest.mark.parametrize("order", ["rising", "falling", "steps"])
def test_scores_that_move_the_maximum(fmt, order):
    """Scores that rise by dozens from page to page, fall, or jump both ways."""
    page, heads, dim, n = 16, 2, 128, 2000
    c = random_cache(fmt, n // page, page, heads, dim, 9)
    c.k_codes.fill_(0x22)
    at = torch.arange(n // page, device="cuda")
    level = {"rising": at % 40, "falling": 40 - at % 40, "steps": (at * 7) % 40}[order]
    if fmt == api.FMT_NVFP4:
        c.k_scales.copy_((0x20 + level).to(torch.uint8)[:, None, None, None].expand_as(c.k_scales))
        c.k_tscale.fill_(1.0)
    else:
        c.k_scales.copy_((110 + level // 2).to(torch.uint8)[:, None, None, None].expand_as(c.k_scales))
    q = (1.0 + torch.rand((1, 2, 8, dim), generator=gen(2), device="cuda")).to(BF)
    table = at.to(torch.int32)[None]
    for scale in (dim ** -0.5, 0.01, -0.02):
        out, lse = api.qf_kv_attention(c, q, table, torch.tensor([n], dtype=torch.int32, device="cuda"), softmax_scale=scale, want_lse=True)
        check_attention(c, q, table, [n], scale, out, lse)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("scale", [0.001, 0.05])
def test_value_ranges_that_change_along_a_sequence(dim, scale):
    """MXFP4 pages whose value scales lie close together, far apart, far below or above the page before, or are those of zeros."""
    page, heads, n = 16, 2, 3000
    g = gen(dim)
    c = random_cache(api.FMT_MXFP4, n // page + 1, page, heads, dim, 9)
    kinds = ((120, 128), (100, 140), (60, 70), (180, 190), (127, 128), (108, 136))
    for i in range(c.pages):
        low, high = kinds[(i * i + i // 7) % len(kinds)]
        c.v_scales[i].copy_(torch.randint(low, high, c.v_scales[i].shape, generator=g, device="cuda", dtype=torch.uint8))
        if i % 9 == 4:
            c.v_scales[i, :, ::3] = 0
            c.v_codes[i, :, ::3] = 0
    table = torch.randperm(c.pages, generator=g, device="cuda").to(torch.int32)[None]
    for group, q_len, m in ((4, 1, n), (5, 4, n - 7), (1, 1, 100)):
        q = torch.randn((1, q_len, heads * group, dim), generator=g, device="cuda").to(BF)
        out, lse = api.qf_kv_attention(c, q, table, torch.tensor([m], dtype=torch.int32, device="cuda"), softmax_scale=scale, want_lse=True)
        check_attention(c, q, table, [m], scale, out, lse)
    # falling and rising by up to 2^60 a step, over and over
    for codes in ((190, 132, 74, 16), (16, 74, 132, 190), (250, 190, 130, 70, 10)):
        for i in range(c.pages):
            c.v_scales[i].fill_(codes[(i // 2) % len(codes)])
        q = torch.randn((1, 1, heads * 4, dim), generator=g, device="cuda").to(BF)
        for m in (40, 190, n):
            out, lse = api.qf_kv_attention(c, q, table, torch.tensor([m], dtype=torch.int32, device="cuda"), softmax_scale=scale, want_lse=True)
            check_attention(c, q, table, [m], scale, out, lse)
    flat = api.KvCache(api.FMT_MXFP4, c.k_codes, c.k_scales, c.v_codes, torch.full_like(c.v_scales, 20), None, None)      # all far below 1
    out, lse = api.qf_kv_attention(flat, q, table, torch.tensor([m], dtype=torch.int32, device="cuda"), softmax_scale=scale, want_lse=True)
    check_attention(flat, q, table, [m], scale, out, lse)


@fmts
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_whatever_stands_behind_the_last_key(fmt, dim):
    """Places that no key owns hold NaN scales and extreme codes; unused table entries hold nonsense."""
    lens, page, heads = [1, 17, 33, 95, 160], 32, 2
    table, n, pages = paged(lens, page)
    clean = random_cache(fmt, pages, page, heads, dim, 4)
    dirty = api.KvCache(fmt, clean.k_codes.clone(), clean.k_scales.clone(), clean.v_codes.clone(), clean.v_scales.clone(), clean.k_tscale, clean.v_tscale)
    own = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    for b, m in enumerate(lens):
        j = torch.arange(m, device="cuda")
        own[table[b, j // page].long(), j % page] = True
    for t in (dirty.k_codes, dirty.k_scales, dirty.v_codes, dirty.v_scales):
        t.copy_(torch.where(own[:, None, :, None], t, 0xFF))
    q = torch.randn((len(lens), 1, heads * 4, dim), generator=gen(1), device="cuda").to(BF)
    a, la = api.qf_kv_attention(clean, q, table, n, want_lse=True)
    nonsense = table.clone()
    nonsense[table < 0] = 2 ** 31 - 1
    b, lb = api.qf_kv_attention(dirty, q, nonsense, n, want_lse=True)
    assert torch.equal(a, b) and torch.equal(la, lb)


@fmts
def test_pages_shared_by_sequences(fmt):
    """A common prompt whose pages several sequences list."""
    page, heads, dim = 16, 2, 128
    c = random_cache(fmt, 12, page, heads, dim, 8)
    table = torch.tensor([[3, 1, 7, 0], [3, 1, 7, 5], [3, 1, 2, 0], [3, 3, 3, 3]], dtype=torch.int32, device="cuda")
    lens = [48, 64, 40, 60]
    q = torch.randn((4, 2, 8, dim), generator=gen(2), device="cuda").to(BF)
    out, lse = api.qf_kv_attention(c, q, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), want_lse=True)
    check_attention(c, q, table, lens, dim ** -0.5, out, lse)


@fmts
@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 3.0])
def test_scales_of_the_softmax(fmt, scale):
    attend(fmt, [3, 100, 400], 16, 2, 4, 128, scale=scale)


@fmts
def test_one_key_takes_all(fmt):
    """Scores hundreds apart, the largest first, last or in the middle."""
    page, heads, dim, n = 16, 1, 128, 320
    for place in (0, 1, 159, 160, n - 1):
        c = filled(fmt, n // page, page, heads, dim, byte=0, k=1.0, v=1.0)
        k = torch.randn((n, heads, dim), generator=gen(place), device="cuda").to(BF)
        k[place] = 6.0
        v = torch.randn((n, heads, dim), generator=gen(place + 1), device="cuda").to(BF)
        api.qf_kv_append(c, k, v, torch.arange(n, device="cuda"))
        table = torch.arange(n // page, dtype=torch.int32, device="cuda")[None]
        q = torch.full((1, 1, 4, dim), 8.0, device="cuda", dtype=BF)
        out, lse = api.qf_kv_attention(c, q, table, torch.tensor([n], dtype=torch.int32, device="cuda"), want_lse=True)
        check_attention(c, q, table, [n], dim ** -0.5, out, lse)
        _, rv = api.qf_kv_read(c, torch.tensor([place], device="cuda"))
        assert torch.allclose(out[0, 0].float(), rv[0].float().expand(4, -1), rtol=2.0 ** -7)


@fmts
def test_magnitudes(fmt):
    """Queries, keys and values whose blocks differ by many powers of two."""
    g = gen(11)
    page, heads, dim, n = 16, 2, 128, 100
    if fmt == api.FMT_MXFP4:
        c = random_cache(fmt, 8, page, heads, dim, 5)
        c.k_scales.copy_(torch.randint(100, 128, c.k_scales.shape, generator=g, device="cuda", dtype=torch.uint8))
        c.v_scales.copy_(torch.randint(60, 190, c.v_scales.shape, generator=g, device="cuda", dtype=torch.uint8))
    else:
        c = random_cache(fmt, 8, page, heads, dim, 5, scale_bytes=(0, 0x7F))
        c.v_tscale.fill_(2.0 ** -90)
        c.k_tscale.fill_(2.0 ** -70)
    q = torch.randn((1, 1, 8, dim), generator=g, device="cuda") * torch.exp2(torch.randint(-20, 1, (1, 1, 8, dim), generator=g, device="cuda"))
    q = (q * (2.0 ** 65 if fmt == api.FMT_NVFP4 else 1.0)).to(BF)
    table = torch.arange(8, dtype=torch.int32, device="cuda")[None]
    out, lse = api.qf_kv_attention(c, q, table, torch.tensor([n], dtype=torch.int32, device="cuda"), want_lse=True)
    check_attention(c, q, table, [n], dim ** -0.5, out, lse)


def test_values_far_below_others_where_the_softmax_takes_them():
    """MXFP4: the weight lies on keys whose values are 2^-60 of the other keys'; and on keys whose values are zero."""
    page, heads, dim, n = 16, 1, 128, 64
    c = random_cache(api.FMT_MXFP4, 4, page, heads, dim, 5)
    c.k_scales.fill_(127)
    c.k_codes.fill_(0x22)                                           # every key element 1 ...
    c.k_codes[1] = 0x77                                             # ... but 6 in the second page
    c.v_scales.fill_(140)
    c.v_scales[1] = 80
    q = torch.full((1, 1, 4, dim), 1.0, device="cuda", dtype=BF)
    table = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    for scale in (1.0, 0.05):
        out, lse = api.qf_kv_attention(c, q, table, lens, softmax_scale=scale, want_lse=True)
        check_attention(c, q, table, [n], scale, out, lse)
    c.v_codes[1] = 0
    c.v_scales[1] = 0
    out, lse = api.qf_kv_attention(c, q, table, lens, softmax_scale=0.001, want_lse=True)
    check_attention(c, q, table, [n], 0.001, out, lse)


@fmts
def test_strided_queries_and_given_outputs(fmt):
    g = gen(21)
    batch, q_len, heads, group, dim, page = 3, 2, 2, 4, 128, 16
    lens = [40, 2, 77]
    table, n, pages = paged(lens, page)
    c = random_cache(fmt, pages, page, heads, dim, 6)
    qkv = torch.randn((batch, q_len, (heads * group + 2 * heads) * dim), generator=g, device="cuda").to(BF)
    q = qkv[..., :heads * group * dim].unflatten(-1, (heads * group, dim))
    want, wl = api.qf_kv_attention(c, q.contiguous(), table, n, want_lse=True)
    out, lse = torch.empty_like(want), torch.empty_like(wl)
    ws = api.workspace(api.OP_KV_ATTENTION, batch * q_len, heads * group, dim, heads)
    ws.fill_(0xFF)
    got, gl = api.qf_kv_attention(c, q, table, n, out=out, lse=lse, ws=ws)
    assert got is out and gl is lse and torch.equal(out, want) and torch.equal(lse, wl)
    with pytest.raises(TypeError):
        api.qf_kv_attention(c, q.transpose(0, 1).contiguous().transpose(0, 1), table, n)


@fmts
def test_lengths_and_pages_out_of_contract_stay_inside(fmt):
    """Meaningless numbers, but numbers: the kernel forces lengths and pages into range."""
    c = random_cache(fmt, 4, 16, 2, 64, 6)
    table = torch.tensor([[0, 1], [99, -5], [2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device="cuda")
    q = torch.randn((3, 1, 8, 64), generator=gen(0), device="cuda").to(BF)
    out, lse = api.qf_kv_attention(c, q, table, torch.tensor([2 ** 31 - 1, 32, 20], dtype=torch.int32, device="cuda"), want_lse=True)
    check_attention(c, q[:1], table[:1], [32], 0.125, out[:1], lse[:1])
    assert torch.isfinite(out.float()).all()
    out, lse = api.qf_kv_attention(c, q, table, torch.tensor([-3, -2 ** 31, 0], dtype=torch.int32, device="cuda"), want_lse=True)
    assert (out == 0).all() and torch.isinf(lse).all()


def test_offsets_past_32_bits():
    """Pages in the last part of buffers of more than 4 GB."""
    page, heads, dim = 128, 8, 256
    pages = (1 << 32) // (page * heads * dim // 2) + 40
    c = api.KvCache.empty(api.FMT_NVFP4, pages, page, heads, dim, *tscales(api.FMT_NVFP4))
    assert c.k_codes.numel() > 1 << 32
    g = gen(3)
    n = 300
    table = torch.tensor([[pages - 1, 1, pages - 20]], dtype=torch.int32, device="cuda")
    at = torch.arange(n, device="cuda")
    slots = table[0, at // page].long() * page + at % page
    k, v = (torch.randn((n, heads, dim), generator=g, device="cuda").to(BF) for _ in "kv")
    api.qf_kv_append(c, k, v, slots)
    rk, rv = api.qf_kv_read(c, slots)
    assert np.array_equal(torch_to_bits(rk), torch_to_bits(quantized(api.FMT_NVFP4, k.cpu(), c.k_tscale)[2]))
    assert np.array_equal(torch_to_bits(rv), torch_to_bits(quantized(api.FMT_NVFP4, v.cpu(), c.v_tscale)[2]))
    q = torch.randn((1, 2, 16, dim), generator=g, device="cuda").to(BF)
    out, lse = api.qf_kv_attention(c, q, table, torch.tensor([n], dtype=torch.int32, device="cuda"), want_lse=True)
    check_attention(c, q, table, [n], dim ** -0.5, out, lse)


@fmts
def test_decode_steps_in_a_graph(fmt):
    """A step (write the new token, attend) captured once and replayed with other tokens, lengths and pages, on a stream of its own."""
    batch, heads, group, dim, page, most = 5, 2, 4, 128, 16, 8
    g = gen(17)
    table = torch.randperm(batch * most, generator=g, device="cuda").to(torch.int32).view(batch, most)
    c = filled(fmt, batch * most, page, heads, dim, byte=0xFF)
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    qkv = torch.zeros((batch, 1, heads * (group + 2), dim), dtype=BF, device="cuda")
    ws = api.workspace(api.OP_KV_ATTENTION, batch, heads * group, dim, heads)
    out = torch.empty((batch, 1, heads * group, dim), dtype=BF, device="cuda")

    def step():
        lens.add_(1)
        j = (lens - 1).long()
        slots = table.gather(1, (j // page)[:, None])[:, 0].long() * page + j % page
        api.qf_kv_append(c, qkv[:, 0, heads * group:heads * (group + 1)], qkv[:, 0, heads * (group + 1):], slots)
        api.qf_kv_attention(c, qkv[:, :, :heads * group], table, lens, out=out, ws=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        lens.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        for i in range(40):
            qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda"))
            graph.replay()
            if i in (0, 1, 15, 16, 39):
                check_attention(c, qkv[:, :, :heads * group], table, [i + 1] * batch, dim ** -0.5, out)
    s.synchronize()


@fmts
@pytest.mark.parametrize("max_pages", [4, 64, 2000])
def test_captured_calls_of_every_cut(fmt, max_pages):
    """One CTA a sequence, a cluster, shares with a second kernel: captured twice in a row with one workspace, replayed with other lengths
    and queries, on two graphs that share the workspace one after the other."""
    batch, heads, group, dim, page = 3, 2, 4, 128, 16
    g = gen(max_pages)
    c = random_cache(fmt, 200, page, heads, dim, 7)
    table = torch.randint(0, 200, (batch, max_pages), generator=g, device="cuda", dtype=torch.int32)
    lens = torch.tensor([1, max_pages * page, 0], dtype=torch.int32, device="cuda")
    q = torch.randn((batch, 1, heads * group, dim), generator=g, device="cuda").to(BF)
    ws = api.workspace(api.OP_KV_ATTENTION, batch, heads * group, dim, heads)
    outs = [torch.empty_like(q) for _ in range(4)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        api.qf_kv_attention(c, q, table, lens, out=outs[0], ws=ws)
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        for i, graph in enumerate(graphs):
            with torch.cuda.graph(graph, stream=s):
                api.qf_kv_attention(c, q, table, lens, out=outs[2 * i], ws=ws)
                api.qf_kv_attention(c, outs[2 * i], table, lens, out=outs[2 * i + 1], ws=ws)
        for n in ([5, 30, 64], [0, 0, 0], [max_pages * page, 1, 17]):
            lens.copy_(torch.tensor(n, dtype=torch.int32))
            q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
            for graph in graphs:
                graph.replay()
            first = api.qf_kv_attention(c, q, table, lens)
            second = api.qf_kv_attention(c, first, table, lens)
            for i in (0, 1):
                assert torch.equal(outs[2 * i], first) and torch.equal(outs[2 * i + 1], second)
            check_attention(c, q, table, [min(x, max_pages * page) for x in n], dim ** -0.5, first)
    s.synchronize()


@fmts
def test_two_streams_with_a_workspace_each(fmt):
    cases = []
    for seed in (1, 2):
        lens = [3000 + 100 * seed, 17, 900]
        table, n, pages = paged(lens, 16, seed=seed)
        c = random_cache(fmt, pages, 16, 4, 128, seed)
        q = torch.randn((3, 1, 16, 128), generator=gen(seed), device="cuda").to(BF)
        ws = api.workspace(api.OP_KV_ATTENTION, 3, 16, 128, 4)
        cases.append((c, q, table, n, ws, api.qf_kv_attention(c, q, table, n)))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(20):
        for i, (c, q, table, n, ws, _w) in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                got[i].append(api.qf_kv_attention(c, q, table, n, ws=ws))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(x, cases[i][5]) for x in got[i])


def test_refusals_of_the_binding():
    c = filled(api.FMT_MXFP4, 4, 16, 2, 64)
    x = torch.zeros((3, 2, 64), dtype=BF, device="cuda")
    slots = torch.arange(3, device="cuda")
    for bad in (x.float(), x.cpu()):
        with pytest.raises(TypeError):
            api.qf_kv_append(c, bad, x, slots)
    for args in ((x[:2], x, slots), (x[:, :1], x, slots), (x, x, slots[None])):
        with pytest.raises(ValueError):
            api.qf_kv_append(c, *args)
    with pytest.raises(TypeError):
        api.qf_kv_append(c, x, x.transpose(1, 2).contiguous().transpose(1, 2), slots)
    with pytest.raises(TypeError):
        api.qf_kv_append(c, x, x, slots.float())
    wide = torch.zeros((3, 2 * 64 + 4), dtype=BF, device="cuda")[:, :128].unflatten(1, (2, 64))
    with pytest.raises(api.QfError):                               # tokens 264 bytes apart
        api.qf_kv_append(c, wide, x, slots)
    with pytest.raises(TypeError):
        api.KvCache(api.FMT_NVFP4, c.k_codes, c.k_scales.repeat(1, 1, 1, 2), c.v_codes, c.v_scales.repeat(1, 1, 1, 2))
    with pytest.raises(ValueError):
        api.KvCache(api.FMT_MXFP4, c.k_codes, c.k_scales[:3], c.v_codes, c.v_scales)
    with pytest.raises(api.QfError):
        api.KvCache(api.FMT_Q4_K, c.k_codes, c.k_scales, c.v_codes, c.v_scales)
    q = torch.zeros((1, 1, 3, 64), dtype=BF, device="cuda")
    table, lens = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(api.QfError):                               # three query heads for two key heads
        api.qf_kv_attention(c, q, table, lens)
    q = q[:, :, :2]
    with pytest.raises(TypeError):
        api.qf_kv_attention(c, q, table.long(), lens)
    with pytest.raises(ValueError):
        api.qf_kv_attention(c, q, table, lens.repeat(2))
    with pytest.raises(api.QfError):
        api.qf_kv_attention(c, q, table, lens, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        api.qf_kv_attention(c, torch.zeros((1, 1, 2, 128), dtype=BF, device="cuda"), table, lens)
