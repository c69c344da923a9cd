"""Attention over the 4-bit cache at the ends of its ranges: values whose size changes along a sequence the other way round than their
scores, NaN and infinities, scores of any size. The 64-bit form and the derived bounds are those of the other attention tests."""
import math

import pytest
import torch

from kv_reference import attention, check_attention, gathered
from paper_2609_39223_b200 import api
from test_gpu_kv import BF, fmts, gen, random_cache

pytestmark = pytest.mark.gpu


def paged_in_order(batch, n, page):
    """A page table of `batch` sequences of n keys each, one behind the other, and the number of pages."""
    each = -(-n // page)
    return torch.arange(batch * each, dtype=torch.int32, device="cuda").view(batch, each), torch.full((batch,), n, dtype=torch.int32, device="cuda"), batch * each


@pytest.mark.parametrize("apart", [20, 27, 33, 45])
@pytest.mark.parametrize("rise", [9, 30, 60, 75])
@pytest.mark.parametrize("dim,q_len,group,batch,heads,n", [(128, 1, 4, 3, 2, 320), (128, 1, 4, 3, 2, 3000), (64, 1, 1, 300, 2, 320), (128, 3, 8, 2, 2, 1500),
                                                           (256, 2, 8, 2, 1, 1500), (64, 4, 8, 40, 4, 1600)])
def test_values_that_grow_where_scores_fall(dim, q_len, group, batch, heads, n, rise, apart):
    """MXFP4: units of 32 keys in turn, one with high scores and small values, one with scores 2^-apart below and values 2^rise above, in either
    order; then the first kind behind the second for good, and the other way round; and values of zero under the high scores."""
    page = 32
    table, lens, pages = paged_in_order(batch, n, page)
    c = random_cache(api.FMT_MXFP4, pages, page, heads, dim, 3)
    c.k_scales.fill_(127)
    place = torch.arange(pages, device="cuda") % table.shape[1]
    q = torch.ones((batch, q_len, heads * group, dim), dtype=BF, device="cuda")
    scale = apart * math.log(2.0) / (2 * dim)                       # keys of 1 and -1
    half = table.shape[1] // 2
    for large in (place % 2 == 1, place % 2 == 0, place >= half, place < half, place % 5 == 3):
        c.k_codes.copy_(torch.where(large, 0xAA, 0x22).to(torch.uint8)[:, None, None, None].expand_as(c.k_codes))
        c.v_scales.copy_(torch.where(large, 100 + rise, 100).to(torch.uint8)[:, None, None, None].expand_as(c.v_scales))
        out, lse = api.qf_kv_attention(c, q, table, lens, softmax_scale=scale, want_lse=True)
        check_attention(c, q[:2], table[:2], [n] * min(batch, 2), scale, out[:2], lse[:2])
    c.v_scales.copy_(torch.where(large, 127, 0).to(torch.uint8)[:, None, None, None].expand_as(c.v_scales))
    codes = c.v_codes.clone()
    c.v_codes.mul_(large[:, None, None, None].to(torch.uint8))
    out, lse = api.qf_kv_attention(c, q, table, lens, softmax_scale=scale, want_lse=True)
    check_attention(c, q[:2], table[:2], [n] * min(batch, 2), scale, out[:2], lse[:2])
    c.v_codes.copy_(codes)
    # several levels, each further down in scores and further up in values than the one before, over and over and back
    level = (place % 6 - 3).abs()                                   # 3 2 1 0 1 2
    c.k_codes.fill_(0x22)
    c.k_scales.copy_((127 - level).to(torch.uint8)[:, None, None, None].expand_as(c.k_scales))
    c.v_scales.copy_((60 + level * rise * 2 // 3).to(torch.uint8)[:, None, None, None].expand_as(c.v_scales))
    out, lse = api.qf_kv_attention(c, q, table, lens, softmax_scale=2 * scale, want_lse=True)
    check_attention(c, q[:2], table[:2], [n] * min(batch, 2), 2 * scale, out[:2], lse[:2])


# (batch, key heads, keys of each): a sequence and head to a warp, a CTA, a cluster; in equal shares, joined by sequence and head or by CTA.
# What the sizes are there for is looked at in test_kv_cut.py.
WAYS = {"warps": (300, 2, 100), "CTAs": (100, 3, 600), "small clusters": (30, 3, 600), "clusters": (2, 2, 1000), "shares": (2, 2, 30000),
        "shares by CTA": (80, 8, 2000)}
CUTS = pytest.mark.parametrize("batch,heads,n", WAYS.values(), ids=[w.replace(" ", "-") for w in WAYS])


@fmts
@CUTS
@pytest.mark.parametrize("dim,q_len,group", [(64, 1, 3), (128, 2, 8), (256, 2, 8)])
def test_queries_with_nan_and_infinity(fmt, dim, q_len, group, batch, heads, n):
    """NaN in the outputs and the logarithm of such a row, as the formula has it, and in no other. (The others' last bits may
    differ: the bases of a tile's rows move together, where any of them has to, and a weight 2^(score - base) is rounded to FP16. So they are held
    to the bounds, which no base enters.)"""
    table, lens, pages = paged_in_order(batch, n, 16)
    c = random_cache(fmt, pages, 16, heads, dim, 3)
    q = torch.randn((batch, q_len, heads * group, dim), generator=gen(1), device="cuda").to(BF)
    clean, (clean_out, clean_lse) = q.clone(), api.qf_kv_attention(c, q, table, lens, want_lse=True)
    rows = torch.zeros(q.shape[:3], dtype=torch.bool, device="cuda")
    for i, what in enumerate((math.nan, math.inf, -math.inf)):
        at = (i % batch, (i + 1) % q_len, (2 * i) % (heads * group))
        q[at][(7 * i) % dim] = what
        rows[at] = True
    rows[0, 0, 1] = True
    q[0, 0, 1] = math.nan
    out, lse = api.qf_kv_attention(c, q, table, lens, want_lse=True)
    assert torch.isnan(out[rows]).all() and torch.isnan(lse[rows]).all()
    out, lse = torch.where(rows[..., None], clean_out, out), torch.where(rows, clean_lse, lse)
    check_attention(c, clean[:3], table[:3], lens[:3], dim ** -0.5, out[:3], lse[:3])
    assert torch.equal(out[3:], clean_out[3:]) and torch.equal(lse[3:], clean_lse[3:])


@fmts
@CUTS
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_tokens_before_one_of_nans(fmt, dim, batch, heads, n):
    """Four tokens of every sequence, the last of which was written with keys and values of NaN: the three that do not see it stay as they
    are. NVFP4: the one that sees it takes it for what qf_kv_read says."""
    table, lens, pages = paged_in_order(batch, n, 16)
    c = random_cache(fmt, pages, 16, heads, dim, 3)
    at = (lens - 1).long()
    slots = table.gather(1, (at // 16)[:, None])[:, 0].long() * 16 + at % 16
    x = torch.full((batch, heads, dim), math.nan, dtype=BF, device="cuda")
    api.qf_kv_append(c, x, x, slots)
    q = torch.randn((batch, 4, heads * 2, dim), generator=gen(1), device="cuda").to(BF)
    q[:, 3] = 0                                                     # scores of 0: the mean of all values
    out, lse = api.qf_kv_attention(c, q, table, lens, want_lse=True)
    check_attention(c, q[:3, :3], table[:3], lens[:3] - 1, dim ** -0.5, out[:3, :3], lse[:3, :3])
    assert torch.isfinite(out[:, :3].float()).all()
    if fmt == api.FMT_NVFP4:
        for b in range(min(batch, 3)):
            every = table[b].long().repeat_interleave(16) * 16 + torch.arange(16, device="cuda").repeat(table.shape[1])
            _, v = api.qf_kv_read(c, every[:n], want_k=False)
            mean, mass = v.double().mean(0).repeat_interleave(2, 0), v.double().abs().mean(0).repeat_interleave(2, 0)
            # BF16 values read back and the BF16 result are off by half a step, 2^-8, weights by 2^-11, sums by less than 2^-19
            assert ((out[b, 3].double() - mean).abs() <= mean.abs() * 2.0 ** -8 + mass * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -19)).all()
            assert (lse[b, 3].double() - math.log(n)).abs().max() <= 2.0 ** -20 * (1.0 + math.log(n))


def test_tensor_scales_at_the_ends_of_their_range():
    """NVFP4: products that are in range although a tensor scale is 2^-126 or 2^124."""
    table, lens, pages = paged_in_order(3, 200, 16)
    c = random_cache(api.FMT_NVFP4, pages, 16, 2, 128, 3, scale_bytes=(0x08, 0x10))            # block scales of 2^-6 and a little more
    for k, v, size in ((-126, 124, 2.0 ** 120), (124, -120, 2.0 ** -124)):
        c.k_tscale.fill_(2.0 ** k)
        c.v_tscale.fill_(2.0 ** v)
        q = (torch.randn((3, 2, 4, 128), generator=gen(k + 200), device="cuda") * size).to(BF)
        out, lse = api.qf_kv_attention(c, q, table, lens, want_lse=True)
        # Outputs of 2^-128 are BF16 subnormals, whose steps are 2^-133 whatever the value: half a step, 2^-134, is more than 2^-8 of
        # them. Moved towards the exact value by up to that much, they have to meet the bounds of the other tests.
        ref = attention(c, q, table, lens, 128 ** -0.5)[0]
        near = out.double() + (ref - out.double()).clamp(-2.0 ** -134, 2.0 ** -134)
        check_attention(c, q, table, lens, 128 ** -0.5, near, lse)


def scored(c, q, table, n, scale):
    """The form in FP32 for scores so far apart, or so large, that only their order matters: exact sums, scores rounded to FP32, their
    differences taken from the rounded ones, in 64 bits from there."""
    page, batch, q_len, q_heads, dim = c.page_size, *q.shape
    out, lse = torch.empty(q.shape, dtype=torch.float64, device=q.device), torch.empty(q.shape[:3], dtype=torch.float64, device=q.device)
    for b in range(batch):
        k, v = gathered(c, table[b], n)
        for i in range(q_len):
            m = n - q_len + i + 1
            s = (torch.einsum("hgd,hjd->hgj", q[b, i].double().view(c.kv_heads, -1, dim), k[:, :m]) * scale).float().double()
            out[b, i] = torch.einsum("hgj,hjd->hgd", torch.softmax(s, -1), v[:, :m]).reshape(q_heads, dim)
            lse[b, i] = torch.logsumexp(s, -1).reshape(-1)
    return out, lse


@fmts
@CUTS
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_size(fmt, dim, sign, batch, heads, n):
    """Equal keys, all of whose scores are +-2^20 to +-2^118: the mean of the values. Keys of two kinds that far apart: the mean over one."""
    table, lens, pages = paged_in_order(batch, n, 32)
    c = random_cache(fmt, pages, 32, heads, dim, 3)
    c.k_codes.fill_(0x22)
    for power in (20, 27, 31, 40, 80, 118):
        k = power // 2 if fmt == api.FMT_MXFP4 else 2
        c.k_scales.fill_(127 + k if fmt == api.FMT_MXFP4 else 0x38)          # keys of 2^k and of 1 times the tensor scale
        if fmt == api.FMT_NVFP4:
            c.k_tscale.fill_(2.0 ** k)
        # queries of seven bits, so that no product is a power of two and sums are exact
        q = torch.full((batch, 2, heads * 2, dim), sign * 1.3125 * 2.0 ** (power - k), dtype=BF, device="cuda")
        q[:, 0] *= -1.171875
        out, lse = api.qf_kv_attention(c, q, table, lens, softmax_scale=0.7 / dim, want_lse=True)
        few = min(batch, 3)
        ref, rlse = scored(c, q[:few], table, n, 0.7 / dim)
        # weights of equal scores are equal but for their FP16 form, 2^-11; one rounding to BF16, 2^-8; their sums, 2^-19: of values of up to 6
        assert torch.isfinite(out.float()).all()
        assert ((out[:few].double() - ref).abs() <= ref.abs() * 2.0 ** -8 + 8 * 2.0 ** -11).all()
        assert ((lse[:few].double() - rlse).abs() <= rlse.abs() * 2.0 ** -21 + 2.0 ** -10).all()
    flip = (torch.arange(pages, device="cuda") % 3 == 1)[:, None, None, None]
    c.k_codes.copy_(torch.where(flip, 0xAA, 0x22).to(torch.uint8).expand_as(c.k_codes))        # the other sign
    out, lse = api.qf_kv_attention(c, q, table, lens, softmax_scale=0.7 / dim, want_lse=True)
    ref, rlse = scored(c, q[:few], table, n, 0.7 / dim)
    assert ((out[:few].double() - ref).abs() <= ref.abs() * 2.0 ** -8 + 8 * 2.0 ** -11).all()
    assert ((lse[:few].double() - rlse).abs() <= rlse.abs() * 2.0 ** -21).all()


@CUTS
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("power", [-105, -110, -113, -116, -120])
def test_small_queries_of_large_keys(dim, power, batch, heads, n):
    """MXFP4: block scales of the keys up to 2^102, the largest that no sum of products can take out of FP32's range, and queries so
    small that scores are ordinary ones or close to 0."""
    table, lens, pages = paged_in_order(batch, n, 16)
    c = random_cache(api.FMT_MXFP4, pages, 16, heads, dim, 3)
    c.k_scales.add_(102)                                            # 225 .. 229
    q = (torch.randn((batch, 2, heads * 2, dim), generator=gen(1), device="cuda") * 2.0 ** power).to(BF)
    q[:, 1] = 2.0 ** power                                          # all of one sign, as the keys below
    out, lse = api.qf_kv_attention(c, q, table, lens, want_lse=True)
    check_attention(c, q[:3], table[:3], lens[:3], dim ** -0.5, out[:3], lse[:3])
    c.k_codes.copy_(torch.where((torch.arange(pages, device="cuda") % 3 == 0)[:, None, None, None], 0x77, 0xFF).to(torch.uint8).expand_as(c.k_codes))
    c.k_scales.fill_(229)
    out, lse = api.qf_kv_attention(c, q, table, lens, want_lse=True)
    check_attention(c, q[:3], table[:3], lens[:3], dim ** -0.5, out[:3], lse[:3])
