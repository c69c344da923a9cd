"""Attention over the 4-bit cache in equal shares whose parts are joined by CTA, the way of large batches: more (sequence, head) pairs than CTAs,
in a table too wide for any other way. Most sequences are short, so that the 64-bit form stays quick."""
import numpy as np
import pytest
import torch

from kv_reference import attention, check_attention
from paper_2609_39223_b200 import api
from test_gpu_kv import BF, fmts, gen, paged, random_cache

pytestmark = pytest.mark.gpu

# (head size, new tokens, query heads per key head, sequences, key heads, keys that the table can hold)
BY_CTA = [(128, 1, 4, 64, 8, 8192), (64, 1, 1, 20, 32, 4096), (128, 5, 4, 45, 8, 6000), (256, 3, 8, 40, 4, 3008), (64, 4, 8, 40, 16, 5008),
          (256, 1, 4, 100, 3, 5008), (128, 2, 4, 500, 1, 9008), (64, 2, 6, 40, 16, 4000)]


def lengths(batch, most, q_len):
    """Empty, short, around the length from which sequences are cut, and a few as long as the table."""
    lens = [int(x) for x in np.random.default_rng(batch).integers(0, 150, batch)]
    lens[::9] = [0] * len(lens[::9])
    lens[1:8] = [383, 384, 385, most, 416, q_len - 1, q_len]
    lens[-3:] = [most // 2 + 1, 0, most]
    return lens


@fmts
@pytest.mark.parametrize("dim,q_len,group,batch,heads,most", BY_CTA)
def test_large_batches(fmt, dim, q_len, group, batch, heads, most):
    page = 16
    cut = api.qf_selftest_kv_attention_cut(fmt, batch, q_len, heads * group, heads, dim, page, most // page)
    assert cut.split == -1 and not cut.by_segment and cut.tasks == cut.ctas
    lens = lengths(batch, most, q_len)
    table, n, pages = paged(lens, page, max_pages=most // page)
    c = random_cache(fmt, pages, page, heads, dim, 5)
    q = torch.randn((batch, q_len, heads * group, dim), generator=gen(2), device="cuda").to(BF)
    ws = api.workspace(api.OP_KV_ATTENTION, batch * q_len, heads * group, dim, heads)
    ws.fill_(0xFF)
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:3], 7.0, device="cuda")
    api.qf_kv_attention(c, q, table, n, out=out, lse=lse, ws=ws)
    check_attention(c, q, table, lens, dim ** -0.5, out, lse)
    # again, over what the call left in the workspace, and with no sequence but one
    assert torch.equal(out, api.qf_kv_attention(c, q, table, n, ws=ws))
    only = [0] * batch
    only[batch // 2] = most
    wide = table.clone()
    wide[batch // 2] = table[-1]
    out, lse = api.qf_kv_attention(c, q, wide, torch.tensor(only, dtype=torch.int32, device="cuda"), want_lse=True, ws=ws)
    check_attention(c, q, wide, only, dim ** -0.5, out, lse)


@fmts
@pytest.mark.parametrize("dim,q_len,group", [(64, 1, 4), (128, 1, 4), (128, 3, 8), (256, 2, 4)])
def test_one_batch_in_tables_of_several_widths(fmt, dim, q_len, group):
    """The same rows in every cut that the width leads to, each compared with the first: no further apart than twice what either may be
    off the exact value (a BF16 rounding, 2^-8, and the weights' FP16 form, 2^-11, with the sums' and scores' bounds of the other tests)."""
    lens, page, heads = [700, 3, 0, 260, 129, 1, 500], 16, 2
    table, n, pages = paged(lens, page)
    c = random_cache(fmt, pages, page, heads, dim, 3)
    q = torch.randn((len(lens), q_len, heads * group, dim), generator=gen(4), device="cuda").to(BF)
    ref, rlse, mass, big = attention(c, q, table, lens, dim ** -0.5)
    score = (dim + 4) * 2.0 ** -23 * big
    bound = ref.abs() * 2.0 ** -8 + mass * (2 * score[..., None] + 2.0 ** -20 + 2.0 ** -11) + max(lens) * 2.0 ** -30 * float(mass.max())
    (first, first_lse), ways = api.qf_kv_attention(c, q, table, n, want_lse=True), set()
    for most in (table.shape[1], 100, 400, 2000, 20000):
        wide, _, _ = paged(lens, page, max_pages=most)
        ways.add(api.qf_selftest_kv_attention_cut(fmt, len(lens), q_len, heads * group, heads, dim, page, most))
        out, lse = api.qf_kv_attention(c, q, wide, n, want_lse=True)
        assert ((out.double() - first.double()).abs() <= 2 * bound).all()
        assert torch.equal(torch.isinf(lse), torch.isinf(first_lse))
        some = ~torch.isinf(lse)
        assert ((lse - first_lse).abs()[some] <= 2 * (score + 2.0 ** -20 + rlse.abs() * 2.0 ** -22)[some]).all()
    assert any(w.split > 1 for w in ways) and any(w.split == -1 for w in ways)
