"""Grouped layers on a buffer with more rows than the segments take (qf_moe_rows_bound is chosen before the routing is known): what
stands in the rows past the last segment, of X and of dY, has no part in any result, whatever the activation format. A chain of
grouped calls passes such rows on as nobody has written them."""
import pytest
import torch

from paper_2609_39223_b200 import api

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NONE, NV, MX, Q4 = api.FMT_NONE, api.FMT_NVFP4, api.FMT_MXFP4, api.FMT_Q4_K


def draw(*shape, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(BF).cuda()


def grouped(X, W, dY, offs, wq, aq, flags, given):
    G = W.shape[0]
    scales = lambda: dict(w_tscale=torch.empty(G, device="cuda") if wq == NV else None,
                          a_tscale=torch.full((1,), given or 0.0, device="cuda") if aq == NV else None)
    if given and aq == NV:
        flags |= api.A_TSCALE_GIVEN
    s = scales()
    y = api.qf_fq_grouped_linear_fwd(X, W, offs, wq, aq, y_dtype=F32, flags=flags, **s)
    a_scale = None if s["a_tscale"] is None else s["a_tscale"].clone()
    dx, dw = api.qf_fq_grouped_linear_bwd(dY, X, W, offs, wq, aq, dx_dtype=F32, dw_dtype=F32, flags=flags, **scales())
    return y, dx, dw, a_scale


@pytest.mark.parametrize("wq,aq", [(NV, NV), (MX, MX), (NONE, NV), (NV, NONE), (Q4, NONE)])
@pytest.mark.parametrize("flags,given", [(0, None), (api.FUSED_QDQ, None), (0, 2e-3)])
@pytest.mark.parametrize("blocks,tail", [((2, 0, 1), 3), ((1, 3, 2, 1), 1), ((2,), 6), ((2,) + (0,) * 299, 1)])
def test_rows_past_the_last_segment_have_no_part(wq, aq, flags, given, blocks, tail):
    N, K, G = 256, 512, len(blocks)
    rows = 128 * sum(blocks)
    offs = torch.tensor([128 * sum(blocks[:i]) for i in range(G + 1)], dtype=torch.int32, device="cuda")
    X, dY, W = draw(rows, K, seed=1), draw(rows, N, seed=2), draw(G, N, K, seed=3, scale=0.05)
    want = grouped(X, W, dY, offs, wq, aq, flags, given)
    assert all(torch.isfinite(t).all() for t in want if t is not None)
    for filler in (0.0, 3e38, float("inf"), float("nan")):
        more = lambda t: torch.cat([t, torch.full((128 * tail, t.shape[1]), filler, dtype=BF, device="cuda")])
        y, dx, dw, a_scale = grouped(more(X), W, more(dY), offs, wq, aq, flags, given)
        assert torch.equal(y[:rows], want[0]) and torch.equal(dx[:rows], want[1]) and torch.equal(dw, want[2]), filler
        assert a_scale is None or torch.equal(a_scale, want[3]), filler


@pytest.mark.parametrize("end", [0, -128, 1 << 30, 200])
def test_an_end_outside_the_buffer_gives_finite_results(end):
    """The table is the caller's device memory: its last entry is forced into the buffer before it bounds the activations' maximum."""
    rows, N, K = 256, 256, 256
    offs = torch.tensor([0, end], dtype=torch.int32, device="cuda")
    X, W, dY = draw(rows, K, seed=1), draw(1, N, K, seed=2), draw(rows, N, seed=3)
    y, dx, dw, a_scale = grouped(X, W, dY, offs, NV, NV, 0, None)
    top = X[:max(0, min(end, rows)) // 128 * 128].abs().max().float().item() if end >= 128 else 0.0
    assert a_scale.item() == (torch.tensor(top) / 2688.0).item() if top else a_scale.item() == 1.0
    assert torch.isfinite(dw).all()


@pytest.mark.parametrize("aq", [NV, MX, NONE])
def test_a_chain_of_grouped_layers_passes_unwritten_rows_on(aq):
    """dispatch -> product -> product, the memory of every intermediate result full of NaN beforehand."""
    T, k, G, H = 60, 2, 6, 256
    ids = torch.randint(0, G, (T, k), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    plan = api.qf_moe_sort(ids, G, rows_padded=128 * (G + 5))
    x, w1, w2 = draw(T, H, seed=1), draw(G, H, H, seed=2, scale=0.05), draw(G, H, H, seed=3, scale=0.05)
    weights = torch.rand((T, k), generator=torch.Generator().manual_seed(2)).cuda()

    def layer(filler):
        xs = api.qf_moe_dispatch(x, plan)
        for w in (w1, w2):
            Y = torch.full_like(xs, filler)
            ts = torch.empty(G, device="cuda")
            xs = api.qf_fq_grouped_linear_fwd(xs, w, plan.group_offsets, NV, aq, w_tscale=ts, Y=Y)
        return api.qf_moe_combine(xs, weights, plan, out_dtype=F32)
    want = layer(0.0)
    assert torch.isfinite(want).all() and want.abs().max() > 0
    assert torch.equal(layer(float("nan")), want) and torch.equal(layer(3e38), want)
