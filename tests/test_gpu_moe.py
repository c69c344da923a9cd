"""Mixture-of-experts routing on the GPU: the routing table, tokens into expert order, the weighted sum and both gradients,
against plain 64-bit forms.

Tolerances. With u = 2^-24 an FP32 sum of n terms in any order is within n * u * (sum of |terms|) of the exact one, to first
order; the comparisons use twice that. A result rounded to BF16 is another 2^-9 of itself away (2^-8 used)."""
import numpy as np
import pytest
import torch

from paper_2609_39223_b200 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def plain_table(ids: np.ndarray, G: int, rows: int):
    """Pair by pair, from the definition."""
    flat = ids.reshape(-1)
    count = [0] * G
    place = []
    for e in flat:
        if 0 <= e < G:
            place.append((int(e), count[e]))
            count[e] += 1
        else:
            place.append(None)
    offs = [0]
    for c in count:
        offs.append(offs[-1] + (c + 127) // 128 * 128)
    row_of = [-1 if q is None or offs[q[0]] + q[1] >= rows else offs[q[0]] + q[1] for q in place]
    counts = [max(0, min(c, rows - o)) for c, o in zip(count, offs)]
    return np.array(row_of, np.int32).reshape(ids.shape), np.minimum(offs, rows).astype(np.int32), np.array(counts, np.int32)


def draw_ids(rng, T, k, G, kind):
    if kind == "one":
        return np.full((T, k), G - 1)
    if kind == "wild":                                        # a third of the ids name no expert
        ids = rng.integers(0, G, (T, k))
        bad = rng.choice([-1, G, G + 7, -2 ** 31, 2 ** 31 - 1], (T, k))
        return np.where(rng.random((T, k)) < 0.33, bad, ids)
    if kind == "skew":
        return np.minimum(rng.geometric(0.2, (T, k)) - 1, G - 1)
    return rng.integers(0, G, (T, k))


def plan_of(T, k, G, seed=0, kind="even", rows=None, dtype=torch.int32):
    ids = draw_ids(np.random.default_rng(seed), T, k, G, kind)
    plan = api.qf_moe_sort(torch.tensor(ids, dtype=dtype, device="cuda").view(T, k), G, rows_padded=rows)
    return ids, plan


def check_table(ids, plan, G):
    row_of, offs, counts = plain_table(ids, G, plan.rows_padded)
    assert np.array_equal(plan.group_offsets.cpu().numpy(), offs)
    assert np.array_equal(plan.counts.cpu().numpy(), counts)
    assert np.array_equal(plan.row_of.cpu().numpy(), row_of)


@pytest.mark.parametrize("T,k,G", [(1, 1, 1), (1, 8, 128), (3, 2, 5), (7, 8, 128), (33, 8, 37), (511, 1, 2), (1025, 2, 1024), (1000, 3, 300),
                                   (4096, 1, 64), (2600, 8, 128), (9001, 4, 256), (16384, 8, 128)])
@pytest.mark.parametrize("kind", ["even", "one", "wild", "skew"])
def test_sort(T, k, G, kind):
    for dtype in (torch.int32, torch.int64):
        ids, plan = plan_of(T, k, G, seed=T + k, kind=kind, dtype=dtype)
        check_table(ids, plan, G)


@pytest.mark.parametrize("rows", [0, 128, 256, 1024, 2048])
def test_sort_with_too_few_rows_drops_the_last(rows):
    for T in (40, 700, 9000):
        ids, plan = plan_of(T, 2, 9, seed=rows, kind="wild", rows=rows)
        check_table(ids, plan, 9)


def test_sort_of_nothing():
    plan = api.qf_moe_sort(torch.empty((0, 4), dtype=torch.int32, device="cuda"), 6)
    assert plan.rows_padded == 0 and plan.group_offsets.tolist() == [0] * 7 and plan.counts.tolist() == [0] * 6
    ids, plan = plan_of(9, 2, 4, kind="even", rows=512)
    ids[:] = -1
    plan = api.qf_moe_sort(torch.tensor(ids, dtype=torch.int64, device="cuda"), 4, rows_padded=512)
    assert plan.row_of.tolist() == [[-1, -1]] * 9 and plan.counts.tolist() == [0] * 4


def test_sort_of_64_bit_ids_looks_at_all_bits():
    ids = torch.tensor([[2 ** 32 + 1, 1], [-(2 ** 32) + 2, 3]], dtype=torch.int64, device="cuda")
    plan = api.qf_moe_sort(ids, 4)
    assert plan.row_of.tolist() == [[-1, 0], [-1, 128]] and plan.counts.tolist() == [0, 1, 0, 1]


def test_sort_agrees_with_the_host_routing_of_the_benchmark():
    from paper_2609_39223_b200 import synth
    r = synth.moe_routing(1000, 16, 4, seed=3)
    g = torch.Generator().manual_seed(3)
    probs = torch.softmax(torch.randn(1000, 16, generator=g, dtype=torch.float32), -1)
    ids = torch.sort(probs, dim=-1, descending=True, stable=True).indices[:, :4].contiguous()
    plan = api.qf_moe_sort(ids.cuda(), 16)
    assert torch.equal(plan.group_offsets.cpu(), r.group_offsets)
    token_of_row = torch.full((plan.rows_padded,), -1, dtype=torch.int64)
    token_of_row[plan.row_of.cpu().long().reshape(-1)] = torch.arange(1000).repeat_interleave(4)
    assert torch.equal(token_of_row[:r.token_of_row.numel()], r.token_of_row)


# ---- rows there and back ------------------------------------------------------------------------------------------------------

SHAPES = [(1, 1, 1, 8), (1, 8, 128, 2048), (3, 2, 5, 24), (37, 8, 16, 264), (130, 3, 7, 1000), (700, 1, 3, 64), (300, 8, 64, 768), (65, 9, 200, 2056),
          (200, 17, 40, 128)]


def put(shape, seed, dtype, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def close(got, want, terms, n, dtype):
    """got within the bound of the module's docstring: `terms` is the sum of the terms' magnitudes."""
    bound = 2 * n * U * terms + (2.0 ** -8 * want.abs() + 2.0 ** -133 if dtype == BF else 0.0)
    assert torch.isfinite(got.double()).all()
    off = (got.double() - want).abs() - bound
    assert (off <= 0).all(), f"largest excess {off.max().item():.3e}"


@pytest.mark.parametrize("T,k,G,H", SHAPES)
@pytest.mark.parametrize("kind", ["even", "wild", "one"])
def test_dispatch(T, k, G, H, kind):
    for rows in (None, 256):
        _, plan = plan_of(T, k, G, seed=T, kind=kind, rows=rows)
        x = put((T, H), 1, BF)
        xs = api.qf_moe_dispatch(x, plan, xs=torch.full((plan.rows_padded, H), float("nan"), dtype=BF, device="cuda"))
        want = torch.zeros((plan.rows_padded + 1, H), dtype=BF, device="cuda")
        r = plan.row_of.long()
        want[torch.where(r >= 0, r, plan.rows_padded)] = x[:, None].expand(-1, k, -1)
        assert torch.equal(xs, want[:-1])


@pytest.mark.parametrize("T,k,G,H", SHAPES)
@pytest.mark.parametrize("din,dout", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
def test_combine_and_dispatch_gradient(T, k, G, H, din, dout):
    for kind in ("even", "wild"):
        _, plan = plan_of(T, k, G, seed=T + 1, kind=kind)
        ys = put((plan.rows_padded, H), 2, din)
        r = plan.row_of.long()
        owned = torch.zeros(plan.rows_padded, dtype=torch.bool, device="cuda")
        owned[r[r >= 0]] = True
        ys[~owned] = float("nan")                              # padding is never read
        w = put((T, k), 3, F32)
        w[r < 0] = float("inf")                                # nor is the weight of a dropped pair
        y = torch.where((r >= 0)[..., None], ys[r.clamp(min=0)].double(), 0.0)
        wt = torch.where(r >= 0, w.double(), 0.0)[..., None]
        close(api.qf_moe_combine(ys, w, plan, out_dtype=dout), (wt * y).sum(1), (wt * y).abs().sum(1), k + 1, dout)
        close(api.qf_moe_dispatch_bwd(ys, plan, dx_dtype=dout), y.sum(1), y.abs().sum(1), k, dout)


@pytest.mark.parametrize("T,k,G,H", SHAPES)
@pytest.mark.parametrize("ddt,ydt", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
def test_combine_gradient(T, k, G, H, ddt, ydt):
    for kind in ("even", "wild"):
        _, plan = plan_of(T, k, G, seed=T + 2, kind=kind)
        ys = put((plan.rows_padded, H), 4, ydt)
        r = plan.row_of.long()
        owned = torch.zeros(plan.rows_padded, dtype=torch.bool, device="cuda")
        owned[r[r >= 0]] = True
        ys[~owned] = float("nan")
        w, d = put((T, k), 5, F32), put((T, H), 6, ddt)
        w[r < 0] = float("nan")
        dys, dw = api.qf_moe_combine_bwd(d, ys, w, plan, dys=torch.full((plan.rows_padded, H), float("nan"), dtype=BF, device="cuda"),
                                         dweights=torch.full((T, k), float("nan"), device="cuda"))
        want = torch.zeros((plan.rows_padded + 1, H), dtype=torch.float64, device="cuda")
        want[torch.where(r >= 0, r, plan.rows_padded)] = w.double()[..., None] * d.double()[:, None]
        close(dys, want[:-1], want[:-1].abs(), 1, BF)
        assert (dys[~owned] == 0).all()
        terms = torch.where((r >= 0)[..., None], ys[r.clamp(min=0)].double(), 0.0) * d.double()[:, None]
        close(dw, terms.sum(-1), terms.abs().sum(-1), H, F32)
        assert (dw[r < 0] == 0).all()
        only, none = api.qf_moe_combine_bwd(d, None, w, plan, want_dweights=False)
        assert none is None and torch.equal(only, dys)


def test_gradients_against_differences():
    """The weighted sum is linear in the weights and in ys, so a central difference of <dout, out> along a direction equals the
    inner product of the gradient with it, up to the rounding of the FP32 outputs; the same for dispatch."""
    T, k, G, H = 50, 4, 9, 320
    _, plan = plan_of(T, k, G, seed=8, kind="wild")
    ys, w, d = put((plan.rows_padded, H), 1, F32), put((T, k), 2, F32), put((T, H), 3, F32)
    dw = api.qf_moe_combine_bwd(d, ys, w, plan)[1]
    v = put((T, k), 4, F32)
    loss = lambda wt, y: (api.qf_moe_combine(y, wt, plan, out_dtype=F32).double() * d.double()).sum().item()
    size = (api.qf_moe_combine(ys.abs(), w.abs() + v.abs(), plan, out_dtype=F32).double() * d.abs().double()).sum().item()
    got = (loss(w + v, ys) - loss(w - v, ys)) / 2
    want = (dw.double() * v.double()).sum().item()
    assert abs(got - want) <= 2 * (H + k + 4) * U * size
    # along a direction in ys; the gradient's rows are rounded to BF16
    z = put((plan.rows_padded, H), 5, F32)
    dys = api.qf_moe_combine_bwd(d, ys, w, plan)[0]
    got = (loss(w, ys + z) - loss(w, ys - z)) / 2
    want = (dys.double() * z.double()).sum().item()
    size = (api.qf_moe_combine(ys.abs() + z.abs(), w.abs(), plan, out_dtype=F32).double() * d.abs().double()).sum().item()
    assert abs(got - want) <= (2 * (k + 4) * U + 2.0 ** -8) * size
    # dispatch: <dispatch(x), e> = <x, gradient(e)>; its outputs are exact copies
    x, e = put((T, H), 6, BF), put((plan.rows_padded, H), 7, F32)
    got = (api.qf_moe_dispatch(x, plan).double() * e.double()).sum().item()
    back = api.qf_moe_dispatch_bwd(e, plan, dx_dtype=F32)
    size = (api.qf_moe_dispatch(x.abs(), plan).double() * e.abs().double()).sum().item()
    assert abs(got - (back.double() * x.double()).sum().item()) <= 2 * k * U * size


def test_combine_without_a_plan_takes_pairs_in_order():
    T, k, H = 19, 6, 136
    ys, w = put((T * k, H), 1, BF), put((T, k), 2, F32)
    y = ys.double().view(T, k, H) * w.double()[..., None]
    close(api.qf_moe_combine(ys, w, out_dtype=F32), y.sum(1), y.abs().sum(1), k + 1, F32)


def test_infinities_and_nan_stay_in_their_places():
    T, k, G, H = 20, 2, 4, 64
    _, plan = plan_of(T, k, G, seed=1)
    x = put((T, H), 1, BF)
    x[3, 5], x[4, 6] = float("inf"), float("nan")
    xs = api.qf_moe_dispatch(x, plan)
    out = api.qf_moe_combine(xs, torch.full((T, k), 0.5, device="cuda"), plan)
    assert torch.equal(out.isnan(), x.isnan()) and torch.equal(out.isinf(), x.isinf())
    rest = torch.isfinite(x)
    assert torch.equal(out[rest], x[rest])                   # 0.5 x + 0.5 x is exact


def test_a_table_that_breaks_the_contract_stays_in_bounds():
    """Entries outside the buffer are dropped pairs; the outputs around the buffer stay untouched."""
    T, k, G, H, rows = 30, 3, 4, 64, 256
    bad = torch.tensor(np.random.default_rng(0).choice([-7, -1, 256, 300, 2 ** 31 - 1, -2 ** 31], (T, k)), dtype=torch.int32, device="cuda")
    offs = torch.tensor([0, -5, 99999, 128, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    counts = torch.tensor([-3, 2 ** 31 - 1, 4, 500], dtype=torch.int32, device="cuda")
    plan = api.MoePlan(bad, offs, counts, rows)
    room = torch.full((rows + 512, H), 7.0, dtype=BF, device="cuda")
    xs = room[256:256 + rows]
    api.qf_moe_dispatch(put((T, H), 1, BF), plan, xs=xs)
    assert (room[:256] == 7).all() and (room[256 + rows:] == 7).all()
    ys, w = put((rows, H), 2, BF), put((T, k), 3, F32)
    assert (api.qf_moe_combine(ys, w, plan) == 0).all() and (api.qf_moe_dispatch_bwd(ys, plan) == 0).all()
    _, dw = api.qf_moe_combine_bwd(put((T, H), 4, BF), ys, w, plan, dys=xs)
    assert (dw == 0).all() and (room[:256] == 7).all() and (room[256 + rows:] == 7).all()


@pytest.mark.parametrize("T,H", [(0, 64), (5, 0)])
def test_empty_tensors(T, H):
    k, G = 2, 4
    ids = torch.zeros((T, k), dtype=torch.int32, device="cuda")
    plan = api.qf_moe_sort(ids, G, rows_padded=256)
    xs = api.qf_moe_dispatch(torch.zeros((T, H), dtype=BF, device="cuda"), plan)
    assert xs.shape == (256, H) and (xs == 0).all()
    w = torch.ones((T, k), device="cuda")
    assert api.qf_moe_combine(xs, w, plan).shape == (T, H) and api.qf_moe_dispatch_bwd(xs, plan).shape == (T, H)
    dys, dw = api.qf_moe_combine_bwd(torch.zeros((T, H), dtype=BF, device="cuda"), xs, w, plan)
    assert dys.shape == (256, H) and (dys == 0).all() and (dw == 0).all()


def test_repeated_calls_give_the_same_bits():
    T, k, G, H = 3000, 8, 128, 512
    _, plan = plan_of(T, k, G, seed=4)
    ys, w, d = put((plan.rows_padded, H), 2, BF), put((T, k), 3, F32), put((T, H), 4, BF)
    one = (api.qf_moe_combine(ys, w, plan, out_dtype=F32), *api.qf_moe_combine_bwd(d, ys, w, plan))
    for _ in range(3):
        for a, b in zip(one, (api.qf_moe_combine(ys, w, plan, out_dtype=F32), *api.qf_moe_combine_bwd(d, ys, w, plan))):
            assert torch.equal(a, b)


def test_a_buffer_of_more_than_2_31_elements():
    T, k, G, H = 150, 2, 3, 8192
    rows = 2 ** 18 + 256                                       # 2^31 elements and two tiles
    row_of = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    row_of[:, 0] = rows - 1 - torch.arange(T, dtype=torch.int32, device="cuda")
    row_of[:50, 1] = torch.arange(50, dtype=torch.int32, device="cuda")
    offs = torch.tensor([0, 128, rows - 256, rows], dtype=torch.int32, device="cuda")
    plan = api.MoePlan(row_of, offs, torch.tensor([50, 0, 0], dtype=torch.int32, device="cuda"), rows)
    # the last segment is filled from its end: say that all of it is real
    plan.counts[2] = 256
    x = put((T, H), 1, BF)
    xs = torch.full((rows, H), 3.0, dtype=BF, device="cuda")
    api.qf_moe_dispatch(x, plan, xs=xs)
    assert torch.equal(xs[rows - T:].flip(0), x) and torch.equal(xs[:50], x[:50])
    assert (xs[50:128] == 0).all() and (xs[2 ** 17:2 ** 17 + 512] == 0).all() and (xs[rows - 512:rows - 256] == 0).all()
    w = torch.ones((T, k), device="cuda")
    out = api.qf_moe_combine(xs, w, plan)
    assert torch.equal(out[50:], x[50:]) and torch.equal(out[:50], (2 * x[:50].float()).to(BF))
    dys, dw = api.qf_moe_combine_bwd(x, xs, w, plan)
    assert torch.equal(dys[rows - T:].flip(0), x) and (dys[rows - 512:rows - 256] == 0).all()
    want = (x.double() ** 2).sum(-1)
    close(dw[:, 0], want, want, H, F32)


def test_on_another_stream_and_in_a_graph():
    T, k, G, H = 64, 4, 8, 256
    ids = torch.randint(0, G, (T, k), device="cuda", dtype=torch.int32)
    x, w = put((T, H), 1, BF), put((T, k), 2, F32)
    def layer():
        plan = api.qf_moe_sort(ids, G)
        return api.qf_moe_combine(api.qf_moe_dispatch(x, plan), w, plan, out_dtype=F32)
    want = layer()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer()
    ids.copy_((ids + 1) % G)
    x.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, layer())
