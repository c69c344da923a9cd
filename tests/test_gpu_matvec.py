"""Products with a few tokens from 4-bit codes, against a plain 64-bit form that decodes codes and scales by the formats'
definitions.

Tolerance. The kernels add up in FP32, partly in tensor-core accumulators, which may truncate (2^-23 per step). For a contraction
of length K the error is held to sqrt(K) * 2^-22 * S, S being the sum of the magnitudes of all terms: no chain of additions
may be longer than about 2 sqrt(K) steps even if every step errs by its most in the same direction. BF16 results are another 2^-9
of themselves away (2^-8 used)."""
import numpy as np
import pytest
import torch

from paper_2609_39223_b200 import api, synth

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
FMTS = [api.FMT_NVFP4, api.FMT_MXFP4, api.FMT_Q4_K]
E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])


def e4m3(b):
    e, m = (b >> 3).astype(np.float64), (b & 7).astype(np.float64)
    return np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7))


def decode(fmt, codes, scales, ts):
    """(values, magnitudes of what they are the difference of) [rows, cols] in 64 bits, from the formats' definitions."""
    rows, cols = codes.shape[0], codes.shape[1] * 2
    if fmt == api.FMT_Q4_K:
        w, a = np.empty((rows, cols)), np.empty((rows, cols))
        meta = scales.reshape(rows, cols // 256, 16)
        f = np.ascontiguousarray(meta[..., :4]).view(np.float16).astype(np.float64)
        for b in range(8):
            if b < 4:
                s6, m6 = meta[..., 4 + b] & 63, meta[..., 8 + b] & 63
            else:
                s6 = (meta[..., 8 + b] & 15) | (meta[..., b] >> 6 << 4)
                m6 = (meta[..., 8 + b] >> 4) | (meta[..., 4 + b] >> 6 << 4)
            byte = codes.reshape(rows, cols // 256, 4, 32)[:, :, b // 2]
            q = (byte >> 4 if b & 1 else byte & 15).astype(np.float64)
            es, em = f[..., :1] * s6[..., None], f[..., 1:] * m6[..., None]
            w.reshape(rows, cols // 256, 8, 32)[:, :, b] = es * q - em
            a.reshape(rows, cols // 256, 8, 32)[:, :, b] = np.abs(es * q) + np.abs(em)
        return w, a
    v = E2M1[np.stack([codes & 15, codes >> 4], -1).reshape(rows, cols)]
    s = e4m3(scales) * float(ts) if fmt == api.FMT_NVFP4 else 2.0 ** (scales.astype(np.float64) - 127)
    w = v * np.repeat(s, api.BLOCK[fmt], 1)
    return w, np.abs(w)


def draw(fmt, lead, N, K, seed, wide=False):
    """Random codes and scales: every code, scales of a trained weight's size or (wide) over most of their range."""
    r = np.random.default_rng(seed)
    codes = r.integers(0, 256, (*lead, N, K // 2), dtype=np.uint8)
    ts = None
    if fmt == api.FMT_Q4_K:
        scales = r.integers(0, 256, (*lead, N, K // 256, 16), dtype=np.uint8)
        f = (r.uniform(0.5, 2, (*lead, N, K // 256, 2)) * 2.0 ** (r.integers(-12, 8) if wide else -10)).astype(np.float16)
        scales[..., :4] = f.view(np.uint8).reshape(*lead, N, K // 256, 4)
    elif fmt == api.FMT_MXFP4:
        scales = r.integers(20, 230, (*lead, N, 1), dtype=np.uint8) + r.integers(0, 8, (*lead, N, K // 32), dtype=np.uint8) if wide else \
            r.integers(117, 125, (*lead, N, K // 32), dtype=np.uint8)
    else:
        scales = r.integers(0, 127, (*lead, N, K // 16), dtype=np.uint8) if wide else r.integers(88, 127, (*lead, N, K // 16), dtype=np.uint8)
        ts = (r.uniform(0.5, 2, lead or (1,)) * 1e-4).astype(np.float32)
    return codes, scales, ts


def gpu(*arrays):
    return [None if a is None else torch.tensor(a, device="cuda") for a in arrays]


def acts(shape, seed):
    return synth.activations_with_outlier_channels(*shape, seed=seed)


def check(got, x, w, a, dtype):
    """got [M, N] against x [M, K] . w [N, K]^T"""
    want, size = x @ w.T, np.abs(x) @ a.T
    bound = np.sqrt(x.shape[-1]) * 2.0 ** -22 * size + (2.0 ** -8 * np.abs(want) if dtype == BF else 0) + 1e-45
    off = np.abs(got.double().cpu().numpy() - want) - bound
    assert np.isfinite(off).all() and (off <= 0).all(), f"largest excess {off.max():.3e}"


SHAPES = [(1, 1, 1), (1, 7, 3), (1, 300, 1), (2, 16, 2), (3, 17, 5), (5, 100, 7), (7, 33, 16), (8, 64, 9), (9, 31, 4), (16, 129, 8), (17, 48, 3), (32, 40, 11), (33, 25, 2),
          (70, 18, 6), (1, 4100, 16), (4, 2000, 33), (2, 15, 56)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,blocks", SHAPES)
def test_matvec(fmt, M, N, blocks):
    for unit in {1: [256], 2: [32, 32 * 3], 3: [16, 48]}[{api.FMT_Q4_K: 1, api.FMT_MXFP4: 2, api.FMT_NVFP4: 3}[fmt]]:
        K = unit * blocks
        codes, scales, ts = draw(fmt, (), N, K, seed=M + N)
        x = acts((M, K), M)
        w, a = decode(fmt, codes, scales, None if ts is None else ts[0])
        c, s, t = gpu(codes, scales, ts)
        for dtype in (BF, F32):
            Y = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
            check(api.qf_fq_matvec(fmt, x.cuda(), c, s, t, Y=Y), x.double().numpy(), w, a, dtype)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("K", [256, 512, 768, 1024, 2048, 4096, 4352, 14336])
def test_matvec_over_lengths(fmt, K):
    for M, N in ((1, 200), (6, 90), (20, 50)):
        codes, scales, ts = draw(fmt, (), N, K, seed=K + M)
        x = acts((M, K), M)
        w, a = decode(fmt, codes, scales, None if ts is None else ts[0])
        check(api.qf_fq_matvec(fmt, x.cuda(), *gpu(codes, scales, ts), y_dtype=F32), x.double().numpy(), w, a, F32)


@pytest.mark.parametrize("fmt", FMTS)
def test_every_code_in_every_place(fmt):
    """One-hot activations read out the dequantized weights: exact in FP32 (one product, or two and a difference)."""
    K = 256
    N = 64
    codes, scales, ts = draw(fmt, (), N, K, seed=5, wide=True)
    w, _ = decode(fmt, codes, scales, None if ts is None else ts[0])
    c, s, t = gpu(codes, scales, ts)
    x = torch.eye(K, dtype=BF, device="cuda")
    got = api.qf_fq_matvec(fmt, x, c, s, t, y_dtype=F32).double().cpu().numpy()
    assert np.allclose(got, w.T, rtol=2.0 ** -22, atol=0) if fmt != api.FMT_Q4_K else np.abs(got - w.T).max() <= 2.0 ** -22 * np.abs(w).max() + \
        2.0 ** -22 * decode(fmt, codes, scales, None)[1].max()


@pytest.mark.parametrize("code", [0, 1, 2, 60, 126, 127, 128, 129, 130, 190, 250, 252])
def test_mxfp4_scales_over_the_whole_range(code):
    """Block scales 2^-127 .. 2^125 with activations that keep the result in range."""
    N, K, M = 24, 320, 3
    r = np.random.default_rng(code)
    codes = r.integers(0, 256, (N, K // 2), dtype=np.uint8)
    scales = np.full((N, K // 32), code, np.uint8)
    x = (torch.randn((M, K), generator=torch.Generator().manual_seed(code)) * 2.0 ** (20 if code < 64 else -20 if code > 190 else 0)).to(BF)
    w, a = decode(api.FMT_MXFP4, codes, scales, None)
    check(api.qf_fq_matvec(api.FMT_MXFP4, x.cuda(), *gpu(codes, scales, None), y_dtype=F32), x.double().numpy(), w, a, F32)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("spread", [0, 20, 60])
def test_activations_over_many_binades(fmt, spread):
    """Large activations meet zero weights, so that the small ones decide the result."""
    N, K, M = 40, 1024, 5
    codes, scales, ts = draw(fmt, (), N, K, seed=spread)
    r = np.random.default_rng(1)
    x = (r.standard_normal((M, K)) * 2.0 ** r.integers(-spread, spread + 1, (M, K))).astype(np.float32)
    if fmt != api.FMT_Q4_K:
        codes[:, :K // 4] = 0                                 # the first half of the weights is zero
        x[:, :K // 2] *= 2.0 ** 40
    x = torch.tensor(x).to(BF)
    w, a = decode(fmt, codes, scales, None if ts is None else ts[0])
    check(api.qf_fq_matvec(fmt, x.cuda(), *gpu(codes, scales, ts), y_dtype=F32), x.double().numpy(), w, a, F32)


@pytest.mark.parametrize("fmt", FMTS)
def test_from_the_quantizer_and_against_the_training_product(fmt):
    """What qf_qdq emits goes in as it is; the result is the training path's up to the BF16 rounding of its weights
    (2^-9 of each, 2^-8 used)."""
    N, K, M = 264, 2048, 6
    W, x = synth.weight_with_outliers(N, K, seed=2).cuda(), acts((M, K), 3).cuda()
    q = api.qf_qdq(fmt, W)
    got = api.qf_fq_matvec(fmt, x, q["codes"], q["scales"], q["tensor_scale"], y_dtype=F32).double()
    train = api.qf_fq_linear_fwd(x, W, fmt, api.FMT_NONE, y_dtype=F32).double()
    size = x.double().abs() @ q["out"].double().abs().T
    assert ((got - train).abs() <= (2.0 ** -8 if fmt != api.FMT_MXFP4 else 0) * size + 2 * K ** 0.5 * 2.0 ** -22 * size).all()
    w, a = decode(fmt, q["codes"].cpu().numpy(), q["scales"].cpu().numpy().reshape(N, -1) if fmt != api.FMT_Q4_K else q["scales"].cpu().numpy(),
                  None if q["tensor_scale"] is None else q["tensor_scale"].item())
    check(got, x.double().cpu().numpy(), w, a, F32)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("T,k,G,N,blocks", [(1, 1, 1, 20, 1), (1, 8, 128, 33, 2), (3, 2, 5, 16, 3), (2, 4, 300, 70, 1), (24, 8, 16, 40, 3), (40, 3, 7, 18, 5), (90, 1, 2, 17, 2),
                                            (11, 6, 64, 500, 4)])
@pytest.mark.parametrize("kind", ["even", "one", "wild"])
def test_grouped_matvec(fmt, T, k, G, N, blocks, kind):
    K = blocks * (256 if fmt == api.FMT_Q4_K else 96 if fmt == api.FMT_MXFP4 else 80)
    r = np.random.default_rng(T + G)
    ids = np.full((T, k), G // 2) if kind == "one" else r.integers(0, G, (T, k))
    if kind == "wild":
        ids = np.where(r.random((T, k)) < 0.3, r.choice([-1, G, 2 ** 31 - 1, -2 ** 31], (T, k)), ids)
    codes, scales, ts = draw(fmt, (G,), N, K, seed=G)
    c, s, t = gpu(codes, scales, ts)
    for own_rows, idt, dtype in ((False, torch.int32, F32), (True, torch.int64, BF)):
        x = acts((T * k if own_rows else T, K), 4)
        Y = torch.full((T * k, N), float("nan"), dtype=dtype, device="cuda")
        got = api.qf_fq_grouped_matvec(fmt, x.cuda(), torch.tensor(ids, dtype=idt, device="cuda"), c, s, t, Y=Y)
        for e in np.unique(ids):
            at = np.nonzero(ids.reshape(-1) == e)[0]
            if not 0 <= e < G:
                assert (got[torch.tensor(at)] == 0).all()
                continue
            w, a = decode(fmt, codes[e], scales[e], None if ts is None else ts[e])
            check(got[torch.tensor(at).cuda()], x.double().numpy()[at if own_rows else at // k], w, a, dtype)


@pytest.mark.parametrize("fmt", FMTS)
def test_grouped_matvec_with_more_pairs_than_a_cta_lists_at_once(fmt):
    """1024 pairs are listed in one go: experts whose pairs lie on both sides, and a last one."""
    T, k, G, N, K = 700, 3, 5, 40, 256
    r = np.random.default_rng(3)
    ids = r.integers(0, G, (T, k))
    ids[:, 0] = np.where(np.arange(T) == T - 1, 4, ids[:, 0] % 4)
    codes, scales, ts = draw(fmt, (G,), N, K, seed=1)
    x = acts((T, K), 1)
    got = api.qf_fq_grouped_matvec(fmt, x.cuda(), torch.tensor(ids, device="cuda"), *gpu(codes, scales, ts), y_dtype=F32)
    for e in range(G):
        at = np.nonzero(ids.reshape(-1) == e)[0]
        w, a = decode(fmt, codes[e], scales[e], None if ts is None else ts[e])
        check(got[torch.tensor(at).cuda()], x.double().numpy()[at // k], w, a, F32)


@pytest.mark.parametrize("fmt,unit", [(api.FMT_NVFP4, 16), (api.FMT_MXFP4, 32)])
@pytest.mark.parametrize("blocks", [1, 2, 3, 5, 7, 9, 15, 17, 31, 33, 65, 129])
def test_contractions_of_any_number_of_blocks(fmt, unit, blocks):
    """Rows that begin anywhere a block can, in tensors that end with their last block."""
    K = unit * blocks
    for M, N in ((1, 37), (3, 161), (11, 18)):
        codes, scales, ts = draw(fmt, (), N, K, seed=blocks + M)
        x = acts((M, K), M)
        w, a = decode(fmt, codes, scales, None if ts is None else ts[0])
        check(api.qf_fq_matvec(fmt, x.cuda(), *gpu(codes, scales, ts), y_dtype=F32), x.double().numpy(), w, a, F32)


@pytest.mark.parametrize("fmt", FMTS)
def test_rows_do_not_influence_one_another(fmt):
    """The same row of X gives the same bits, whatever stands beside it; NaN and infinities stay in their rows."""
    N, K = 70, 512
    codes, scales, ts = gpu(*draw(fmt, (), N, K, seed=9))
    x = acts((9, K), 1).cuda()
    want = api.qf_fq_matvec(fmt, x, codes, scales, ts, y_dtype=F32)
    x2 = x.clone()
    x2[3, 7], x2[8, 100] = float("nan"), float("inf")
    got = api.qf_fq_matvec(fmt, x2, codes, scales, ts, y_dtype=F32)
    keep = [i for i in range(9) if i not in (3, 8)]
    assert torch.equal(got[keep], want[keep]) and got[3].isnan().any() and not torch.isfinite(got[8]).all()


def test_empty_products():
    for fmt in FMTS:
        codes, scales, ts = gpu(*draw(fmt, (), 12, 256, seed=1))
        assert api.qf_fq_matvec(fmt, torch.empty((0, 256), dtype=BF, device="cuda"), codes, scales, ts).shape == (0, 12)
        assert api.qf_fq_matvec(fmt, torch.ones((3, 256), dtype=BF, device="cuda"), codes[:0], scales[:0], ts).shape == (3, 0)
        y = api.qf_fq_matvec(fmt, torch.empty((3, 0), dtype=BF, device="cuda"), torch.empty((12, 0), dtype=torch.uint8, device="cuda"),
                             torch.empty(api.scales_shape(fmt, 12, 0), dtype=torch.uint8, device="cuda"), ts)
        assert y.shape == (3, 12) and (y == 0).all()
        ids = torch.empty((0, 4), dtype=torch.int32, device="cuda")
        assert api.qf_fq_grouped_matvec(fmt, torch.empty((0, 256), dtype=BF, device="cuda"), ids, codes[None], scales[None], ts).shape == (0, 12)


@pytest.mark.parametrize("fmt", FMTS)
def test_codes_past_2_32_bytes(fmt):
    """A weight of more than 2^33 elements; only its first and last rows are decoded for the comparison."""
    K = 65536
    N = 2 ** 33 // K + 40
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    if fmt == api.FMT_Q4_K:
        scales = torch.randint(0, 256, (N, K // 256, 16), generator=g, device="cuda", dtype=torch.uint8)
        scales[..., :4] = torch.tensor(np.array([0.001, 0.002], np.float16).view(np.uint8), device="cuda")
    else:
        lo, hi = (88, 127) if fmt == api.FMT_NVFP4 else (117, 125)
        scales = torch.randint(lo, hi, api.scales_shape(fmt, N, K), generator=g, device="cuda", dtype=torch.uint8)
    ts = torch.tensor([2e-4], device="cuda") if fmt == api.FMT_NVFP4 else None
    x = acts((2, K), 1)
    got = api.qf_fq_matvec(fmt, x.cuda(), codes, scales, ts, y_dtype=F32)
    at = torch.cat([torch.arange(3), torch.arange(N - 21, N)])
    w, a = decode(fmt, codes[at].cpu().numpy(), scales[at].cpu().numpy(), None if ts is None else ts.item())
    check(got[:, at], x.double().numpy(), w, a, F32)


def test_on_another_stream_and_in_a_graph():
    fmt, N, K = api.FMT_NVFP4, 300, 1024
    codes, scales, ts = gpu(*draw(fmt, (6,), N, K, seed=2))
    x, ids = acts((5, K), 1).cuda(), torch.randint(0, 6, (5, 2), device="cuda")
    def both():
        return api.qf_fq_matvec(fmt, x, codes[1], scales[1], ts[1:2], y_dtype=F32), api.qf_fq_grouped_matvec(fmt, x, ids, codes, scales, ts, y_dtype=F32)
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    x.mul_(-3)
    ids.copy_((ids + 1) % 6)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(held, both()))


@pytest.mark.parametrize("fmt", FMTS)
def test_calls_one_after_another_see_what_the_last_one_wrote(fmt):
    """A chain of short products in the same buffers, each reading what the one before wrote (their launches overlap), gives the bits of
    the same chain with a wait after every call."""
    N = K = 1024
    codes, scales, ts = gpu(*draw(fmt, (), N, K, seed=3))
    def chain(wait):
        a, b = acts((3, K), 5).cuda(), torch.empty((3, N), dtype=BF, device="cuda")
        for _ in range(60):
            for src, dst in ((a, b), (b, a)):
                api.qf_fq_matvec(fmt, src, codes, scales, ts, Y=dst)
                if wait:
                    torch.cuda.synchronize()
                dst.div_(dst.abs().amax() / 4)
                if wait:
                    torch.cuda.synchronize()
            api.qf_fq_matvec(fmt, a, codes, scales, ts, Y=b)          # two products of ours in a row
            api.qf_fq_matvec(fmt, b.clamp_(-8, 8), codes, scales, ts, Y=a)
            a.div_(a.abs().amax() / 4)
        return a
    assert torch.equal(chain(False), chain(True))
