"""Products with a few tokens one directly after the other, nothing between them: their launches overlap (the CTAs of one are placed while
the one before it runs), so each has to wait for what the one before wrote, and until it has read what this one overwrites. Every chain
is put behind a few milliseconds of other work, so that the GPU finds all its launches in the queue, and is compared bit for bit
with the same calls, each waited for."""
import math

import pytest
import torch

from paper_2609_39223_b200 import api

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
FMTS = {"nvfp4": api.FMT_NVFP4, "mxfp4": api.FMT_MXFP4, "q4_k": api.FMT_Q4_K}


def weight(fmt, N, K, seed, lead=()):
    """Random codes, with scales that keep the mean square of a row of N(0, 1) values about 1 (MXFP4: powers of two, two of them)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (*lead, N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    gain = math.sqrt(8.5625 * K)                       # mean square of the 16 values of E2M1
    if fmt == api.FMT_NVFP4:                           # block scales of 1
        return codes, torch.full((*lead, N, K // 16), 56, dtype=torch.uint8, device="cuda"), torch.full(lead or (1,), 1 / gain, device="cuda")
    if fmt == api.FMT_MXFP4:
        p = math.floor(math.log2(gain))
        share = (4 * (2 ** p / gain) ** 2 - 1) / 3     # of rows with 2^-p, the others have 2^-(p + 1)
        scales = torch.full((*lead, N, K // 32), 127 - p, dtype=torch.uint8, device="cuda")
        scales[..., torch.rand(N, generator=g, device="cuda") >= share, :] -= 1
        return codes, scales, None
    scales = torch.empty((*lead, N, K // 256, 16), dtype=torch.uint8, device="cuda")
    d = 1 / (32 * math.sqrt(21.25 * K))                # 32 d (q - 7.5)
    scales[..., :4] = torch.tensor([d, 7.5 * d], dtype=torch.float16, device="cuda").view(torch.uint8)
    scales[..., 4:12], scales[..., 12:] = 32 | 2 << 6, 0
    return codes, scales, None


def compare(build, steps, least=1e-3):
    """build(seed) gives the buffers; steps(buffers) yields after every call."""
    def run(seed, wait):
        bufs = build(seed)
        torch.cuda.synchronize()
        if not wait:
            torch.cuda._sleep(8_000_000)
        for _ in steps(bufs):
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return bufs
    for seed in range(6):
        want = run(seed, True)
        assert all(torch.isfinite(w).all() and w.float().abs().max() > least for w in want)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(run(seed, False), want)), seed
    # the same in a graph, whose launches keep their overlap
    bufs = build(0)
    first = [b.clone() for b in bufs]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in steps(bufs):
            pass
    want = run(0, True)
    for _ in range(5):
        for b, f in zip(bufs, first):
            b.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(bufs, want))


def rows(M, K, seed):
    return torch.randn((M, K), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(BF)


def nothing(M, K):
    return torch.full((M, K), float("nan"), dtype=BF, device="cuda")


@pytest.mark.parametrize("kind", FMTS)
@pytest.mark.parametrize("M", [1, 3, 12])
def test_there_and_back(kind, M):
    """a -> b -> a: every product reads what the last one wrote and overwrites what it read."""
    fmt, N = FMTS[kind], 2048
    w = weight(fmt, N, N, 1)

    def steps(bufs):
        a, b = bufs
        for _ in range(20):
            for src, dst in ((a, b), (b, a)):
                api.qf_fq_matvec(fmt, src, *w, Y=dst)
                yield
    compare(lambda seed: [rows(M, N, seed), nothing(M, N)], steps)


@pytest.mark.parametrize("kind", FMTS)
def test_there_and_back_of_small_values(kind):
    """Values around 2^-40, below what FP16 holds: every product reads its X a second time, for the BF16 route."""
    fmt, M, N = FMTS[kind], 5, 2048
    w = weight(fmt, N, N, 1)

    def steps(bufs):
        a, b = bufs
        for _ in range(10):
            for src, dst in ((a, b), (b, a)):
                api.qf_fq_matvec(fmt, src, *w, Y=dst)
                yield
    compare(lambda seed: [rows(M, N, seed) * 2.0 ** -40, nothing(M, N)], steps, least=2.0 ** -50)


@pytest.mark.parametrize("kind", FMTS)
def test_the_last_of_two_writers_stays(kind):
    """A long product and a short one write the same rows; a third reads them."""
    fmt, N, long, short = FMTS[kind], 512, 32768, 256
    wl, ws, wn = weight(fmt, N, long, 1), weight(fmt, N, short, 2), weight(fmt, N, N, 3)
    xl = rows(2, long, 100)

    def steps(bufs):
        xs, y, z = bufs
        for _ in range(10):
            api.qf_fq_matvec(fmt, xl, *wl, Y=y)
            yield
            api.qf_fq_matvec(fmt, xs, *ws, Y=y)
            yield
            api.qf_fq_matvec(fmt, y, *wn, Y=z)
            yield
            api.qf_fq_matvec(fmt, z, *wn, Y=y)
            yield
            xs.copy_(y[:, :short])
            yield
    compare(lambda seed: [rows(2, short, seed), nothing(2, N), nothing(2, N)], steps)


@pytest.mark.parametrize("kind", FMTS)
def test_plain_and_grouped_with_and_without_clusters(kind):
    """Products with clusters, without them and per expert in turn, sharing three buffers."""
    fmt, M, G, wide, narrow = FMTS[kind], 4, 6, 8192, 256
    up, down, experts = weight(fmt, wide, narrow, 1), weight(fmt, narrow, wide, 2), weight(fmt, narrow, narrow, 3, (G,))
    cuts = [api.qf_selftest_matvec_cut(fmt, M, *s) for s in ((wide, narrow), (narrow, wide), (narrow, narrow, G))]
    assert cuts[1].nz > 1 and any(c.nz == 1 for c in cuts)
    ids = torch.tensor([5, 0, 0, 3], device="cuda")

    def steps(bufs):
        a, b, c = bufs
        for _ in range(15):
            api.qf_fq_matvec(fmt, a, *up, Y=b)
            yield
            api.qf_fq_matvec(fmt, b, *down, Y=c)
            yield
            api.qf_fq_grouped_matvec(fmt, c, ids, *experts, Y=a)
            yield
            api.qf_fq_matvec(fmt, a, *up, Y=b)
            yield
            api.qf_fq_matvec(fmt, b, *down, Y=a)
            yield
    compare(lambda seed: [rows(M, narrow, seed), nothing(M, wide), nothing(M, narrow)], steps)
