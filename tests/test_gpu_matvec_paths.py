"""Products with a few tokens over every way in which the kernel cuts them: one or several row tiles for a CTA, the contraction
whole, split over the warps of a CTA or over a cluster, X staged at once or piece by piece, rows on 16 bytes or off them, one or two
token tiles, several passes over the tokens, pairs listed by pair or by expert. The cut is chosen by an estimate, so the sizes are looked for:
the smallest of a list that the estimate cuts the wanted way. Every output is compared with a 64-bit product of the decoded weights.

Tolerance: that of the products' other tests. FP32 sums, partly in tensor-core accumulators that may truncate (2^-23 per step), held to
sqrt(K) * 2^-22 * (sum of the magnitudes of all terms); a BF16 result is another 2^-8 of itself away at most."""
import itertools

import pytest
import torch

from paper_2609_39223_b200 import api

pytestmark = pytest.mark.gpu
BF, F32, F64 = torch.bfloat16, torch.float32, torch.float64
NV, MX, Q4 = api.FMT_NVFP4, api.FMT_MXFP4, api.FMT_Q4_K
FMTS = {"nvfp4": NV, "mxfp4": MX, "q4_k": Q4}
E2M1 = [0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6]
ROWS = [70, 131, 263, 579, 1157, 2507, 4803, 9663, 10331, 21207, 28547, 29403, 37907, 57433, 70203]
STEPS = [1, 2, 3, 4, 7, 8, 10, 13, 16, 17, 19, 21, 23, 24, 25, 26, 29, 33, 37, 42, 52, 57, 65, 91, 104, 127, 139, 166]      # of 256


def lengths(fmt, loose):
    """Contractions whose rows start on 16 bytes (multiples of 128), or a block more."""
    return [256 * s + loose * api.BLOCK[fmt] for s in STEPS if s * 256 < 45000]


def way(c):
    return ("cluster" if c.nz > 1 else "warps" if c.kw > 1 else "whole", "several" if c.blocks > c.grid_x else "one",
            "at once" if c.kc >= c.kz else "pieces")


def smallest(fmt, loose, tiles, wanted, Ms, Gs, most):
    """(M, G, N, K) of the smallest product of the lists that is cut the wanted way, or None."""
    sizes = sorted(itertools.product(ROWS, lengths(fmt, loose)), key=lambda s: s[0] * s[1])
    for (N, K), G, M in itertools.product(sizes, Gs, Ms):
        if N * K * max(G, 1) <= most:
            c = api.qf_selftest_matvec_cut(fmt, M, N, K, G)
            if c.token_tiles == tiles and c.loose == loose and way(c) == wanted:
                return M, G, N, K
    return None


def draw(fmt, lead, N, K, rare, g):
    """Random codes and scales on the GPU. rare: some rows of MXFP4 with scales outside the FP16 window."""
    make = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.uint8)
    codes = make(0, 256, *lead, N, K // 2)
    if fmt == Q4:
        scales = make(0, 256, *lead, N, K // 256, 16)
        d = (torch.rand((*lead, N, K // 256, 2), generator=g, device="cuda") + 0.5) * 2.0 ** -10
        scales[..., :4] = d.half().view(torch.uint8)
        return codes, scales, None
    if fmt == MX:
        scales = make(117, 125, *lead, N, K // 32)
        if rare:
            scales[..., ::29, :] = make(60, 190, *lead, (N + 28) // 29, K // 32)
        return codes, scales, None
    return codes, make(88, 127, *lead, N, K // 16), (torch.rand(lead or (1,), generator=g, device="cuda") + 0.5) * 1e-4


def decode(fmt, codes, scales, ts):
    """Values and magnitudes (of what they are the difference of) [rows, K] in 64 bits."""
    rows, K = codes.shape[0], codes.shape[1] * 2
    if fmt == Q4:
        f = scales[..., :4].contiguous().view(torch.float16).to(F64)
        a, b, c = scales[..., 4:8].int(), scales[..., 8:12].int(), scales[..., 12:].int()
        s6 = torch.cat([a & 63, (c & 15) | (a >> 6) << 4], -1).to(F64)
        m6 = torch.cat([b & 63, c >> 4 | (b >> 6) << 4], -1).to(F64)
        q = codes.view(rows, K // 256, 4, 1, 32)
        q = torch.cat([q & 15, q >> 4], 3).view(rows, K // 256, 8, 32).to(F64)
        up, off = (f[..., :1] * s6)[..., None] * q, ((f[..., 1:] * m6)[..., None]).expand(-1, -1, -1, 32)
        return (up - off).reshape(rows, K), (up.abs() + off.abs()).reshape(rows, K)
    v = torch.tensor(E2M1, dtype=F64, device="cuda")[torch.stack([codes & 15, codes >> 4], -1).view(rows, K).int()]
    s = scales.to(F64)
    if fmt == MX:
        s = torch.exp2(s - 127)
    else:
        e, m = torch.floor(s / 8), s % 8
        s = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2(e - 7)) * ts.to(F64)
    w = v * s.repeat_interleave(api.BLOCK[fmt], 1)
    return w, w.abs()


def acts(M, K, rare, g):
    """N(0, 1) with outlier channels. rare: a first token with tiny values here and there, a last one with large values at its end:
    steps of the contraction that the FP16 route cannot take."""
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, torch.randperm(K, generator=g, device="cuda")[:8]] *= 30
    if rare:
        x[0, ::997] *= 2.0 ** -40
        x[-1, -100:] *= 2.0 ** 13
    return x.to(BF)


def check(got, x, weight, what, rows=8192):
    """got [M, N] against x . w^T, weight(i, j) being the decoded rows i to j and their magnitudes."""
    K, x = x.shape[1], x.to(F64)
    for i in range(0, got.shape[1], rows):
        w, size = weight(i, min(i + rows, got.shape[1]))
        want = x @ w.T
        bound = K ** 0.5 * 2.0 ** -22 * (x.abs() @ size.T) + (2.0 ** -8 * want.abs() if got.dtype == BF else 0)
        off = (got[:, i:i + rows].to(F64) - want).abs() - bound
        assert torch.isfinite(off).all() and (off <= 0).all(), f"{what}, rows from {i}: largest excess {off.max().item():.3e}"


WAYS = list(itertools.product(("whole", "warps", "cluster"), ("one", "several"), ("at once", "pieces")))
KINDS = [(f, loose) for f in FMTS for loose in (0, 1) if not (f == "q4_k" and loose)]


def plain_size(kind, loose, tiles, wanted):
    return smallest(FMTS[kind], loose, tiles, wanted, (8, 3) if tiles == 1 else (27, 11), (0,), 380 << 20)


def grouped_size(kind, loose, tiles, listed, wanted):
    Ms = (2, 5, 15, 38) if listed == "by pair" else (6, 19, 46, 150) if tiles == 1 else (21, 90, 1100)
    found = [smallest(FMTS[kind], loose, tiles, wanted, [M for M in Ms if (M <= G) == (listed == "by pair")], (G,), 220 << 20) for G in (2, 5, 16, 40)]
    return min((s for s in found if s), key=lambda s: s[1] * s[2] * s[3], default=None)


@pytest.mark.parametrize("kind,loose", KINDS)
@pytest.mark.parametrize("tiles", [1, 2])
def test_plain(kind, loose, tiles):
    fmt = FMTS[kind]
    for wanted in WAYS:
        size = plain_size(kind, loose, tiles, wanted)
        if size is None:                                   # the estimate cuts nothing that way
            continue
        M, _, N, K = size
        g = torch.Generator(device="cuda").manual_seed(N + K)
        for rare, dtype in ((False, F32), (True, F32), (True, BF)):
            codes, scales, ts = draw(fmt, (), N, K, rare, g)
            x = acts(M, K, rare, g)
            Y = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
            api.qf_fq_matvec(fmt, x, codes, scales, ts, Y=Y)
            check(Y, x, lambda i, j: decode(fmt, codes[i:j], scales[i:j], ts), (wanted, size))


@pytest.mark.parametrize("kind,loose", KINDS)
@pytest.mark.parametrize("tiles,listed", [(1, "by pair"), (1, "by expert"), (2, "by expert")])
def test_grouped(kind, loose, tiles, listed):
    fmt = FMTS[kind]
    for wanted in WAYS:
        size = grouped_size(kind, loose, tiles, listed, wanted)
        if size is None:
            continue
        M, G, N, K = size
        g = torch.Generator(device="cuda").manual_seed(N + K)
        ids = torch.randint(0, G, (M,), generator=g, device="cuda")
        if M > 2:
            ids[M // 2], ids[-2] = -1, G
        x_rows = M if M % 2 else M // 2
        for rare, dtype in ((False, F32), (True, BF)):
            codes, scales, ts = draw(fmt, (G,), N, K, rare, g)
            x = acts(x_rows, K, rare, g)
            Y = torch.full((M, N), float("nan"), dtype=dtype, device="cuda")
            api.qf_fq_grouped_matvec(fmt, x, ids, codes, scales, ts, Y=Y)
            rows = x.repeat_interleave(M // x_rows, 0)
            for e in range(G):
                at = torch.nonzero(ids == e)[:, 0]
                if at.numel():
                    check(Y[at], rows[at], lambda i, j: decode(fmt, codes[e, i:j], scales[e, i:j], None if ts is None else ts[e]), (wanted, size))
            assert (Y[(ids < 0) | (ids >= G)] == 0).all(), (wanted, size)
