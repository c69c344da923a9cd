"""Plain 64-bit statements of the 4-bit key/value cache calls, for the tests: no code of the library."""
import math

import torch

from paper_2609_39223_b200 import api

_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def values(fmt: int, codes: torch.Tensor, scales: torch.Tensor, tscale) -> torch.Tensor:
    """Codes [..., dim / 2] and block scales [..., dim / block] -> values [..., dim] in 64 bits, unrounded."""
    grid = torch.tensor(_E2M1 + [-v for v in _E2M1], dtype=torch.float64, device=codes.device)
    v = grid[torch.stack([codes & 15, codes >> 4], -1).long()].flatten(-2)
    if fmt == api.FMT_MXFP4:
        s = torch.exp2(scales.double() - 127.0)
    else:
        s = (scales & 127).view(torch.float8_e4m3fn).double() * float(tscale)
    return v * s.repeat_interleave(api.BLOCK[fmt], -1)


def gathered(cache: "api.KvCache", table_row: torch.Tensor, n: int):
    """Keys and values [kv_heads, n, dim] in 64 bits of the first n places that a page table row lists."""
    pages = table_row[: -(-n // cache.page_size)].long()
    out = []
    for codes, scales, ts in ((cache.k_codes, cache.k_scales, cache.k_tscale), (cache.v_codes, cache.v_scales, cache.v_tscale)):
        v = values(cache.fmt, codes[pages], scales[pages], ts)
        out.append(v.transpose(0, 1).flatten(1, 2)[:, :n])
    return out


def attention(cache, q: torch.Tensor, table: torch.Tensor, lens, scale: float):
    """out, lse in 64 bits and, for the tolerance, sum of p |v| and the largest scale * sum over d of |q_d k_jd| of every row."""
    batch, q_len, q_heads, dim = q.shape
    group = q_heads // cache.kv_heads
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    mass = torch.zeros_like(out)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device=q.device)
    big = torch.zeros(q.shape[:3], dtype=torch.float64, device=q.device)
    for b in range(batch):
        n = min(max(int(lens[b]), 0), table.shape[1] * cache.page_size)
        if n == 0:
            continue
        k, v = gathered(cache, table[b], n)
        for i in range(q_len):
            m = n - q_len + i + 1
            if m <= 0:
                continue
            qi = q[b, i].double().view(cache.kv_heads, group, dim)
            s = torch.einsum("hgd,hjd->hgj", qi, k[:, :m]) * scale
            p = torch.softmax(s, -1)
            out[b, i] = torch.einsum("hgj,hjd->hgd", p, v[:, :m]).reshape(q_heads, dim)
            mass[b, i] = torch.einsum("hgj,hjd->hgd", p, v[:, :m].abs()).reshape(q_heads, dim)
            lse[b, i] = torch.logsumexp(s, -1).reshape(-1)
            big[b, i] = (torch.einsum("hgd,hjd->hgj", qi.abs(), k[:, :m].abs()).amax(-1) * abs(scale)).reshape(-1)
    return out, lse, mass, big


def check_attention(cache, q, table, lens, scale, out, lse=None):
    """Largest errors that the arithmetic allows. A score is a sum of dim exact products whose partial sums (at most `big`) may each be
    truncated to FP32: off by dim * 2^-23 * big, and by 2^-22 of itself for the scale and the exponential's argument; the weight is off
    by that, by 2^-21 for exponentials and their sums, and by 2^-11 for its FP16 form (2^-30 of the largest weight where that is
    subnormal, which keys * 2^-30 of the largest value covers); one rounding to BF16, 2^-8."""
    ref, rlse, mass, big = attention(cache, q, table, lens, scale)
    keys = int(max(int(x) for x in lens)) if len(lens) else 0
    top = float(mass.max()) if mass.numel() else 0.0
    score = (q.shape[-1] + 4) * 2.0 ** -23 * big
    tol = ref.abs() * 2.0 ** -8 + mass * (2 * score[..., None] + 2.0 ** -20 + 2.0 ** -11) + keys * 2.0 ** -30 * top
    assert torch.isfinite(out.double()).all()
    worst = ((out.double() - ref).abs() - tol).max()
    assert float(worst) <= 0.0, f"outputs are {float(worst)} over the tolerance"
    empty = torch.isinf(rlse)
    assert (out[empty.unsqueeze(-1).expand_as(out)] == 0).all()
    if lse is not None:
        assert torch.equal(torch.isinf(lse), empty) and (lse[empty] < 0).all()
        off = (lse.double() - rlse).abs() - (score + 2.0 ** -20 + rlse.abs() * 2.0 ** -22)
        assert float(off[~empty].max() if (~empty).any() else 0.0) <= 0.0
