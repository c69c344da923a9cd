"""The 4-bit key/value cache as measured workloads: writing keys and values into it as they are quantized, reading them back, and
attention of a few tokens over it. The cases, their inputs, a plain form in elementary FP32 torch operations, and the calls a user
makes of the library.

The cache is paged: codes [pages, heads, page_size, dim / 2] with block scales [pages, heads, page_size, dim / block] for the keys and
for the values. A slot is page * page_size + place in the page; a page table lists the pages of every sequence in order. Formats:
NVFP4 (E2M1, 16-element blocks with an E4M3 scale, one FP32 tensor scale for the keys and one for the values) and MXFP4 (E2M1,
32-element blocks with a power-of-two scale)."""
import math

import torch

own = False

BLOCK = {"nvfp4": 16, "mxfp4": 32}
SCALE_BYTES = {"nvfp4": 1.0 / 16, "mxfp4": 1.0 / 32}             # per element
DT = {"i32": torch.int32, "i64": torch.int64}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]
K_SCALE, V_SCALE = 30.0 / (6.0 * 448.0), 6.0 / (6.0 * 448.0)     # NVFP4 tensor scales from a calibration's largest key and value


# ---- cases -------------------------------------------------------------------------------------------------------------------

def listed():
    wide = dict(heads=8, dim=128)
    dense = dict(q_heads=32, heads=8, dim=128)
    return [
        # a decode batch's new keys and values, slices of the fused projection's output, written and read back: the smallest write
        dict(name="write nvfp4 t33", op="write", fmt="nvfp4", tokens=33, page=64, slots="i64", fused=True, dropped=0.0, **wide),
        # a padded batch of narrow heads, whose padding goes nowhere
        dict(name="write nvfp4 t1003 d64", op="write", fmt="nvfp4", tokens=1003, page=48, slots="i32", fused=False, dropped=0.1, heads=4, dim=64),
        # the prompt of a long sequence, or of many: the largest write
        dict(name="write mxfp4 t16384", op="write", fmt="mxfp4", tokens=16384, page=64, slots="i64", fused=True, dropped=0.0, **wide),
        # one short sequence for a prefill that goes on behind it
        dict(name="read mxfp4 1x777 d64", op="read", fmt="mxfp4", batch=1, length=777, page=16, slots="i32", heads=8, dim=64),
        # the contexts of a batch, of any length up to the largest
        dict(name="read nvfp4 16x8192", op="read", fmt="nvfp4", batch=16, length=8192, page=64, slots="i64", **wide),
        # one sequence's decode step at a short context: the smallest attention
        dict(name="attend mxfp4 1x1000", op="attend", fmt="mxfp4", batch=1, q_len=1, length=1000, ragged=False, page=64, lse=False, **dense),
        # one sequence at a long context, where the keys are split over the whole GPU
        dict(name="attend nvfp4 1x131072", op="attend", fmt="nvfp4", batch=1, q_len=1, length=131072, ragged=False, page=64, lse=False, **dense),
        # a rollout batch of every length, small pages, with an empty place in it
        dict(name="attend nvfp4 64x8192", op="attend", fmt="nvfp4", batch=64, q_len=1, length=8192, ragged=True, page=16, lse=False, **dense),
        # drafted tokens checked together, five a sequence
        dict(name="attend mxfp4 16x4096 q5", op="attend", fmt="mxfp4", batch=16, q_len=5, length=4096, ragged=True, page=64, lse=False, **dense),
        # a key head for every query head, narrow heads
        dict(name="attend nvfp4 20x4096 d64", op="attend", fmt="nvfp4", batch=20, q_len=1, length=4096, ragged=True, page=32, lse=False,
             q_heads=32, heads=32, dim=64),
        # wide heads, with the sums' logarithms for joining with other keys
        dict(name="attend mxfp4 7x2500 d256", op="attend", fmt="mxfp4", batch=7, q_len=1, length=2500, ragged=True, page=48, lse=True,
             q_heads=16, heads=2, dim=256),
        # a full rollout batch of equal lengths: the largest
        dict(name="attend mxfp4 128x8192", op="attend", fmt="mxfp4", batch=128, q_len=1, length=8192, ragged=False, page=64, lse=False,
             q_heads=64, heads=8, dim=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "read", "attend", "attend", "attend"])
    fmt = rng.choice(["nvfp4", "mxfp4"])
    dim = rng.choice([64, 128, 128, 256])
    page = rng.choice([16, 32, 48, 64, 128])
    slots = rng.choice(["i32", "i64"])
    if op == "write":
        heads = _log(rng, 1, 16)
        return dict(op=op, fmt=fmt, tokens=_log(rng, 1, 16384 * 1024 // max(1024, heads * dim)), page=page, slots=slots, fused=rng.random() < 0.5,
                    dropped=rng.choice([0.0, 0.0, 0.1]), heads=heads, dim=dim)
    heads = _log(rng, 1, 32)
    if op == "read":
        batch = _log(rng, 1, 32)
        return dict(op=op, fmt=fmt, batch=batch, length=_log(rng, 1, max(2, 64 * 1024 * 1024 // (batch * max(1024, heads * dim)))), page=page, slots=slots,
                    heads=heads, dim=dim)
    batch, q_len, group = _log(rng, 1, 128), rng.choice([1, 1, 1, 2, 3, 5, 8]), rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 16])
    most = 1024 * 1024 * 1024 // (batch * heads * dim * max(1, q_len * group // 8))
    return dict(op=op, fmt=fmt, batch=batch, q_len=q_len, length=_log(rng, q_len, max(q_len + 1, min(131072, most))), ragged=rng.random() < 0.7, page=page,
                lse=rng.random() < 0.3, q_heads=heads * group, heads=heads, dim=dim)


def _spread(case):
    """Keys of a batch's sequences, the new tokens' own among them: even steps up to the full length in a ragged batch, with, from four
    sequences on, an empty place in a batch that attends."""
    batch, low, high = case["batch"], case.get("q_len", 1), case["length"]
    if not case.get("ragged", True):
        return [high] * batch
    lens = [low + (high - low) * (i + 1) // batch for i in range(batch)]
    if batch >= 4 and case["op"] == "attend":
        lens[0] = 0
    return lens


def _mean_length(case):
    return sum(_spread(case)) / case["batch"]


def work(case):
    element = 0.5 + SCALE_BYTES[case["fmt"]]
    row = 2 * case["heads"] * case["dim"]                          # a token's keys and values
    if case["op"] == "write":                                      # read in BF16, written in 4 bits; read from 4 bits, written in BF16
        kept = case["tokens"] * (1.0 - case["dropped"])
        return {"bytes": row * (kept * (2.0 + 2 * element) + case["tokens"] * 2.0), "flops": 0.0}
    if case["op"] == "read":
        return {"bytes": case["batch"] * _mean_length(case) * row * (2.0 + element), "flops": 0.0}
    # the cache once; a new token's scores and sums take four operations per key, query head and dimension
    pairs = case["batch"] * case["q_len"] * max(1.0, _mean_length(case) - (case["q_len"] - 1) / 2.0)
    io = case["batch"] * case["q_len"] * case["q_heads"] * (4 * case["dim"] + (4 if case["lse"] else 0))
    return {"bytes": case["batch"] * _mean_length(case) * row * element + io, "flops": 4.0 * pairs * case["q_heads"] * case["dim"]}


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _keys(g, *shape):
    """N(0, 1), four of the dimensions five times as large."""
    k = torch.randn(shape, generator=g, device="cuda")
    k[..., torch.randperm(shape[-1], generator=g, device="cuda")[:4]] *= 5.0
    return k


def _lengths(g, case):
    lens = torch.tensor(_spread(case), dtype=torch.int32, device="cuda")
    return lens[torch.randperm(case["batch"], generator=g, device="cuda")]


def _page_table(g, lens, length, page):
    """Every sequence's pages in any order, and how many pages the cache has; unused entries are page 0."""
    need = (lens + (page - 1)) // page
    most = max(1, -(-length // page))
    pages = int(need.sum()) + 3
    order = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int32)
    at = torch.arange(most, device="cuda")[None, :]
    first = torch.cumsum(need, 0) - need
    table = order[(first[:, None] + at).clamp(max=pages - 1)]
    return torch.where(at < need[:, None], table, 0).to(torch.int32).contiguous(), pages


def _slots_of(table, lens, page):
    """The slots of all sequences' keys, one sequence behind the other."""
    at = torch.arange(table.shape[1] * page, device="cuda")
    slot = table.long().repeat_interleave(page, 1) * page + at % page
    return slot[at[None, :] < lens[:, None]]


def prepare(case, seed):
    g = _generator(seed)
    op, fmt, heads, dim, page = case["op"], case["fmt"], case["heads"], case["dim"], case["page"]
    s = {"case": case, "k_tscale": None, "v_tscale": None}
    if fmt == "nvfp4":
        s["k_tscale"] = torch.full((1,), K_SCALE, device="cuda")
        s["v_tscale"] = torch.full((1,), V_SCALE, device="cuda")
    if op == "write":
        T = case["tokens"]
        pages = -(-T // page) + 4
        slots = torch.randperm(pages * page, generator=g, device="cuda")[:T] if T < 256 else torch.arange(T, device="cuda") + page
        drop = torch.rand((T,), generator=g, device="cuda") < case["dropped"]
        s["slots"] = torch.where(drop, -1, slots).to(DT[case["slots"]])
        for name in ("k", "v"):
            values = torch.zeros((pages, heads, page, dim), device="cuda")
            s[name + "_codes"], s[name + "_scales"] = _quantized(fmt, values, s[name + "_tscale"])
        k = _keys(g, T, heads, dim).to(torch.bfloat16)
        v = torch.randn((T, heads, dim), generator=g, device="cuda").to(torch.bfloat16)
        if case["fused"]:                                          # queries of four times as many heads come first in the projection
            both = torch.cat([torch.zeros((T, 4 * heads, dim), dtype=torch.bfloat16, device="cuda"), k, v], 1)
            k, v = both[:, 4 * heads:5 * heads], both[:, 5 * heads:]
        s["k"], s["v"] = k, v
        return s
    lens = _lengths(g, case)
    table, pages = _page_table(g, lens, case["length"], page)
    s["k_codes"], s["k_scales"] = _quantized(fmt, _keys(g, pages, heads, page, dim), s["k_tscale"])
    s["v_codes"], s["v_scales"] = _quantized(fmt, torch.randn((pages, heads, page, dim), generator=g, device="cuda"), s["v_tscale"])
    if op == "read":
        s["slots"] = _slots_of(table, lens, page).to(DT[case["slots"]])
        return s
    s["q"] = torch.randn((case["batch"], case["q_len"], case["q_heads"], dim), generator=g, device="cuda").to(torch.bfloat16)
    s["table"], s["lens"] = table, lens
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------------

def _power(p):
    """2^p for whole numbers p, at least 2^-126 (a smaller one only comes with a block of zeros)."""
    return ((p.int().clamp(-126, 127) + 127) << 23).view(torch.float32)


def _quantized(fmt, x, tscale):
    """Packed codes and block scales of the rows of x (FP32): each block's scale from its largest value, every element to the nearest
    value of the format, ties to the even code."""
    b = x.view(*x.shape[:-1], x.shape[-1] // BLOCK[fmt], BLOCK[fmt])
    top = b.abs().amax(-1)
    if fmt == "mxfp4":
        p = (torch.frexp(top).exponent - 3).clamp(min=-127)
        p = torch.where(top == 0, -127, p)
        scales = (p + 127).to(torch.uint8)
        v = b * _power(-p)[..., None]
    else:
        sb = (top / (6.0 * tscale)).clamp(max=448.0).to(torch.float8_e4m3fn)
        scales = sb.view(torch.uint8)
        step = (tscale * sb.float())[..., None]
        v = torch.where(step > 0, b / step, 0.0)
    a = v.abs()
    code = (a > 0.25).to(torch.uint8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    code = (code | (torch.signbit(v).to(torch.uint8) << 3)).view(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), scales


def _values(fmt, codes, scales, tscale):
    """FP32 values of packed codes [..., dim / 2]: (block scale * code) * tensor scale."""
    q = torch.stack([codes & 15, codes >> 4], -1).view(*scales.shape, BLOCK[fmt])
    v = torch.tensor(E2M1, device=codes.device)[q.int()]
    if fmt == "mxfp4":
        v = v * _power(scales.int() - 127)[..., None]
    else:
        v = v * scales.view(torch.float8_e4m3fn).float()[..., None] * tscale
    return v.view(*codes.shape[:-1], codes.shape[-1] * 2)


def _plain_read(s, name):
    """The BF16 rows of s["slots"]; zeros where a slot is outside the cache."""
    page, slots = s["case"]["page"], s["slots"].long()
    codes, scales = s[name + "_codes"], s[name + "_scales"]
    live = (slots >= 0) & (slots < codes.shape[0] * page)
    at = torch.where(live, slots, 0)
    rows = _values(s["case"]["fmt"], codes[at // page, :, at % page], scales[at // page, :, at % page], s[name + "_tscale"])
    return torch.where(live[:, None, None], rows, 0.0).to(torch.bfloat16)


def _plain_write(s, name):
    page, slots = s["case"]["page"], s["slots"].long()
    codes, scales = _quantized(s["case"]["fmt"], s[name].float(), s[name + "_tscale"])
    live = torch.nonzero((slots >= 0) & (slots < s[name + "_codes"].shape[0] * page))[:, 0]
    at = slots[live]
    s[name + "_codes"][at // page, :, at % page] = codes[live]
    s[name + "_scales"][at // page, :, at % page] = scales[live]


def _gathered(s, name):
    """FP32 values [batch, heads, most keys, dim] of all sequences' pages."""
    case = s["case"]
    table = s["table"].long()
    v = _values(case["fmt"], s[name + "_codes"][table].transpose(1, 2), s[name + "_scales"][table].transpose(1, 2), s[name + "_tscale"])
    return v.reshape(case["batch"], case["heads"], -1, case["dim"])


def _plain_attend(s):
    case = s["case"]
    batch, q_len, q_heads, heads, dim = case["batch"], case["q_len"], case["q_heads"], case["heads"], case["dim"]
    group = q_heads // heads
    q = s["q"].float().view(batch, q_len, heads, group, dim).permute(0, 2, 1, 3, 4).reshape(batch, heads, q_len * group, dim)
    score = torch.matmul(q, _gathered(s, "k").transpose(2, 3)) * (1.0 / math.sqrt(dim))
    score = score.view(batch, heads, q_len, group, -1)
    # new token i of a sequence sees the keys up to its own, the (length - q_len + i)-th
    last = s["lens"][:, None] - q_len + torch.arange(q_len, device=q.device)
    seen = torch.arange(score.shape[-1], device=q.device) <= last[..., None]
    score = torch.where(seen[:, None, :, None, :], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    some = top > -math.inf
    top = torch.where(some, top, 0.0)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    p = torch.where(some, p / total, 0.0).view(batch, heads, q_len * group, -1)
    out = torch.matmul(p, _gathered(s, "v")).view(batch, heads, q_len, group, dim)
    out = out.permute(0, 2, 1, 3, 4).reshape(batch, q_len, q_heads, dim).to(torch.bfloat16)
    lse = torch.where(some, top + torch.log(total), -math.inf)[..., 0]
    return (out, lse.permute(0, 2, 1, 3).reshape(batch, q_len, q_heads)) if case["lse"] else (out,)


def _plain(s):
    op = s["case"]["op"]
    if op == "attend":
        return _plain_attend(s)
    if op == "write":
        _plain_write(s, "k")
        _plain_write(s, "v")
    return _plain_read(s, "k"), _plain_read(s, "v")


# ---- the library's calls -----------------------------------------------------------------------------------------------------

def _library(s):
    from paper_2609_39223_b200 import api
    case = s["case"]
    if "cache" not in s:                                           # the handle and the workspace that a serving loop keeps
        s["cache"] = api.KvCache(api.FORMATS[case["fmt"]], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["k_tscale"], s["v_tscale"])
        if case["op"] == "attend":
            s["ws"] = api.workspace(api.OP_KV_ATTENTION, case["batch"] * case["q_len"], case["q_heads"], case["dim"], case["heads"])
    cache = s["cache"]
    if case["op"] == "attend":
        if case["lse"]:
            return api.qf_kv_attention(cache, s["q"], s["table"], s["lens"], want_lse=True, ws=s["ws"])
        return (api.qf_kv_attention(cache, s["q"], s["table"], s["lens"], ws=s["ws"]),)
    if case["op"] == "write":
        api.qf_kv_append(cache, s["k"], s["v"], s["slots"])
    return api.qf_kv_read(cache, s["slots"])


def run(state):
    return _library(state) if own else _plain(state)


# ---- 64 bits -----------------------------------------------------------------------------------------------------------------

def _e2m1_64(n):
    """Values of 4-bit codes (whole numbers in 64 bits)."""
    e, m = torch.floor(torch.remainder(n, 8.0) / 2.0), torch.remainder(n, 2.0)
    return (1.0 - 2.0 * torch.floor(n / 8.0)) * torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.exp2(e - 1.0))


def _e4m3_64(n):
    e, m = torch.floor(n / 8.0), torch.remainder(n, 8.0)           # four exponent bits with bias 7, three of fraction
    return torch.where(e == 0, m * 2.0 ** -9, (1.0 + m / 8.0) * torch.exp2(e - 7.0))


def _exact_rows(fmt, codes, scales, tscale):
    """Values of rows of codes in 64 bits."""
    v = torch.empty((*codes.shape[:-1], 2 * codes.shape[-1]), dtype=torch.float64, device=codes.device)
    v[..., 0::2], v[..., 1::2] = _e2m1_64((codes % 16).double()), _e2m1_64((codes // 16).double())
    step = torch.exp2(scales.double() - 127.0) if fmt == "mxfp4" else _e4m3_64(scales.double()) * tscale.double()
    return v * step.repeat_interleave(BLOCK[fmt], -1)


def _nearest(x, grid):
    """The value of an ascending grid that lies nearest, of two the one with the even place."""
    up = torch.searchsorted(grid, x).clamp(max=len(grid) - 1)
    down = (up - 1).clamp(min=0)
    a, b = x - grid[down], grid[up] - x
    return grid[torch.where((a < b) | ((a == b) & (down % 2 == 0)), down, up)]


def _exact_written(fmt, x, tscale):
    """What a row of BF16 values reads as after quantization. The format defines its quotients as FP32 numbers; a quotient of two FP32
    numbers in 64 bits rounded to 32 is that number."""
    b = x.double().view(*x.shape[:-1], -1, BLOCK[fmt])
    top = b.abs().amax(-1)
    grid = _e2m1_64(torch.arange(8, dtype=torch.float64, device=x.device))
    if fmt == "mxfp4":
        step = torch.exp2((torch.frexp(top).exponent - 3).double().clamp(min=-127.0))
        v = b / step[..., None]
    else:
        t = tscale.double()
        q = (top / (6.0 * t).float().double()).float().double()
        sb = _nearest(q, _e4m3_64(torch.arange(127, dtype=torch.float64, device=x.device)))
        step = sb * t
        v = torch.where(step[..., None] > 0, (b / step.float().double()[..., None]).float().double(), 0.0)
    return (torch.sign(v) * _nearest(v.abs().contiguous(), grid) * step[..., None]).view(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    fmt, page, heads, dim = case["fmt"], case["page"], case["heads"], case["dim"]
    if case["op"] == "write":
        kept = (s["slots"] >= 0)[:, None, None]
        return tuple(_exact_written(fmt, s[n], s[n + "_tscale"]) * kept for n in ("k", "v"))
    if case["op"] == "read":
        at = s["slots"].long()
        return tuple(_exact_rows(fmt, s[n + "_codes"][at // page, :, at % page], s[n + "_scales"][at // page, :, at % page], s[n + "_tscale"])
                     for n in ("k", "v"))
    batch, q_len, q_heads = case["batch"], case["q_len"], case["q_heads"]
    out = torch.zeros((batch, q_len, q_heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((batch, q_len, q_heads), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):                     # a sequence at a time, each new token with the keys it sees
        if n == 0:
            continue
        pages = s["table"][b, :-(-n // page)].long()
        k, v = (_exact_rows(fmt, s[x + "_codes"][pages], s[x + "_scales"][pages], s[x + "_tscale"]).transpose(0, 1).reshape(heads, -1, dim)
                for x in ("k", "v"))
        for i in range(q_len):
            m = n - q_len + i + 1
            q = s["q"][b, i].double().view(heads, -1, dim)
            a = q @ k[:, :m].transpose(1, 2) / math.sqrt(dim)
            lse[b, i] = torch.logsumexp(a, -1).reshape(-1)
            out[b, i] = (torch.softmax(a, -1) @ v[:, :m]).reshape(q_heads, dim)
    return (out, lse) if case["lse"] else (out,)
