"""The mixture-of-experts routing operators and the 4-bit matrix-vector products as measured workloads: the cases, their inputs,
a plain form in elementary FP32 torch operations, and the calls a user makes of the library.

Weights are quantized here, from N(0, 0.02) values, by the formats' formulas: NVFP4 (E2M1 codes, 16-element blocks with an E4M3
scale, FP32 tensor scale), MXFP4 (E2M1, 32-element blocks with a power-of-two scale) and Q4_K (unsigned codes, 256-weight
super-blocks of 8 sub-blocks with 6-bit scales and offsets under FP16 factors)."""
import math

import torch

own = False

ALIGN = 128                                   # rows of an expert's segment are padded to a multiple of this
VOCAB = 128256
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "i32": torch.int32, "i64": torch.int64}
SIZE = {"bf16": 2, "f32": 4, "i32": 4, "i64": 8}
BLOCK = {"nvfp4": 16, "mxfp4": 32, "q4_k": 256}
SCALE_BYTES = {"nvfp4": 1.0 / 16, "mxfp4": 1.0 / 32, "q4_k": 1.0 / 16}      # per weight
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]
MIDDLE = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]


# ---- cases -------------------------------------------------------------------------------------------------------------------

def listed():
    moe = dict(experts=128, top_k=8)
    return [
        # the key projection of a dense decoder (8 heads of 128 from a hidden size of 4096) for one token: the shortest product
        dict(name="matvec nvfp4 1024x4096 m1", op="matvec", fmt="nvfp4", M=1, N=1024, K=4096, y="bf16"),
        # the MLP's up projection for one token, the ordinary decode step
        dict(name="matvec q4_k 14336x4096 m1", op="matvec", fmt="q4_k", M=1, N=14336, K=4096, y="bf16"),
        # the MLP's down projection for an odd small batch, FP32 result (an input of a residual sum)
        dict(name="matvec nvfp4 4096x14336 m5", op="matvec", fmt="nvfp4", M=5, N=4096, K=14336, y="f32"),
        # logits over the whole vocabulary for sixteen sequences: the longest product
        dict(name="matvec mxfp4 128256x4096 m16", op="matvec", fmt="mxfp4", M=16, N=VOCAB, K=4096, y="f32"),
        # one token's gate and up projections in its eight experts
        dict(name="experts mxfp4 1536x2048 t1", op="experts", fmt="mxfp4", tokens=1, N=1536, K=2048, y="bf16", shared_x=True, **moe),
        # the experts' down projections for a decode batch of 24 sequences, each pair with an input of its own
        dict(name="experts nvfp4 2048x768 t24", op="experts", fmt="nvfp4", tokens=24, N=2048, K=768, y="bf16", shared_x=False, **moe),
        # routing table of a small rollout batch
        dict(name="sort t7", op="sort", tokens=7, ids="i64", dropped=0.0, room=1.0, **moe),
        # routing table of a training batch of 16384 tokens
        dict(name="sort t16384", op="sort", tokens=16384, ids="i32", dropped=0.0, room=1.0, **moe),
        # the training batch's rows into expert order
        dict(name="dispatch t16384", op="dispatch", tokens=16384, hidden=2048, dropped=0.0, **moe),
        # its gradient for an odd number of tokens, a few of them dropped, from an FP32 dX
        dict(name="dispatch gradient t5003", op="dispatch_bwd", tokens=5003, hidden=2048, dx="f32", out="bf16", dropped=0.01, **moe),
        # the experts' outputs of a decode batch, weighted and added
        dict(name="combine t33", op="combine", tokens=33, hidden=2048, ys="bf16", out="bf16", dropped=0.0, **moe),
        # gradient of the weighted sum for the training batch: rows and router weights
        dict(name="combine gradient t16384", op="combine_bwd", tokens=16384, hidden=2048, ys="bf16", dout="bf16", dropped=0.0, **moe),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _sized(rng, unit, lo, hi):
    return max(1, _log(rng, lo, hi) // unit) * unit


def draw(rng):
    op = rng.choice(["matvec", "matvec", "experts", "experts", "sort", "dispatch", "dispatch_bwd", "combine", "combine_bwd"])
    if op in ("matvec", "experts"):
        fmt = rng.choice(["nvfp4", "mxfp4", "q4_k"])
        y = rng.choice(["bf16", "f32"])
        if op == "matvec":
            K = _sized(rng, BLOCK[fmt], 256, 14336)
            return dict(op=op, fmt=fmt, M=_log(rng, 1, 16), N=_log(rng, 64, min(VOCAB, VOCAB * 4096 // K)), K=K, y=y)
        K = _sized(rng, BLOCK[fmt], 256, 4096)
        G = _log(rng, 4, 128)
        k = rng.randint(1, min(8, G))
        tokens = _log(rng, 1, 32)
        return dict(op=op, fmt=fmt, tokens=tokens, N=_log(rng, 64, min(4096, VOCAB * 1024 // (K * max(G, tokens * k)) + 65)), K=K, y=y,
                    shared_x=rng.random() < 0.5, experts=G, top_k=k, dropped=rng.choice([0.0, 0.0, 0.1]))
    G = _log(rng, 4, 256)
    k = rng.randint(1, min(8, G))
    case = dict(op=op, experts=G, top_k=k, tokens=_log(rng, 1, 16384), dropped=rng.choice([0.0, 0.0, 0.03, 0.5]))
    if op == "sort":
        return dict(case, ids=rng.choice(["i32", "i64"]), room=rng.choice([1.0, 1.0, 0.7]))
    case["hidden"] = _sized(rng, 8, 64, 2048)
    if op == "dispatch_bwd":
        case.update(dx=rng.choice(["bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
    if op == "combine":
        case.update(ys=rng.choice(["bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
    if op == "combine_bwd":
        case.update(ys="bf16", dout=rng.choice(["bf16", "f32"]))
    return case


def _room(case):
    """Rows of a sorted buffer that is large enough whatever the routing, so that its size is known without waiting for the
    GPU: a multiple of 128."""
    pairs = case["tokens"] * case["top_k"]
    return (pairs + (ALIGN - 1) * min(case["experts"], pairs)) // ALIGN * ALIGN


def _distinct(case):
    """Expected number of distinct experts that a batch meets under even routing."""
    G = case["experts"]
    return G * (1.0 - (1.0 - case["top_k"] / G) ** case["tokens"])


def work(case):
    op = case["op"]
    if op == "matvec":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * K * (0.5 + SCALE_BYTES[case["fmt"]]) + M * K * 2 + M * N * SIZE[case["y"]], "flops": 2.0 * M * N * K}
    if op == "experts":
        N, K, pairs = case["N"], case["K"], case["tokens"] * case["top_k"]
        rows_x = case["tokens"] if case["shared_x"] else pairs
        return {"bytes": _distinct(case) * N * K * (0.5 + SCALE_BYTES[case["fmt"]]) + rows_x * K * 2 + pairs * (N * SIZE[case["y"]] + 4),
                "flops": 2.0 * pairs * N * K}
    T, k, G = case["tokens"], case["top_k"], case["experts"]
    live = T * k * (1.0 - case["dropped"])
    if op == "sort":
        return {"bytes": T * k * (SIZE[case["ids"]] + 4.0) + (2 * G + 1) * 4, "flops": 0.0}
    H = case["hidden"]
    if op == "dispatch":
        return {"bytes": T * H * 2 + _room(case) * H * 2 + T * k * 4, "flops": 0.0}
    if op == "dispatch_bwd":
        return {"bytes": live * H * SIZE[case["dx"]] + T * H * SIZE[case["out"]] + T * k * 4, "flops": live * H}
    if op == "combine":
        return {"bytes": live * H * SIZE[case["ys"]] + T * H * SIZE[case["out"]] + T * k * 8, "flops": 2.0 * live * H}
    return {"bytes": T * H * SIZE[case["dout"]] + live * H * SIZE[case["ys"]] + _room(case) * H * 2 + T * k * 12, "flops": 3.0 * live * H}


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _activations(g, rows, cols):
    """N(0, 1) with eight outlier channels thirty times as large."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    at = torch.randperm(cols, generator=g, device="cuda")[:8]
    x[:, at] *= 30.0
    return x.to(torch.bfloat16)


def _pack_pairs(codes):
    """Element 2j in the low nibble of byte j, element 2j + 1 in the high one."""
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _e2m1_codes(v):
    return torch.bucketize(v.abs(), torch.tensor(MIDDLE, device=v.device), out_int32=True).to(torch.uint8) | ((v < 0).to(torch.uint8) << 3)


def _quantized(g, fmt, rows, cols):
    """Codes, scales and (NVFP4) tensor scale of a random weight [rows, cols]."""
    w = torch.randn((rows, cols), generator=g, device="cuda") * 0.02
    if fmt == "q4_k":
        b = w.view(rows, cols // 256, 8, 32)
        off = -b.amin(-1).clamp(max=0.0)
        sc = (b.amax(-1) + off) / 15.0
        d, dmin = (sc.amax(-1) / 63.0).half(), (off.amax(-1) / 63.0).half()
        s6 = (sc / d.float()[..., None]).round().clamp(0, 63)
        m6 = (off / dmin.float()[..., None]).round().clamp(0, 63)
        es, em = d.float()[..., None] * s6, dmin.float()[..., None] * m6
        q = ((b + em[..., None]) / es[..., None]).round().clamp(0, 15).to(torch.uint8).view(rows, cols // 256, 4, 2, 32)
        codes = (q[..., 0, :] | (q[..., 1, :] << 4)).reshape(rows, cols // 2)
        s, m = s6.to(torch.uint8), m6.to(torch.uint8)
        low = s[..., :4] | ((s[..., 4:] >> 4) << 6)
        mid = m[..., :4] | ((m[..., 4:] >> 4) << 6)
        high = (s[..., 4:] & 15) | ((m[..., 4:] & 15) << 4)
        head = torch.stack([d, dmin], -1).view(torch.uint8).view(rows, cols // 256, 4)
        return codes, torch.cat([head, low, mid, high], -1).contiguous(), None
    b = w.view(rows, cols // BLOCK[fmt], BLOCK[fmt])
    top = b.abs().amax(-1)
    if fmt == "mxfp4":
        p = torch.floor(torch.log2(top)) - 2
        codes = _e2m1_codes(b / torch.exp2(p)[..., None])
        return _pack_pairs(codes.view(rows, cols)), (p + 127).to(torch.uint8), None
    ts = (w.abs().max() / (6.0 * 448.0)).reshape(1)
    sb = (top / (6.0 * ts)).clamp(max=448.0).to(torch.float8_e4m3fn)
    codes = _e2m1_codes(b / (ts * sb.float())[..., None].clamp(min=1e-30))
    return _pack_pairs(codes.view(rows, cols)), sb.view(torch.uint8), ts


def _routing(g, case, dtype=torch.int32):
    """Top-k of N(0, 1) router logits; a share of the pairs dropped by the router (expert -1); their softmax weights."""
    logits = torch.randn((case["tokens"], case["experts"]), generator=g, device="cuda")
    top = torch.topk(torch.softmax(logits, -1), case["top_k"], dim=-1)
    drop = torch.rand((case["tokens"], case["top_k"]), generator=g, device="cuda") < case.get("dropped", 0.0)
    ids = torch.where(drop, -1, top.indices).to(dtype)
    return ids, top.values / top.values.sum(-1, keepdim=True)


def _table(ids, experts, rows):
    """The routing table of expert ids: real rows per expert, segment starts, the row of every pair."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < experts), flat, experts)
    counts = torch.zeros(experts + 1, dtype=torch.int64, device=ids.device).index_add_(0, key, torch.ones_like(key))
    padded = (counts + ALIGN - 1) // ALIGN * ALIGN
    starts = torch.cumsum(padded, 0) - padded
    first = torch.cumsum(counts, 0) - counts
    key, order = torch.sort(key, stable=True)
    row = starts[key] + torch.arange(key.numel(), device=ids.device) - first[key]
    row = torch.where((key < experts) & (row < rows), row, -1)
    row_of = torch.empty_like(row).index_copy_(0, order, row).view(ids.shape)
    real = torch.minimum(counts[:experts], (rows - starts[:experts]).clamp(min=0))
    return row_of.int(), starts.clamp(max=rows).int(), real.int()


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    s = {"case": case}
    if op == "matvec":
        s["x"] = _activations(g, case["M"], case["K"])
        s["codes"], s["scales"], s["ts"] = _quantized(g, case["fmt"], case["N"], case["K"])
        return s
    if op == "experts":
        G, N, K = case["experts"], case["N"], case["K"]
        s["ids"], _ = _routing(g, case)
        s["x"] = _activations(g, case["tokens"] * (1 if case["shared_x"] else case["top_k"]), K)
        codes, scales, ts = _quantized(g, case["fmt"], G * N, K)
        s["codes"], s["scales"] = codes.view(G, N, K // 2), scales.view(G, N, *scales.shape[1:])
        # every expert has a tensor scale of its own
        s["ts"] = None if ts is None else ts * (0.5 + torch.rand(G, generator=g, device="cuda"))
        return s
    T, k, G = case["tokens"], case["top_k"], case["experts"]
    if op == "sort":
        s["ids"], _ = _routing(g, case, DT[case["ids"]])
        s["rows"] = max(ALIGN, int(_room(case) * case["room"]) // ALIGN * ALIGN)
        return s
    H = case["hidden"]
    ids, s["w"] = _routing(g, case)
    s["rows"] = max(ALIGN, _room(case))
    s["row_of"], s["offs"], s["counts"] = _table(ids, G, s["rows"])
    if op == "dispatch":
        s["x"] = _activations(g, T, H)
    elif op == "dispatch_bwd":
        s["dxs"] = _normal(g, (s["rows"], H), 1e-3, DT[case["dx"]])
    elif op == "combine":
        s["ys"] = _normal(g, (s["rows"], H), 1.0, DT[case["ys"]])
    else:
        s["ys"] = _normal(g, (s["rows"], H), 1.0, DT[case["ys"]])
        s["dout"] = _normal(g, (T, H), 1e-3, DT[case["dout"]])
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------------

def _values(fmt, codes, scales, ts, real):
    """Dequantized weights [..., rows, cols] in the floating type `real`."""
    lead, cols = codes.shape[:-1], codes.shape[-1] * 2
    if fmt == "q4_k":
        f = scales[..., :4].contiguous().view(torch.float16).to(real)
        pk = scales[..., 4:]
        s6 = torch.cat([pk[..., :4] & 63, (pk[..., 8:] & 15) | ((pk[..., :4] >> 6) << 4)], -1).to(real)
        m6 = torch.cat([pk[..., 4:8] & 63, (pk[..., 8:] >> 4) | ((pk[..., 4:8] >> 6) << 4)], -1).to(real)
        q = codes.view(*lead, cols // 256, 4, 32)
        q = torch.stack([q & 15, q >> 4], -2).view(*lead, cols // 256, 8, 32)
        return ((f[..., :1] * s6)[..., None] * q.to(real) - (f[..., 1:] * m6)[..., None]).view(*lead, cols)
    q = torch.stack([codes & 15, codes >> 4], -1).view(*lead, cols // BLOCK[fmt], BLOCK[fmt])
    v = torch.tensor(E2M1, dtype=real, device=codes.device)[q.int()]
    if fmt == "mxfp4":
        s = torch.exp2(scales.to(real) - 127)
    else:
        s = scales.view(torch.float8_e4m3fn).to(real) * ts.to(real).view(-1, *([1] * (scales.dim() - 1)))
    return (v * s[..., None]).view(*lead, cols)


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "matvec":
        ts = None if s["ts"] is None else s["ts"]
        w = _values(case["fmt"], s["codes"], s["scales"], ts, torch.float32)
        return (s["x"].float() @ w.t()).to(DT[case["y"]])
    if op == "experts":
        ids = s["ids"].reshape(-1).long()
        e = ids.clamp(min=0)
        w = _values(case["fmt"], s["codes"][e], s["scales"][e], None if s["ts"] is None else s["ts"][e], torch.float32)
        x = s["x"].float()
        x = x.repeat_interleave(case["top_k"], 0) if case["shared_x"] else x
        return torch.where(ids[:, None] >= 0, torch.bmm(w, x[..., None])[..., 0], 0.0).to(DT[case["y"]])
    if op == "sort":
        return _table(s["ids"], case["experts"], s["rows"])
    row = s["row_of"].long()
    live = (row >= 0)[..., None]
    if op == "dispatch":
        # a row past the end takes what is dropped
        xs = torch.zeros((s["rows"] + 1, case["hidden"]), dtype=torch.bfloat16, device=row.device)
        xs[torch.where(row >= 0, row, s["rows"])] = s["x"][:, None, :].expand(-1, case["top_k"], -1)
        return xs[:-1]
    if op == "dispatch_bwd":
        return torch.where(live, s["dxs"][row.clamp(min=0)].float(), 0.0).sum(1).to(DT[case["out"]])
    ys = torch.where(live, s["ys"][row.clamp(min=0)].float(), 0.0)
    if op == "combine":
        return (ys * s["w"][..., None]).sum(1).to(DT[case["out"]])
    dout = s["dout"].float()[:, None, :]
    dys = torch.zeros((s["rows"] + 1, case["hidden"]), dtype=torch.bfloat16, device=row.device)
    dys[torch.where(row >= 0, row, s["rows"])] = (s["w"][..., None] * dout).to(torch.bfloat16)
    return dys[:-1], (ys * dout).sum(-1)


# ---- the library's calls -----------------------------------------------------------------------------------------------------

def _library(s):
    from paper_2609_39223_b200 import api
    case = s["case"]
    op = case["op"]
    if op == "matvec":
        return api.qf_fq_matvec(api.FORMATS[case["fmt"]], s["x"], s["codes"], s["scales"], s["ts"], y_dtype=DT[case["y"]])
    if op == "experts":
        return api.qf_fq_grouped_matvec(api.FORMATS[case["fmt"]], s["x"], s["ids"], s["codes"], s["scales"], s["ts"], y_dtype=DT[case["y"]])
    if op == "sort":
        plan = api.qf_moe_sort(s["ids"], case["experts"], rows_padded=s["rows"])
        return plan.row_of, plan.group_offsets, plan.counts
    plan = api.MoePlan(s["row_of"], s["offs"], s["counts"], s["rows"])
    if op == "dispatch":
        return api.qf_moe_dispatch(s["x"], plan)
    if op == "dispatch_bwd":
        return api.qf_moe_dispatch_bwd(s["dxs"], plan, dx_dtype=DT[case["out"]])
    if op == "combine":
        return api.qf_moe_combine(s["ys"], s["w"], plan, out_dtype=DT[case["out"]])
    return api.qf_moe_combine_bwd(s["dout"], s["ys"], s["w"], plan)


def run(state):
    return _library(state) if own else _plain(state)


# ---- 64 bits -----------------------------------------------------------------------------------------------------------------

def _exact_weight(fmt, codes, scales, ts):
    """Weights [rows, cols] in 64 bits, a sub-block at a time from the definition of the format."""
    rows, cols = codes.shape[0], codes.shape[1] * 2
    w = torch.empty((rows, cols), dtype=torch.float64, device=codes.device)
    if fmt == "q4_k":
        c, r = codes.view(rows, -1, 128), scales.view(rows, -1, 16)
        d, dmin = (r[..., 2 * i:2 * i + 2].contiguous().view(torch.float16)[..., 0].double() for i in (0, 1))
        out = w.view(rows, -1, 256)
        for b in range(8):
            if b < 4:
                s6, m6 = r[..., 4 + b] % 64, r[..., 8 + b] % 64
            else:
                s6 = r[..., 8 + b] % 16 + 16 * (r[..., b] // 64)
                m6 = r[..., 8 + b] // 16 + 16 * (r[..., 4 + b] // 64)
            byte = c[..., 32 * (b // 2):32 * (b // 2) + 32]
            q = (byte % 16 if b % 2 == 0 else byte // 16).double()
            out[..., 32 * b:32 * b + 32] = (d * s6.double())[..., None] * q - (dmin * m6.double())[..., None]
        return w
    for half in (0, 1):
        n = (codes % 16 if half == 0 else codes // 16).double()
        sign = 1.0 - 2.0 * torch.floor(n / 8)
        e, m = torch.floor((n % 8) / 2), n % 2
        w[:, half::2] = sign * torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * torch.exp2(e - 1.0))
    if fmt == "mxfp4":
        scale = torch.exp2(scales.double() - 127.0)
    else:
        n = scales.double()                                        # E4M3: four exponent bits with bias 7, three of fraction
        e, m = torch.floor(n / 8), n % 8
        scale = torch.where(e == 0, m * 2.0 ** -9, (1.0 + m / 8.0) * torch.exp2(e - 7.0)) * ts.double()
    return w * scale.repeat_interleave(BLOCK[fmt], 1)


def exact(case, seed):
    op = case["op"]
    if op == "sort":
        return None                                                # whole numbers: nothing to round
    s = prepare(case, seed)
    if op == "matvec":
        x, step = s["x"].double(), 8192
        return torch.cat([x @ _exact_weight(case["fmt"], s["codes"][r:r + step], s["scales"][r:r + step], s["ts"]).t()
                          for r in range(0, case["N"], step)], 1)
    if op == "experts":
        y = []
        for p, e in enumerate(s["ids"].reshape(-1).tolist()):
            x = s["x"][p // case["top_k"] if case["shared_x"] else p].double() * (e >= 0)      # a dropped pair gives zeros
            y.append(_exact_weight(case["fmt"], s["codes"][e], s["scales"][e], None if s["ts"] is None else s["ts"][e]) @ x)
        return torch.stack(y)
    T, H = case["tokens"], case["hidden"]
    row = s["row_of"].long()
    if op == "dispatch":
        xs = torch.zeros((s["rows"], H), dtype=torch.float64, device="cuda")
        for j in range(case["top_k"]):
            t = torch.nonzero(row[:, j] >= 0)[:, 0]
            xs[row[t, j]] = s["x"][t].double()
        return xs
    if op in ("dispatch_bwd", "combine"):
        out = torch.zeros((T, H), dtype=torch.float64, device="cuda")
        for j in range(case["top_k"]):
            t = torch.nonzero(row[:, j] >= 0)[:, 0]
            out[t] += s["dxs"][row[t, j]].double() if op == "dispatch_bwd" else s["w"][t, j, None].double() * s["ys"][row[t, j]].double()
        return out
    dys = torch.zeros((s["rows"], H), dtype=torch.float64, device="cuda")
    dw = torch.zeros((T, case["top_k"]), dtype=torch.float64, device="cuda")
    for j in range(case["top_k"]):
        t = torch.nonzero(row[:, j] >= 0)[:, 0]
        dys[row[t, j]] = s["w"][t, j, None].double() * s["dout"][t].double()
        dw[t, j] = (s["dout"][t].double() * s["ys"][row[t, j]].double()).sum(-1)
    return dys, dw
