"""The cache calls and the products from codes together, as examples/attention_layer.py uses them, against the layer in 64 bits.

Quantization jumps, so the 64-bit layer takes the library's projected rows as they are (checked by themselves), quantizes them with the
oracle and computes the rest. Tolerances in relative 2-norm: a rounding to BF16 is off by 2^-9 / sqrt(3) = 1.1e-3 in the mean square;
a projection has one (NVFP4's weights in the prompt one more), attention one and its FP16 weights 2^-12 / sqrt(3), the output one more, and in the
prompt queries, keys, values and the weights of the dense attention are BF16 too: 6 of them, 2.8e-3. 1e-2 is asked for."""
import importlib.util
from pathlib import Path

import pytest
import torch

import oracle
from paper_2609_39223_b200 import api
from util import bits_to_torch, torch_to_bits

pytestmark = pytest.mark.gpu
spec = importlib.util.spec_from_file_location("attention_layer", Path(__file__).resolve().parent.parent / "examples" / "attention_layer.py")
attention_layer = importlib.util.module_from_spec(spec)
spec.loader.exec_module(attention_layer)


def off(got, want):
    return ((got.double() - want.double()).norm() / want.double().norm()).item()


def written(layer, x, ts):
    """What the cache makes of rows x [tokens, kv_heads, dim]."""
    r = oracle.qdq(layer.fmt, torch_to_bits(x.cpu().reshape(-1, layer.dim)), None if ts is None else float(ts))
    return bits_to_torch(r["out"]).view(x.shape).double().cuda()


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4"])
@pytest.mark.parametrize("batch,hidden,heads,kv_heads,dim,prompt,steps", [(1, 256, 4, 4, 64, 1, 3), (3, 512, 8, 2, 128, 33, 40)])
def test_layer(fmt, batch, hidden, heads, kv_heads, dim, prompt, steps):
    per = (prompt + steps + 15) // 16
    layer = attention_layer.AttentionLayer(api.FORMATS[fmt], hidden, heads, kv_heads, dim, batch * per, seed=batch)
    g = torch.Generator(device="cuda").manual_seed(batch)
    table = torch.randperm(batch * per, generator=g, device="cuda").to(torch.int32).view(batch, per)
    hats = [api.qf_dequant(layer.fmt, p["codes"], p["scales"], p.get("tensor_scale"), w.shape[0], w.shape[1]).double()
            for w, p in zip((layer.w_qkv, layer.w_out), layer.packed)]
    seen = [[[], []] for _ in range(batch)]

    def attend(q, b):
        k, v = (torch.cat(s).repeat_interleave(heads // kv_heads, 1) for s in seen[b])
        s = torch.einsum("qhd,jhd->hqj", q.double(), k) * dim ** -0.5
        s += torch.full(s.shape[1:], -torch.inf, device="cuda", dtype=torch.float64).triu(s.shape[2] - s.shape[1] + 1)
        return torch.einsum("hqj,jhd->qhd", torch.softmax(s, -1), v).flatten(1)

    for b in range(batch):
        x = torch.randn((prompt, hidden), generator=g, device="cuda").to(torch.bfloat16)
        out = layer.prompt(x, table[b:b + 1])
        qkv = api.qf_fq_linear_fwd(x, layer.w_qkv, layer.fmt, api.FMT_NONE, **(dict(w_tscale=layer.packed[0]["tensor_scale"], flags=api.W_TSCALE_GIVEN) if fmt == "nvfp4" else {}))
        assert off(qkv, x.double() @ hats[0].t()) < 1e-2
        q, k, v = layer.split(qkv)
        for s, rows, ts in zip(seen[b], (k, v), (layer.cache.k_tscale, layer.cache.v_tscale)):
            s.append(written(layer, rows.contiguous(), ts))
        assert off(out, attend(q, b) @ hats[1].t()) < 1e-2

    lens = torch.full((batch,), prompt, dtype=torch.int32, device="cuda")
    x = torch.randn((batch, hidden), generator=g, device="cuda").to(torch.bfloat16)
    ws = api.workspace(api.OP_KV_ATTENTION, batch, heads, dim, kv_heads)
    for _ in range(steps):
        lens += 1
        qkv = layer.matvec(0, x)
        assert off(qkv, x.double() @ hats[0].t()) < 1e-2
        q, k, v = layer.split(qkv)
        out = layer.step(x, table, lens, ws)
        want = []
        for b in range(batch):
            for s, rows, ts in zip(seen[b], (k, v), (layer.cache.k_tscale, layer.cache.v_tscale)):
                s.append(written(layer, rows[b:b + 1].contiguous(), ts))
            want.append(attend(q[b:b + 1], b))
        assert off(out, torch.cat(want) @ hats[1].t()) < 1e-2
        x = (out / out.float().square().mean(-1, keepdim=True).sqrt()).to(torch.bfloat16)


def test_example_runs(capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["attention_layer.py", "--format", "mxfp4", "--prompt", "17", "--steps", "2", "--batch", "2"])
    attention_layer.main()
    assert "2 tokens for 2 sequences" in capsys.readouterr().out
