"""An attention layer that answers from 4-bit weights and a 4-bit key/value cache, as a rollout runs it.

A prompt goes through the quantization-aware product (qf_fq_linear_fwd), its keys and values are quantized into the cache (qf_kv_append) and
read back (qf_kv_read) for the dense attention of the prompt, so that every token of it sees what later tokens will see. Then tokens
come one by one for a batch of sequences: products from the codes (qf_fq_matvec), a row written, attention over the cache
(qf_kv_attention). Nothing is read back from the GPU in between, and a step can be captured into a graph.

    python examples/attention_layer.py [--format nvfp4|mxfp4] [--prompt 100] [--steps 20] [--batch 4] [--hidden 512] [--heads 8] [--kv-heads 2]
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))

from paper_2609_39223_b200 import api  # noqa: E402


class AttentionLayer:
    """W_qkv [(heads + 2 * kv_heads) * dim, hidden] (queries, keys, values) and W_out [hidden, heads * dim] in BF16, and a paged cache that all
    sequences share. Positions (rotary embeddings, say) are the caller's and left out."""

    def __init__(self, fmt: int, hidden: int, heads: int, kv_heads: int, dim: int, pages: int, page_size: int = 16, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        make = lambda *shape: (torch.randn(shape, generator=g, device=device) * shape[-1] ** -0.5).to(torch.bfloat16)
        self.fmt, self.hidden, self.heads, self.kv_heads, self.dim = fmt, hidden, heads, kv_heads, dim
        self.w_qkv, self.w_out = make((heads + 2 * kv_heads) * dim, hidden), make(hidden, heads * dim)
        self.packed = [api.qf_qdq(fmt, w, want_out=False) for w in (self.w_qkv, self.w_out)]
        # tensor scales for keys and values of about N(0, 1), as a calibration would give them
        scale = lambda: torch.full((1,), 6.0 / (6.0 * 448.0), device=device) if fmt == api.FMT_NVFP4 else None
        self.cache = api.KvCache.empty(fmt, pages, page_size, kv_heads, dim, scale(), scale(), device=device)

    def slots(self, table: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        """Slots of the given positions [batch, n] of the sequences."""
        size = self.cache.page_size
        return (table.gather(1, positions // size).long() * size + positions % size).reshape(-1)

    def split(self, qkv: torch.Tensor):
        """Queries, keys and values [tokens, heads, dim] of a projection's rows, as slices."""
        return qkv.unflatten(-1, (-1, self.dim)).split((self.heads, self.kv_heads, self.kv_heads), -2)

    def prompt(self, x: torch.Tensor, table: torch.Tensor) -> torch.Tensor:
        """Output [tokens, hidden] for one sequence's prompt x [tokens, hidden], whose pages table [1, pages] lists."""
        tokens = x.shape[0]
        given = dict(w_tscale=self.packed[0].get("tensor_scale"), flags=api.W_TSCALE_GIVEN) if self.fmt == api.FMT_NVFP4 else {}
        q, k, v = self.split(api.qf_fq_linear_fwd(x, self.w_qkv, self.fmt, api.FMT_NONE, **given))
        slots = self.slots(table, torch.arange(tokens, device=x.device)[None])
        api.qf_kv_append(self.cache, k, v, slots)
        k, v = api.qf_kv_read(self.cache, slots)
        a = torch.nn.functional.scaled_dot_product_attention(*(t.transpose(0, 1)[None] for t in (q, k, v)), is_causal=True, enable_gqa=True)
        given = dict(w_tscale=self.packed[1].get("tensor_scale"), flags=api.W_TSCALE_GIVEN) if self.fmt == api.FMT_NVFP4 else {}
        return api.qf_fq_linear_fwd(a[0].transpose(0, 1).reshape(tokens, -1).contiguous(), self.w_out, self.fmt, api.FMT_NONE, **given)

    def matvec(self, which: int, x: torch.Tensor) -> torch.Tensor:
        w = self.packed[which]
        return api.qf_fq_matvec(self.fmt, x, w["codes"], w["scales"], w.get("tensor_scale"))

    def step(self, x: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, ws: torch.Tensor | None = None) -> torch.Tensor:
        """Output [batch, hidden] for one new token x [batch, hidden] of every sequence; lens [batch] counts them already."""
        q, k, v = self.split(self.matvec(0, x))
        api.qf_kv_append(self.cache, k, v, self.slots(table, (lens - 1).long()[:, None]))
        return self.matvec(1, api.qf_kv_attention(self.cache, q[:, None], table, lens, ws=ws).flatten(1))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--format", default="nvfp4", choices=("nvfp4", "mxfp4"))
    for name, default in (("prompt", 100), ("steps", 20), ("batch", 4), ("hidden", 512), ("heads", 8), ("kv-heads", 2), ("dim", 64)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args()
    per = (a.prompt + a.steps + 15) // 16
    layer = AttentionLayer(api.FORMATS[a.format], a.hidden, a.heads, a.kv_heads, a.dim, a.batch * per)
    g = torch.Generator(device="cuda").manual_seed(1)
    table = torch.randperm(a.batch * per, generator=g, device="cuda").to(torch.int32).view(a.batch, per)
    for b in range(a.batch):
        out = layer.prompt(torch.randn((a.prompt, a.hidden), generator=g, device="cuda").to(torch.bfloat16), table[b:b + 1])
    print(f"prompts of {a.prompt} tokens: |out| {out.float().norm():.4f}")
    lens = torch.full((a.batch,), a.prompt, dtype=torch.int32, device="cuda")
    x = torch.randn((a.batch, a.hidden), generator=g, device="cuda").to(torch.bfloat16)
    ws = api.workspace(api.OP_KV_ATTENTION, a.batch, a.heads, a.dim, a.kv_heads)
    for _ in range(a.steps):
        lens += 1
        x = layer.step(x, table, lens, ws)
    print(f"{a.steps} tokens for {a.batch} sequences from 4-bit codes: |out| {x.float().norm():.4f}")


if __name__ == "__main__":
    main()
