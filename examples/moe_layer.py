"""A mixture-of-experts SwiGLU layer on the library's calls, as it is trained and as it answers.

Training runs the quantization-aware grouped products on rows in expert order (qf_moe_sort, qf_moe_dispatch,
qf_fq_grouped_linear_fwd / _bwd, qf_moe_combine and the gradients). Decoding runs the same weights from their 4-bit codes
(qf_qdq_batched, qf_fq_grouped_matvec, qf_moe_combine). Nothing is read back from the GPU in between.

    python examples/moe_layer.py [--format nvfp4|mxfp4|q4_k] [--tokens 512] [--experts 32] [--hidden 512] [--mlp 256] [--top-k 4]
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


class MoeLayer:
    """W_gate_up [experts, 2 * mlp, hidden] (gate rows first) and W_down [experts, hidden, mlp] in BF16; the router's product is the
    caller's. ``fmt`` is the deployment format of the weights; activations stay BF16."""

    def __init__(self, fmt: int, experts: int, hidden: int, mlp: int, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        make = lambda *shape: (torch.randn(shape, generator=g, device=device) * 0.02).to(torch.bfloat16)
        self.fmt, self.experts = fmt, experts
        self.w_gate_up, self.w_down = make(experts, 2 * mlp, hidden), make(experts, hidden, mlp)

    @staticmethod
    def route(logits: torch.Tensor, top_k: int):
        """Expert ids [tokens, top_k] and FP32 weights that add up to 1 per token."""
        top = torch.topk(torch.softmax(logits, -1), top_k, dim=-1)
        return top.indices, top.values / top.values.sum(-1, keepdim=True)

    @staticmethod
    def swiglu(gate_up: torch.Tensor) -> torch.Tensor:
        gate, up = gate_up.float().chunk(2, -1)
        return (torch.nn.functional.silu(gate) * up).to(torch.bfloat16)

    @staticmethod
    def swiglu_backward(d: torch.Tensor, gate_up: torch.Tensor) -> torch.Tensor:
        gate, up = gate_up.float().chunk(2, -1)
        s, d = torch.sigmoid(gate), d.float()
        return torch.cat([d * up * s * (1 + gate * (1 - s)), d * gate * s], -1).to(torch.bfloat16)

    def _scales(self):
        return torch.empty(self.experts, dtype=torch.float32, device=self.w_down.device)      # NVFP4: one tensor scale per expert

    def forward(self, x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor):
        """Output [tokens, hidden] and what the backward needs."""
        plan = api.qf_moe_sort(ids, self.experts)
        offs = plan.group_offsets
        xs = api.qf_moe_dispatch(x, plan)
        gate_up = api.qf_fq_grouped_linear_fwd(xs, self.w_gate_up, offs, self.fmt, api.FMT_NONE, w_tscale=self._scales())
        # rows past the last segment are not written by the product; no pair owns them and the next product leaves them out
        h = self.swiglu(gate_up)
        ys = api.qf_fq_grouped_linear_fwd(h, self.w_down, offs, self.fmt, api.FMT_NONE, w_tscale=self._scales())
        return api.qf_moe_combine(ys, weights, plan), (plan, xs, gate_up, h, ys, weights)

    def backward(self, dout: torch.Tensor, saved):
        """Gradients of the input, the router's weights and both weight tensors (straight through the quantizer)."""
        plan, xs, gate_up, h, ys, weights = saved
        offs = plan.group_offsets
        dys, dweights = api.qf_moe_combine_bwd(dout, ys, weights, plan)
        dh, dw_down = api.qf_fq_grouped_linear_bwd(dys, h, self.w_down, offs, self.fmt, api.FMT_NONE, w_tscale=self._scales())
        dgate_up = self.swiglu_backward(dh, gate_up)
        dxs, dw_gate_up = api.qf_fq_grouped_linear_bwd(dgate_up, xs, self.w_gate_up, offs, self.fmt, api.FMT_NONE, w_tscale=self._scales(),
                                                       dx_dtype=torch.float32)
        return api.qf_moe_dispatch_bwd(dxs, plan), dweights, dw_gate_up, dw_down

    def quantize(self):
        """The payload a serving process keeps: codes, scales and tensor scales of both weights."""
        packed = []
        for w in (self.w_gate_up, self.w_down):
            b = api.qf_qdq_batched(self.fmt, list(w), want_out=False)
            packed.append((torch.stack(b.codes), torch.stack(b.scales), b.tensor_scales))
        return packed

    def decode(self, packed, x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor) -> torch.Tensor:
        """The layer for a few tokens, from the codes: an expert's weights are read once per eight of its tokens, and only those of
        experts in use."""
        gate_up = api.qf_fq_grouped_matvec(self.fmt, x, ids, *packed[0])
        ys = api.qf_fq_grouped_matvec(self.fmt, self.swiglu(gate_up), ids, *packed[1])
        return api.qf_moe_combine(ys, weights)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--format", default="nvfp4", choices=("nvfp4", "mxfp4", "q4_k"))
    for name, default in (("tokens", 512), ("experts", 32), ("hidden", 512), ("mlp", 256), ("top-k", 4)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args()
    layer = MoeLayer(api.FORMATS[a.format], a.experts, a.hidden, a.mlp)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((a.tokens, a.hidden), generator=g, device="cuda").to(torch.bfloat16)
    ids, weights = layer.route(torch.randn((a.tokens, a.experts), generator=g, device="cuda"), a.top_k)
    out, saved = layer.forward(x, ids, weights)
    dx, dweights, dw_gate_up, dw_down = layer.backward(out, saved)          # gradient of |out|^2 / 2
    print(f"trained on {a.tokens} tokens: |out| {out.float().norm():.4f}  |dx| {dx.float().norm():.4f}  |dweights| {dweights.norm():.4f}  "
          f"|dW| {dw_gate_up.norm():.4f} {dw_down.norm():.4f}")
    few = min(4, a.tokens)
    answer = layer.decode(layer.quantize(), x[:few].contiguous(), ids[:few].contiguous(), weights[:few].contiguous())
    off = (answer.float() - out[:few].float()).norm() / out[:few].float().norm()
    print(f"decoded {few} tokens from the codes: {off:.2e} from the training forward")


if __name__ == "__main__":
    main()
