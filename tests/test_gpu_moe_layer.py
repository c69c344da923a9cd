"""The routing calls, the grouped products and the products from codes together, as examples/moe_layer.py uses them, against the
layer written out token by token in 64 bits with autograd.

Tolerance. The chain rounds to BF16 about six times (gate/up, SwiGLU, expert outputs, the result; as many gradients on the way
back); each rounding moves a value by up to 2^-9 of itself, by 2^-9 / sqrt(3) in the mean square, so six of them make 2.8e-3 of
relative 2-norm, and NVFP4's and Q4_K's dequantized weights in decoding are unrounded where training rounds them, once more the
same. 1e-2 is asked for."""
import importlib.util
from pathlib import Path

import pytest
import torch

from paper_2609_39223_b200 import api

pytestmark = pytest.mark.gpu
spec = importlib.util.spec_from_file_location("moe_layer", Path(__file__).resolve().parent.parent / "examples" / "moe_layer.py")
moe_layer = importlib.util.module_from_spec(spec)
spec.loader.exec_module(moe_layer)


def off(got, want):
    return ((got.double() - want.double()).norm() / want.double().norm()).item()


@pytest.mark.parametrize("fmt", ["nvfp4", "mxfp4", "q4_k"])
@pytest.mark.parametrize("tokens,experts,hidden,mlp,top_k", [(1, 4, 256, 256, 1), (37, 8, 512, 256, 3), (300, 5, 256, 512, 2)])
def test_layer(fmt, tokens, experts, hidden, mlp, top_k):
    layer = moe_layer.MoeLayer(api.FORMATS[fmt], experts, hidden, mlp, seed=tokens)
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x = torch.randn((tokens, hidden), generator=g, device="cuda").to(torch.bfloat16)
    ids, weights = layer.route(torch.randn((tokens, experts), generator=g, device="cuda"), top_k)
    if tokens > 1:
        ids[tokens // 2] = -1                                   # a token that the router drops
    out, saved = layer.forward(x, ids, weights)
    dout = torch.randn((tokens, hidden), generator=g, device="cuda").to(torch.bfloat16)
    grads = layer.backward(dout, saved)

    hat = lambda w: torch.stack([api.qf_qdq(api.FORMATS[fmt], e.contiguous())["out"] for e in w]).double().requires_grad_()
    xd, wd, gu, dn = x.double().requires_grad_(), weights.double().requires_grad_(), hat(layer.w_gate_up), hat(layer.w_down)
    ref = torch.zeros((tokens, hidden), dtype=torch.float64, device="cuda")
    for e in range(experts):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if t.numel():
            gate, up = (xd[t] @ gu[e].T).chunk(2, -1)
            ref = ref.index_add(0, t, wd[t, j, None] * ((torch.nn.functional.silu(gate) * up) @ dn[e].T))
    (ref * dout.double()).sum().backward()
    assert off(out, ref.detach()) <= 1e-2
    for got, want in zip(grads, (xd.grad, wd.grad, gu.grad, dn.grad)):
        assert off(got, want) <= 1e-2
    if tokens > 1:
        assert (out[tokens // 2] == 0).all() and (grads[0][tokens // 2] == 0).all() and (grads[1][tokens // 2] == 0).all()

    few = min(9, tokens)
    packed = layer.quantize()
    answer = layer.decode(packed, x[:few].contiguous(), ids[:few].contiguous(), weights[:few].contiguous())
    assert off(answer, ref[:few].detach()) <= 1e-2


def test_example_runs(capsys):
    import sys
    argv, sys.argv = sys.argv, ["moe_layer.py", "--tokens", "64", "--experts", "8", "--hidden", "256", "--mlp", "256", "--top-k", "2"]
    try:
        moe_layer.main()
    finally:
        sys.argv = argv
    assert "decoded 4 tokens" in capsys.readouterr().out
