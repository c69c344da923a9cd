"""The binding of the routing calls and of the products with a few tokens refuses tensors that are not all on the current device, whichever
tensor it is: a kernel would follow an address of another GPU. Host only: the tensors are stand-ins and the library is never called."""
import pytest
import torch

from paper_2609_39223_b200 import api

BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class Stand:
    """What the binding asks of a tensor."""

    def __init__(self, dtype, *shape, device=0):
        self.dtype, self.shape, self.device = dtype, torch.Size(shape), device
        self.is_cuda = device >= 0

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return self.shape.numel()

    def new_empty(self, shape, dtype):
        return Stand(dtype, *(shape if isinstance(shape, tuple) else (shape,)))


class Called(Exception):
    pass


@pytest.fixture(autouse=True)
def no_gpu(monkeypatch):
    class Lib:
        def __getattr__(self, name):
            def called(*args):
                raise Called(name)
            return called
    monkeypatch.setattr(api, "lib", lambda: Lib())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0)


T, K, G, H, ROWS = 6, 2, 4, 64, 512
PLAN = dict(row_of=(I32, T, K), group_offsets=(I32, G + 1), counts=(I32, G))


def plan(t):
    return api.MoePlan(t["row_of"], t["group_offsets"], t["counts"], ROWS)


CALLS = {
    "sort": (dict(ids=(I32, T, K)), lambda t: api.qf_moe_sort(t["ids"], G, rows_padded=ROWS)),
    "dispatch": (dict(PLAN, x=(BF, T, H), xs=(BF, ROWS, H)), lambda t: api.qf_moe_dispatch(t["x"], plan(t), xs=t["xs"])),
    "dispatch_bwd": (dict(row_of=(I32, T, K), dxs=(F32, ROWS, H), dx=(BF, T, H)),
                     lambda t: api.qf_moe_dispatch_bwd(t["dxs"], api.MoePlan(t["row_of"], None, None, ROWS), dx=t["dx"])),
    "combine": (dict(row_of=(I32, T, K), ys=(BF, ROWS, H), weights=(F32, T, K), out=(BF, T, H)),
                lambda t: api.qf_moe_combine(t["ys"], t["weights"], api.MoePlan(t["row_of"], None, None, ROWS), out=t["out"])),
    "combine_bwd": (dict(PLAN, dout=(BF, T, H), ys=(BF, ROWS, H), weights=(F32, T, K), dys=(BF, ROWS, H), dweights=(F32, T, K)),
                    lambda t: api.qf_moe_combine_bwd(t["dout"], t["ys"], t["weights"], plan(t), dys=t["dys"], dweights=t["dweights"])),
    "matvec": (dict(x=(BF, T, H), codes=(U8, 10, H // 2), scales=(U8, 10, H // 16), ts=(F32, 1), y=(F32, T, 10)),
               lambda t: api.qf_fq_matvec(api.FMT_NVFP4, t["x"], t["codes"], t["scales"], t["ts"], Y=t["y"])),
    "grouped_matvec": (dict(x=(BF, T, H), ids=(I32, T, K), codes=(U8, G, 10, H // 2), scales=(U8, G, 10, H // 16), ts=(F32, G), y=(F32, T * K, 10)),
                       lambda t: api.qf_fq_grouped_matvec(api.FMT_NVFP4, t["x"], t["ids"], t["codes"], t["scales"], t["ts"], Y=t["y"])),
}


@pytest.mark.parametrize("call", CALLS)
def test_every_tensor_has_to_be_on_the_current_device(call):
    kinds, go = CALLS[call]
    make = lambda other=None, device=1: {n: Stand(*k, device=device if n == other else 0) for n, k in kinds.items()}
    with pytest.raises(Called):
        go(make())
    for name in kinds:
        with pytest.raises(ValueError, match="cuda:1"):
            go(make(name))
        with pytest.raises(TypeError):
            go(make(name, device=-1))
