"""A product's bias of another length, type or stride is refused: the kernels read m floats from its address on."""
import pytest
import torch

import paper_2007_09835_b200 as rt3d
import rt3d_synth as synth
from paper_2007_09835_b200 import nets

BAD = [torch.zeros(15), torch.zeros(17), torch.zeros(0), torch.zeros(16, dtype=torch.bfloat16), torch.zeros(16, dtype=torch.float64), torch.zeros(32)[::2]]


class OnDevice(torch.Tensor):
    """A tensor that says it is on a CUDA device: what is looked at before the address is used."""

    def get_device(self):
        return 0


@pytest.mark.parametrize("bias", BAD)
@pytest.mark.parametrize("described", [False, True])
def test_products(bias, described, monkeypatch):
    from paper_2007_09835_b200 import binding as B
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    on = lambda t: t.as_subclass(OnDevice)          # noqa: E731
    module = B.pycall()
    module.setup(torch.float32, torch.bfloat16, lambda device: 0, lambda: 0)
    try:
        q = rt3d.W4Weights(16, 64, 32, device="cpu")
        object.__setattr__(q, "index", 0)
        x, y = on(torch.zeros(2, 1, 1, 1, 64)), on(torch.zeros(2, 1, 1, 1, 16))
        with rt3d.planning(), pytest.raises(ValueError, match="bias"):              # nothing is launched either way
            rt3d.rt3d_linear_w4(rt3d.tensor_desc(x) if described else x, q, on(bias), rt3d.tensor_desc(y) if described else y, stream=0)
        with rt3d.planning():
            for good in (None, on(torch.zeros(16)), on(torch.zeros(16, 1))):
                rt3d.rt3d_linear_w4(rt3d.tensor_desc(x) if described else x, q, good, rt3d.tensor_desc(y) if described else y, stream=0)
    finally:
        module.setup(torch.float32, torch.bfloat16, torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice)


@pytest.mark.parametrize("count", [0, 95, 97])
def test_layers(count):
    spec = synth.ConvSpec("f", 200, 96, (1, 1, 1), (1, 1, 1), (0, 0, 0))
    with pytest.raises(ValueError, match="bias"):
        nets.LinearW4Layer(spec, rt3d.W4Weights(96, 200, 32, device="cpu"), torch.zeros(count), device="cpu")
