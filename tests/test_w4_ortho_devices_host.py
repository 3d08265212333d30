"""Tensors in host memory are refused before their addresses reach a kernel."""
import pytest
import torch

import paper_2007_09835_b200 as rt3d


@pytest.fixture
def weights():
    return rt3d.W4Weights(16, 64, 32, zeros=True, device="cpu")


def test_quantisation_and_its_inverse(weights):
    for call in (lambda: rt3d.rt3d_w4_quantize(torch.zeros(16, 64), weights), lambda: rt3d.rt3d_w4_unpack(weights, torch.zeros(16, 64)),
                 lambda: rt3d.rt3d_w4_quantize(torch.zeros(16, 64), weights, stream=0)):
        with pytest.raises(ValueError, match="host"):
            call()


@pytest.mark.parametrize("described", [False, True])
def test_products(weights, described):
    x, y, bias = torch.zeros(2, 1, 1, 1, 64), torch.zeros(2, 1, 1, 1, 16), torch.zeros(16)
    if described:
        x, y = rt3d.tensor_desc(x), rt3d.tensor_desc(y)
    for b in (None, bias):
        with pytest.raises(ValueError):
            rt3d.rt3d_linear_w4(x, weights, b, y, stream=0)


def test_orthogonalised_updates():
    m, k = 16, 64
    w, momentum, g, mask = torch.zeros(m, k), torch.zeros(m, k), torch.zeros(m, k), torch.ones(m, k, dtype=torch.uint8)
    out, ws = torch.zeros(m, k, dtype=torch.bfloat16), torch.zeros(rt3d.rt3d_ortho_workspace(m, k), dtype=torch.uint8)
    with pytest.raises(ValueError, match="device"):
        rt3d.rt3d_orthogonalize(g, out, ws, stream=0)
    for mk in (None, mask):
        with pytest.raises(ValueError, match="device"):
            rt3d.rt3d_ortho_update(w, momentum, g, mk, ws, lr=0.1, stream=0)
