"""Calls with one tensor in host memory are refused, whichever it is."""
import pytest
import torch

import paper_2007_09835_b200 as rt3d

pytestmark = pytest.mark.gpu


def variants(tensors):
    """The tensors with one of them in host memory, by name."""
    for name, t in tensors.items():
        if t is not None:
            yield name, {**tensors, name: t.cpu()}


def test_four_bit_calls():
    q = rt3d.W4Weights(16, 64, 32)
    before = rt3d.rt3d_launch_count()
    w = torch.zeros(16, 64)
    for call in (lambda: rt3d.rt3d_w4_quantize(w, q), lambda: rt3d.rt3d_w4_unpack(q, w)):
        with pytest.raises(ValueError):
            call()
    tensors = dict(x=torch.zeros(2, 1, 1, 1, 64, device="cuda"), bias=torch.zeros(16, device="cuda"), y=torch.zeros(2, 1, 1, 1, 16, device="cuda"))
    for name, v in variants(tensors):
        with pytest.raises(ValueError):
            rt3d.rt3d_linear_w4(v["x"], q, v["bias"], v["y"])
        if name == "bias":
            with pytest.raises(ValueError):
                rt3d.rt3d_linear_w4(rt3d.tensor_desc(v["x"]), q, v["bias"], rt3d.tensor_desc(v["y"]))
    host = rt3d.W4Weights(16, 64, 32, device="cpu")
    with pytest.raises(ValueError):
        rt3d.rt3d_linear_w4(tensors["x"], host, None, tensors["y"])
    assert rt3d.rt3d_launch_count() == before


def test_orthogonalised_updates():
    m, k = 16, 64
    ws = torch.zeros(rt3d.rt3d_ortho_workspace(m, k), dtype=torch.uint8, device="cuda")
    g = torch.ones(m, k, device="cuda")
    before = rt3d.rt3d_launch_count()
    for _, v in variants(dict(g=g, out=torch.zeros(m, k, dtype=torch.bfloat16, device="cuda"), workspace=ws)):
        with pytest.raises(ValueError):
            rt3d.rt3d_orthogonalize(**v)
    tensors = dict(w=torch.zeros(m, k, device="cuda"), momentum=torch.zeros(m, k, device="cuda"), g=g, mask=torch.ones(m, k, dtype=torch.uint8, device="cuda"),
                   workspace=ws)
    for _, v in variants(tensors):
        with pytest.raises(ValueError):
            rt3d.rt3d_ortho_update(**v, lr=0.1)
    assert rt3d.rt3d_launch_count() == before
