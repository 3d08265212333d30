"""4-bit layers among a network's own, and the way of a layer's weights: pruned, updated under the mask, quantised, used."""
import numpy as np
import pytest
import torch

import orthoref
import paper_2007_09835_b200 as rt3d
import rt3d_synth as synth
import w4ref
from paper_2007_09835_b200 import nets

pytestmark = pytest.mark.gpu

PLAN = [synth.ConvSpec("conv1", 3, 16, (3, 3, 3), (1, 1, 1), (1, 1, 1), True), synth.PoolSpec("pool1", (2, 2, 2), (2, 2, 2), (0, 0, 0))]
FC = [synth.ConvSpec("fc6", 512, 200, (1, 1, 1), (1, 1, 1), (0, 0, 0), True), synth.ConvSpec("fc7", 200, 96, (1, 1, 1), (1, 1, 1), (0, 0, 0), True),
      synth.ConvSpec("fc8", 96, 11, (1, 1, 1), (1, 1, 1), (0, 0, 0), False)]


def network(group=32, zeros=True):
    conv = synth.make_layer(PLAN[0], 7, 0, 4, 4, "bernoulli", 0.5)
    layers = {"conv1": nets.ConvLayer(PLAN[0], conv["w"], conv["bias"], conv["mask"], 4, 4, torch.bfloat16)}
    fc = [synth.make_layer(sp, 7, 10 + i, 4, 4, "none", None) for i, sp in enumerate(FC)]
    return nets.C3DNet(PLAN, layers, fc_layers=[nets.LinearW4Layer(sp, L["w"], L["bias"], group, zeros) for sp, L in zip(FC, fc)]), fc


def check(net, fc, x, group, zeros, y=None):
    """Layer by layer against 64 bits on what the layer before has put out."""
    keep = {}
    last = net.forward(x, keep=keep).clone()
    cur = keep["pool1"].reshape(x.shape[0], -1).float().cpu().numpy()
    for sp, L in zip(FC, fc):
        codes, scales, zero = w4ref.quantize(L["w"].reshape(sp.cout, sp.cin).astype(np.float32), group, zeros)
        want, size = w4ref.linear(cur, w4ref.values(codes, scales, zero, group), L["bias"].astype(np.float64), sp.relu)
        tol = w4ref.tolerance(size, sp.cin, group)
        got = keep[sp.name][..., :sp.cout].reshape(x.shape[0], -1).float().cpu().numpy()
        assert (np.abs(got - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol)).all(), sp.name
        cur = got
    if y is not None:
        assert torch.equal(y[..., :11], last[..., :11])
    return last


@pytest.mark.parametrize("n", [1, 3, 40])
@pytest.mark.parametrize("group,zeros", [(32, True), (128, False)])
def test_layers_of_a_network(n, group, zeros):
    net, fc = network(group, zeros)
    x = nets.to_device(synth.make_input(7, (n, 4, 8, 8, 3)))
    with rt3d.planning():
        net.forward(x)
    for _ in range(3):                                              # the first pass is noted, the others are issued from the notes
        y = net.forward(x)
    check(net, fc, x, group, zeros, y)
    before = rt3d.rt3d_launch_count()
    net.forward(x)
    assert rt3d.rt3d_launch_count() - before == 2 + len(FC)         # nothing of a noted pass is left out
    graphed = nets.GraphedForward(net, x)
    graphed()
    torch.cuda.synchronize()
    assert torch.equal(graphed.y[..., :11], y[..., :11])
    assert rt3d.rt3d_last_device_status() == rt3d.OK


def test_a_noted_pass_follows_its_layers():
    net, fc = network()
    x = nets.to_device(synth.make_input(7, (2, 4, 8, 8, 3)))
    net.forward(x), net.forward(x)
    fc[1]["w"] = fc[1]["w"] * np.float32(0.5)                       # new weights into the same arrays
    net.fc_layers[1].quantize(fc[1]["w"])
    check(net, fc, x, 32, True, net.forward(x).clone())
    fc[2]["w"] = fc[2]["w"][::-1].copy()                            # another layer in its place
    net.fc_layers[2] = nets.LinearW4Layer(FC[2], fc[2]["w"], fc[2]["bias"], 32, True)
    check(net, fc, x, 32, True, net.forward(x).clone())
    fc[0]["bias"] = fc[0]["bias"] + np.float32(1)                   # another bias
    net.fc_layers[0].bias = torch.from_numpy(fc[0]["bias"]).cuda()
    check(net, fc, x, 32, True, net.forward(x).clone())
    q = rt3d.W4Weights(96, 200, 32, zeros=True)                     # other weights
    rt3d.rt3d_w4_quantize(torch.from_numpy(fc[1]["w"]).cuda(), q)
    net.fc_layers[1].weights = q
    check(net, fc, x, 32, True, net.forward(x).clone())


def test_layers_that_are_refused():
    w = np.zeros((96, 200, 1, 1, 1), np.float32)
    with pytest.raises(ValueError):
        nets.LinearW4Layer(synth.ConvSpec("f", 200, 96, (1, 1, 1), (2, 1, 1), (0, 0, 0)), w, None)
    with pytest.raises(ValueError):
        nets.LinearW4Layer(synth.ConvSpec("f", 200, 64, (1, 1, 1), (1, 1, 1), (0, 0, 0)), w, None)
    with pytest.raises(ValueError):
        nets.LinearW4Layer(FC[1], rt3d.W4Weights(96, 128, 32), None)
    q = rt3d.W4Weights(96, 200, 32)
    with pytest.raises(AttributeError):
        q.codes = q.codes.clone()
    with pytest.raises(ValueError):
        rt3d.W4Weights(96, 200, 32, codes=q.codes[:-1], scales=q.scales)
    with pytest.raises(ValueError):
        rt3d.W4Weights(96, 200, 32, codes=q.codes, scales=q.scales.float())
    with pytest.raises(rt3d.Rt3dError):
        rt3d.W4Weights(96, 200, 48)
    layer = nets.LinearW4Layer(FC[1], w, None)
    with pytest.raises(rt3d.Rt3dError) as e:
        layer(torch.zeros(1, 1, 1, 1, 200, device="cuda"))          # float32 rows, a bfloat16 layer's output
    assert e.value.status == rt3d.ERR_SHAPE


def test_pruned_updated_quantised_used():
    """Pruning decision -> mask -> masked updates -> 4-bit weights -> products, each against its definition on what the stage before
    has left on the device."""
    m, k, group = 200, 512, 64
    gen = torch.Generator().manual_seed(5)
    w = (torch.randn(m, k, generator=gen) * 0.05).cuda()
    norms = torch.empty(m // 4, k // 4, 1, device="cuda")
    rt3d.rt3d_kgs_group_norms(w.view(m, k, 1, 1, 1), 4, 4, 2, norms)
    keep = torch.empty(m // 4, k // 4, 1, dtype=torch.uint8, device="cuda")
    rt3d.rt3d_kgs_reweight(norms, 1e-3, float(norms.median()), None, keep)
    mask = torch.empty(m, k, 1, 1, 1, dtype=torch.uint8, device="cuda")
    rt3d.rt3d_kgs_expand_mask(keep, m, k, 1, 1, 1, 4, 4, mask)
    mask = mask.view(m, k)
    assert 0.3 < mask.float().mean() < 0.7
    momentum = torch.zeros_like(w)
    ws = torch.empty(rt3d.rt3d_ortho_workspace(m, k), dtype=torch.uint8, device="cuda")
    lr, scale = 1e-2, 0.2 * k ** 0.5
    for step in range(3):
        g = (orthoref.matrix("falling", m, k, step) * 0.01).float().cuda()
        want, want_m, o = orthoref.update(w.double(), momentum.double(), g, mask, lr, 0.9, True, 0.1, scale)
        rt3d.rt3d_ortho_update(w, momentum, g, mask, ws, lr=lr, momentum_factor=0.9, weight_decay=0.1, scale=scale)
        size = lr * scale * o.norm()
        assert (w.double() - want).norm() <= 1e-4 * size + 2.0 ** -22 * (want.norm() + size)
        assert (momentum.double() - want_m).norm() <= 2.0 ** -23 * (want_m.norm() + g.double().norm())
        assert bool((w[mask == 0] == 0).all())
    q = rt3d.W4Weights(m, k, group)
    rt3d.rt3d_w4_quantize(w, q)
    codes, scales, zero = w4ref.quantize(w.cpu().numpy(), group, False)
    values = w4ref.values(codes, scales, zero, group)
    back = torch.empty_like(w)
    rt3d.rt3d_w4_unpack(q, back)
    assert np.array_equal(back.cpu().numpy(), values.astype(np.float32)) and bool((back[mask == 0] == 0).all())    # the mask survives
    x = torch.rand(5, 1, 1, 1, k, generator=gen).to(torch.bfloat16).cuda()
    y = torch.zeros(5, 1, 1, 1, m, dtype=torch.bfloat16, device="cuda")
    rt3d.rt3d_linear_w4(x, q, None, y, relu=True)
    want, size = w4ref.linear(x.view(5, k).float().cpu().numpy(), values, None, True)
    tol = w4ref.tolerance(size, k, group)
    assert (np.abs(y.view(5, m).float().cpu().numpy() - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol)).all()
