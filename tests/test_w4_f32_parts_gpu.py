"""fp32 rows through 4-bit weights: all 24 bits of a value arrive, in both kernels, and in a network's layers."""
import numpy as np
import pytest
import torch

import paper_2007_09835_b200 as rt3d
import rt3d_synth as synth
import w4ref
from paper_2007_09835_b200 import nets

pytestmark = pytest.mark.gpu


def picking(m, k, group, zeros):
    """Weights of which filter i has one that is not zero: 1 code step, 2^-3, at input 37 i mod k."""
    codes, at = np.full((m, k), 8, np.uint8), 37 * np.arange(m) % k
    codes[np.arange(m), at] = 9
    q = rt3d.W4Weights(m, k, group, zeros=zeros)
    q.codes.copy_(torch.from_numpy(w4ref.laid_out(codes, np.full((m, -(-k // 64) * 64), 8, np.uint8))))
    q.scales.copy_(torch.from_numpy(w4ref.tiled(np.full((m, -(-k // group)), 0.125, np.float32))))
    if zeros:
        q.zeros.copy_(torch.from_numpy(w4ref.tiled(np.full((m, -(-k // group)), 8, np.uint8))))
    return q, at


@pytest.mark.parametrize("rows", [1, 5, 8, 9, 13, 16, 17, 40, 64, 65, 130])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("exponents", [(0, 0), (-100, 100), (-110, -100)])
def test_values_arrive_whole(rows, group, zeros, exponents):
    """(c - z) x s is x / 8, and every sum on the way to it holds 24 bits: the result is exact."""
    m, k = 301, 330
    q, at = picking(m, k, group, zeros)
    rng = np.random.default_rng(rows)
    mantissa = (1 + (2 * rng.integers(0, 1 << 22, (rows, k)) + 1) * 2.0 ** -23) * rng.choice([-1, 1], (rows, k))         # the last bit is set
    values = (mantissa * 2.0 ** rng.integers(exponents[0], exponents[1] + 1, (rows, k))).astype(np.float32)
    x = torch.zeros(rows, 1, 1, 1, 332, device="cuda")
    x[..., :k] = torch.from_numpy(values).view(rows, 1, 1, 1, k).cuda()
    y = torch.zeros(rows, 1, 1, 1, 304, device="cuda")
    rt3d.rt3d_linear_w4(rt3d.tensor_desc(x, k), q, None, rt3d.tensor_desc(y, m))
    np.testing.assert_array_equal(y[..., :m].cpu().numpy().reshape(rows, m), values[:, at] * np.float32(0.125))


@pytest.mark.parametrize("rows", [2, 20])
def test_what_lies_under_2_to_the_minus_133_is_lost(rows):
    m, k = 40, 64
    q, at = picking(m, k, 32, False)
    values = (np.random.default_rng(1).uniform(-1, 1, (rows, k)) * 2.0 ** -120).astype(np.float32)
    x, y = torch.from_numpy(values).view(rows, 1, 1, 1, k).cuda(), torch.zeros(rows, 1, 1, 1, m, device="cuda")
    rt3d.rt3d_linear_w4(x, q, None, y)
    got, want = y.cpu().numpy().reshape(rows, m).astype(np.float64), values[:, at].astype(np.float64) / 8
    assert (np.abs(got - want) <= 2.0 ** -136).all()


@pytest.mark.parametrize("n", [1, 3, 40])
def test_layers_of_a_network(n):
    plan = [synth.ConvSpec("conv1", 3, 16, (3, 3, 3), (1, 1, 1), (1, 1, 1), True), synth.PoolSpec("pool1", (2, 2, 2), (2, 2, 2), (0, 0, 0))]
    specs = [synth.ConvSpec("fc6", 512, 200, (1, 1, 1), (1, 1, 1), (0, 0, 0), True), synth.ConvSpec("fc7", 200, 11, (1, 1, 1), (1, 1, 1), (0, 0, 0), False)]
    L = synth.make_layer(plan[0], 7, 0, 4, 4, "bernoulli", 0.5)
    fc = [synth.make_layer(sp, 7, 10 + i, 4, 4, "none", None) for i, sp in enumerate(specs)]
    net = nets.C3DNet(plan, {"conv1": nets.ConvLayer(plan[0], L["w"], L["bias"], L["mask"], 4, 4, torch.float32)},
                      fc_layers=[nets.LinearW4Layer(sp, f["w"], f["bias"], 32, True, dtype=torch.float32) for sp, f in zip(specs, fc)])
    x = nets.to_device(synth.make_input(7, (n, 4, 8, 8, 3)), torch.float32)
    for _ in range(2):
        y = net.forward(x)
    keep = {}
    last = net.forward(x, keep=keep).clone()
    assert torch.equal(net.forward(x)[..., :11], last[..., :11]) and y.dtype == torch.float32
    cur = keep["pool1"].reshape(n, -1).cpu().numpy()
    for sp, f in zip(specs, fc):
        codes, scales, zero = w4ref.quantize(f["w"].reshape(sp.cout, sp.cin).astype(np.float32), 32, True)
        want, size = w4ref.linear(cur, w4ref.values(codes, scales, zero, 32), f["bias"].astype(np.float64), sp.relu)
        got = keep[sp.name][..., :sp.cout].reshape(n, -1).cpu().numpy()
        assert (np.abs(got - want) <= w4ref.tolerance(size, sp.cin, 32)).all(), sp.name
        cur = got
    assert rt3d.rt3d_last_device_status() == rt3d.OK
