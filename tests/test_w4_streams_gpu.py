"""Layers on a stream that is not the current one: what a call makes for itself is in that stream's order."""
import numpy as np
import pytest
import torch

import rt3d_synth as synth
import w4ref
from paper_2007_09835_b200 import nets

pytestmark = pytest.mark.gpu

BUSY = 1 << 26                                      # clocks, some 35 ms


def spec(m, k, relu=False):
    return synth.ConvSpec("fc", k, m, (1, 1, 1), (1, 1, 1), (0, 0, 0), relu)


def weights(m, k, seed):
    return (np.random.default_rng(seed).standard_normal((m, k)) * 0.05).astype(np.float32)


def codes_of(w, group, zeros):
    codes, scales, zero = w4ref.quantize(w, group, zeros)
    return w4ref.laid_out(codes, np.repeat(zero, group, 1)), w4ref.tiled(scales)


@pytest.mark.parametrize("source", ["numpy", "host tensor"])
def test_weights_from_the_host_are_quantised_on_a_side_stream(source):
    m, k, group = 512, 1024, 64
    layer = nets.LinearW4Layer(spec(m, k), weights(m, k, 0), None, group, True)
    w = weights(m, k, 1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    layer.quantize(w if source == "numpy" else torch.from_numpy(w), stream=side.cuda_stream)
    junk = [torch.full((m, k), 7.0, device="cuda") for _ in range(4)]            # the current stream's next allocations
    torch.cuda.synchronize()
    codes, scales = codes_of(w, group, True)
    np.testing.assert_array_equal(layer.weights.codes.cpu().numpy(), codes)
    np.testing.assert_array_equal(layer.weights.scales.float().cpu().numpy(), scales)
    assert all(bool((j == 7).all()) for j in junk)


def test_the_default_stream_by_its_handle():
    """Handle 0 is the default stream; named from inside another one."""
    m, k, group = 64, 128, 32
    layer = nets.LinearW4Layer(spec(m, k), weights(m, k, 0), None, group, False)
    w = weights(m, k, 2)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        layer.quantize(w, stream=0)
    torch.cuda.synchronize()
    codes, scales = codes_of(w, group, False)
    np.testing.assert_array_equal(layer.weights.codes.cpu().numpy(), codes)
    np.testing.assert_array_equal(layer.weights.scales.float().cpu().numpy(), scales)


@pytest.mark.parametrize("kind", ["4-bit", "dense"])
def test_an_output_made_by_the_call_is_zeroed_before_the_kernel(kind):
    """The current stream is busy: zeros that it brought would come after the products."""
    m, k = 40, 64
    w = weights(m, k, 3)
    make = nets.LinearW4Layer if kind == "4-bit" else lambda sp, w, b, group: nets.ConvLayer(sp, w.reshape(m, k, 1, 1, 1), b, None, dense=True)
    layer = make(spec(m, k), w, np.ones(m, np.float32), 32)
    x = torch.rand(3, 1, 1, 1, k, device="cuda").to(torch.bfloat16)
    want = layer(x).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(BUSY)
    y = layer(x, stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert bool((want != 0).any()) and torch.equal(y, want)


def test_pools_and_sums_that_make_their_output():
    pool = synth.PoolSpec("p", (2, 2, 2), (2, 2, 2), (0, 0, 0))
    a, b = (torch.rand(2, 4, 6, 6, 16, device="cuda").to(torch.bfloat16) for _ in range(2))
    for call in (lambda s: nets.maxpool(a, 16, pool, stream=s), lambda s: nets.add_relu(a, b, 16, stream=s)):
        want = call(None).clone()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        torch.cuda._sleep(BUSY)
        y = call(side.cuda_stream)
        torch.cuda.synchronize()
        assert bool((want != 0).any()) and torch.equal(y, want)


@pytest.mark.parametrize("keep", [False, True])
def test_a_networks_first_pass_on_a_side_stream(keep):
    plan = [synth.ConvSpec("conv1", 3, 16, (3, 3, 3), (1, 1, 1), (1, 1, 1), True), synth.PoolSpec("pool1", (2, 2, 2), (2, 2, 2), (0, 0, 0))]
    L = synth.make_layer(plan[0], 7, 0, 4, 4, "bernoulli", 0.5)
    layers = {"conv1": nets.ConvLayer(plan[0], L["w"], L["bias"], L["mask"], 4, 4, torch.bfloat16)}
    fc = [nets.LinearW4Layer(spec(200, 512, True), weights(200, 512, 1), np.ones(200, np.float32), 32)]
    x = nets.to_device(synth.make_input(7, (2, 4, 8, 8, 3)))
    first = {}
    want = nets.C3DNet(plan, layers, fc_layers=fc).forward(x, keep=first).clone()
    net = nets.C3DNet(plan, layers, fc_layers=fc)                    # without buffers
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(BUSY)
    y = net.forward(x, keep={} if keep else None, stream=side.cuda_stream)
    torch.cuda.synchronize()
    assert bool((want != 0).any()) and torch.equal(y, want)
