"""4-bit layers on a stream that is not the current one: what a call makes for itself is in that stream's order."""
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
