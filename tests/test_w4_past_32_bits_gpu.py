"""Quantisation and its inverse on more than 2^32 weights: the last and a middle tile against the same filters on their own."""
import pytest
import torch

import paper_2007_09835_b200 as rt3d

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group,zeros", [(32, True), (128, False)])
def test_tiles_far_behind(group, zeros):
    m, k = 66016, 65600
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("60 GB of free device memory wanted")
    w = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
    for at in range(0, m, 4096):
        w[at:at + 4096].normal_()
    q = rt3d.W4Weights(m, k, group, zeros=zeros)
    rt3d.rt3d_w4_quantize(w, q)
    back = torch.empty_like(w)
    rt3d.rt3d_w4_unpack(q, back)
    tile = q.codes.numel() // (m // 16)
    for t in (m // 32, m // 16 - 1):
        part, alone = w[16 * t:16 * t + 16], rt3d.W4Weights(16, k, group, zeros=zeros)
        rt3d.rt3d_w4_quantize(part, alone)
        assert torch.equal(q.codes[t * tile:(t + 1) * tile], alone.codes)
        assert torch.equal(q.scales[t], alone.scales[0]) and (not zeros or torch.equal(q.zeros[t], alone.zeros[0]))
        values = torch.empty_like(part)
        rt3d.rt3d_w4_unpack(alone, values)
        assert torch.equal(back[16 * t:16 * t + 16], values) and bool((values != 0).any())
