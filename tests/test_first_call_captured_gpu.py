"""The library's first calls of a process, captured into a graph: calls that allocate nothing leave a capture whole."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import sys
import torch
import paper_2007_09835_b200 as rt3d

torch.manual_seed(0)
w, g = torch.randn(200, 512, device="cuda"), torch.randn(200, 512, device="cuda")
x, y = torch.rand(ROWS, 1, 1, 1, 512, device="cuda").to(torch.bfloat16), torch.zeros(ROWS, 1, 1, 1, 200, device="cuda", dtype=torch.bfloat16)
q, out = rt3d.W4Weights(200, 512, 64), torch.zeros(200, 512, dtype=torch.bfloat16, device="cuda")
ws = torch.empty(rt3d.rt3d_ortho_workspace(200, 512), dtype=torch.uint8, device="cuda")
torch.cuda.synchronize()


def calls():
    rt3d.rt3d_w4_quantize(w, q)
    rt3d.rt3d_linear_w4(x, q, None, y)
    rt3d.rt3d_orthogonalize(g, out, ws)


graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
graph.replay()
torch.cuda.synchronize()
got = y.clone(), out.clone()
y.zero_(), out.zero_()
calls()
torch.cuda.synchronize()
assert all(bool((t != 0).any()) for t in got)
assert torch.equal(got[0], y) and torch.equal(got[1], out)
assert rt3d.rt3d_last_device_status() == rt3d.OK
print("replayed")
"""


@pytest.mark.parametrize("rows", [2, 40])
def test_first_calls_of_a_process_are_captured(rows):
    done = subprocess.run([sys.executable, "-c", PROGRAM.replace("ROWS", str(rows))], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "replayed" in done.stdout, done.stderr[-2000:]
