"""Orthogonalised updates of matrices of more than 2^32 values (16 x (2^28 + 40), both orientations): some 80 GB on the device."""
import pytest
import torch

import orthoref
import paper_2007_09835_b200 as rt3d

pytestmark = pytest.mark.gpu

N, L, STEP = 16, (1 << 28) + 40, 1 << 23


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("100 GB of free device memory wanted")
    yield
    torch.cuda.empty_cache()


def filled(shape, scale, dtype, seed):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 28):
        part = flat[at:at + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=gen, device="cuda") * scale)
    return out


def long_side(t, at):
    """A window of the long side, [N][up to STEP] in 64 bits."""
    return (t[:, at:at + STEP] if t.shape[0] == N else t[at:at + STEP].t()).double()


def polynomial(u):
    """Q of O(u) = Q u, from the small matrix in 64 bits."""
    gram = torch.zeros(N, N, dtype=torch.float64, device="cuda")
    for at in range(0, L, STEP):
        x = long_side(u, at)
        gram += x @ x.t()
    norm = gram.diagonal().sum().sqrt() + 1e-7
    gram, q = gram / norm ** 2, torch.eye(N, dtype=torch.float64, device="cuda") / norm
    for a, b, c in [orthoref.USUAL] * 5:
        p = a * torch.eye(N, dtype=torch.float64, device="cuda") + b * gram + c * gram @ gram
        gram, q = p @ gram @ p, p @ q
    return q


WINDOWS = [0, (1 << 27) - STEP // 2, (1 << 28) - STEP + 40]          # the last reaches the end, the middle one the place 2^31


@pytest.mark.parametrize("shape", [(N, L), (L, N)])
def test_directions(shape):
    g = filled(shape, 1e-3, torch.bfloat16, 1)
    out = torch.empty_like(g)
    ws = torch.empty(rt3d.rt3d_ortho_workspace(*shape), dtype=torch.uint8, device="cuda")
    rt3d.rt3d_orthogonalize(g, out, ws)
    torch.cuda.synchronize()
    assert rt3d.rt3d_last_device_status() == rt3d.OK
    q = polynomial(g)
    for at in WINDOWS:
        want = q @ long_side(g, at)
        assert (long_side(out, at) - want).norm() <= (2.0 ** -8 + 1e-4) * want.norm(), at


@pytest.mark.parametrize("shape", [(N, L), (L, N)])
def test_updates(shape):
    g = filled(shape, 1e-3, torch.bfloat16, 2)
    w, momentum = torch.zeros(shape, device="cuda"), torch.zeros(shape, device="cuda")
    ws = torch.empty(rt3d.rt3d_ortho_workspace(*shape), dtype=torch.uint8, device="cuda")
    rt3d.rt3d_ortho_update(w, momentum, g, None, ws, lr=1.0, momentum_factor=0.5, nesterov=True, scale=1.0)
    torch.cuda.synchronize()
    assert rt3d.rt3d_last_device_status() == rt3d.OK
    q = polynomial(g)                                # u = 1.5 g, whose direction is that of g but for eps
    for at in WINDOWS:
        x = long_side(g, at)
        assert torch.equal(long_side(momentum, at), x)
        assert (long_side(w, at) + q @ x).norm() <= 1e-4 * (q @ x).norm(), at
