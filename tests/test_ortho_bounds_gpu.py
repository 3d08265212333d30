"""Directions within the bound of include/rt3d.h: tiny gradients, long sums, few directions, other numbers of steps and coefficients.

The bound.  A value in two fp16 parts is off by at most 2^-23 of itself: the first leaves at most 2^-11 of it, of which the second has
11 bits.  A product of two such values leaves out that of the second parts, 2^-22, and its result is held in two parts again:
2 2^-23 + 2^-22 + 2^-23 = 0.63 2^-20.  The tensor core cuts off what lies under the last bit of an accumulator, half a bit or 2^-24 of it
on average; in a sum of one sign, over 512 inputs in 96 additions, that is 96 2^-24 of half the sum, 3.0 2^-20.  Together under 2^-18 for
one product.  Of a step a X has one (P X), b A X two (A, P X), c A A X four (A twice, A A, P X).  The later steps enlarge what that
leaves by their largest |a + b s + c s s| where it lies in directions of small singular values.  So, of the Frobenius norm,
2^-18 S max(|O|, |X|), S the sum over the steps of (|a| + 2 |b| + 4 |c|) times the later steps' largest |p|, |X| = |u| / (|u| + eps).
"""
import numpy as np
import pytest
import torch

import orthoref
import paper_2007_09835_b200 as rt3d

pytestmark = pytest.mark.gpu


def enlargement(steps, coefs=None):
    """S of the bound."""
    coefs = [orthoref.USUAL] * steps if coefs is None else coefs
    top, most = 1.0, []
    for a, b, c in coefs:
        s = np.linspace(0, top, 20001)
        p = a + b * s ** 2 + c * s ** 4
        most.append(np.abs(p).max())
        top = np.abs(s * p).max()
    return sum((abs(a) + 2 * abs(b) + 4 * abs(c)) * np.prod(most[i + 1:]) for i, (a, b, c) in enumerate(coefs))


def allowed(o, u, steps=5, coefs=None, eps=1e-7):
    norm = u.double().norm().item()
    return 2.0 ** -18 * enlargement(steps, coefs) * max(o.norm().item(), norm / (norm + eps))


def workspace(m, k):
    return torch.full((rt3d.rt3d_ortho_workspace(m, k),), 0xFF, dtype=torch.uint8, device="cuda")


def fp32_direction(u, **kw):
    """O(u) as an update of weights of zero leaves it."""
    w, momentum = torch.zeros(u.shape, device="cuda"), torch.zeros(u.shape, device="cuda")
    rt3d.rt3d_ortho_update(w, momentum, u, None, workspace(*u.shape), lr=1.0, momentum_factor=0.0, nesterov=False, weight_decay=0.0, scale=1.0, **kw)
    torch.cuda.synchronize()
    assert rt3d.rt3d_last_device_status() == rt3d.OK
    return -w


def check(u, steps=5, coefs=None, few=False):
    """`few`: directions of u are zero but for rounding, of u itself too, and no bound but the general one holds."""
    got = fp32_direction(u, steps=steps, coefs=coefs).double()
    want = orthoref.direction(u, steps, coefs=coefs)
    off, most = (got - want).norm().item(), allowed(want, u, steps, coefs)
    if steps <= 5 and coefs is None and not few:
        most = min(most, 1e-4 * want.norm().item())                  # what the usual five steps are documented to keep
    assert off <= most, (off, most, want.norm().item())


def noise(m, k, seed=0):
    return torch.randn(m, k, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def of_rank(rank, m, k, seed=0):
    return (noise(m, rank, seed).double() @ noise(rank, k, seed + 1).double()).float()


# ------------------------------------------------------------------------------------------- gradients next to eps, and shrinking steps
@pytest.mark.parametrize("scale", [1e-6, 1e-12, 1e-18, 1e-24, 1e-30])
@pytest.mark.parametrize("m,k", [(512, 1000), (70, 90), (90, 70), (130, 3000)])
def test_tiny_gradients(m, k, scale):
    check(noise(m, k) * scale)


@pytest.mark.parametrize("steps", [1, 8, 10, 16])
@pytest.mark.parametrize("scale", [1e-10, 1e-20, 1e-30])
def test_tiny_gradients_and_numbers_of_steps(steps, scale):
    for m, k in ((70, 90), (512, 1000), (65, 2000)):
        check(noise(m, k) * scale, steps)
        out = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
        u = noise(m, k) * scale
        rt3d.rt3d_orthogonalize(u, out, workspace(m, k), steps=steps)
        want = orthoref.direction(u, steps)
        assert (out.double() - want).norm() <= 2.0 ** -8 * want.norm() + allowed(want, u, steps)


@pytest.mark.parametrize("coefs", [[(0.25, 0.0, 0.0)] * 12, [(0.1, -0.1, 0.05)] * 6, [(0.01, 0.0, 0.0), (1.9, 0.0, 0.0), (3.0, -1.0, 0.1)], [(1.5, -0.5, 0.0)] * 7,
                                   [(0.5, 0.0, 0.0)] * 3 + [(3.4, 0.0, 0.0)] * 2])
@pytest.mark.parametrize("scale", [1.0, 1e-8, 1e-20])
def test_steps_that_shrink(coefs, scale):
    for m, k in ((70, 90), (65, 2000)):
        u = noise(m, k) * scale
        got = fp32_direction(u, steps=len(coefs), coefs=coefs).double()
        want = orthoref.direction(u, len(coefs), coefs=coefs)
        # no direction is small beside the others here: every step's 2^-21 of its own, and the fp32 result's rounding
        assert (got - want).norm() <= (len(coefs) + 1) * 2.0 ** -21 * want.norm(), ((got - want).norm() / want.norm()).item()


# --------------------------------------------------------------------------------------------------------------------- long sums
@pytest.mark.parametrize("m,k", [(1536, 65536), (65536, 1536), (64, 1 << 18), (1 << 18, 64), (130, 1 << 18), (1100, 4096), (2100, 1300), (1500, 20000)])
def test_long_sums(m, k):
    check(noise(m, k, m) * 1e-3)
    if m * k <= 1 << 25:
        check(noise(m, k, m).abs() * 1e-3)           # of one sign


# ------------------------------------------------------------------------------------ few directions, numbers of steps, coefficients
@pytest.mark.parametrize("steps", [1, 2, 3, 5, 7, 10, 16])
@pytest.mark.parametrize("rank,m,k", [(1, 60, 400), (16, 256, 1500), (3, 1300, 200), (40, 300, 5000), (5, 1100, 1200), (2, 2000, 3000)])
def test_few_directions(rank, m, k, steps):
    check(of_rank(rank, m, k), steps, few=True)


@pytest.mark.parametrize("coefs", [[(1.5, -0.5, 0.0)] * 8, [(2.0, -1.5, 0.5)] * 6, [(1.875, -1.25, 0.375)] * 3, [(-1.0, 0.0, 0.0)], [(1.0, 0.0, 0.0)] * 16,
                                   [(7.5, -21.0, 14.5), (2.0, -1.0, 0.17), (2.2, -1.6, 0.4), (1.875, -1.25, 0.375), (1.875, -1.25, 0.375)], [(1.0, -1.0, 0.0)] * 2])
@pytest.mark.parametrize("rank,m,k", [(1, 60, 400), (16, 256, 1500), (60, 80, 60)])
def test_other_coefficients(coefs, rank, m, k):
    check(of_rank(rank, m, k), len(coefs), coefs)


# ----------------------------------------------------------------------------------------------- bf16 results are the fp32 ones, rounded
@pytest.mark.parametrize("m,k", [(64, 576), (129, 127), (300, 517), (512, 4096), (1300, 1100), (130, 20000)])
def test_directions_are_rounded_once(m, k):
    u = (orthoref.matrix("falling", m, k, 3) * 1e-3).float().cuda()
    out = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
    rt3d.rt3d_orthogonalize(u, out, workspace(m, k))
    assert torch.equal(out, fp32_direction(u).to(torch.bfloat16))


@pytest.mark.parametrize("m,k", [(329, 283), (366, 2759), (2003, 1357)])
def test_one_step_on_values_of_one_sign(m, k):
    """Where a step enlarges nothing, what the sums cut off is the most of it."""
    for coefs in ([(0.3, 0.2, 0.1)], [(1.5, -0.5, 0.0)]):
        check(noise(m, k).abs(), 1, coefs)
