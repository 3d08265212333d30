"""Orthogonalised updates on the GPU against the definition in 64 bits.

Tolerances, all of the Frobenius norm.  rt3d_orthogonalize rounds its result to bf16, at most 2^-8 of every value, and the matrix between
two runs of steps to fp16, 2^-12 of every value, which the steps left enlarge by at most 3.4445^2 where it lies in directions of
small singular values: 2^-12 * 11.9 = 2.9e-3 of |X|, and |X| there is at most |O| times the largest share of a value that has not
been enlarged yet: 3e-3 |O| covers it.  rt3d_ortho_update has 22 bits of every value and documents 1e-4 |O|."""
import math

import pytest
import torch

import orthoref
import paper_2007_09835_b200 as rt3d

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 300), (300, 1), (2, 3), (16, 16), (63, 65), (64, 576), (65, 64), (128, 128), (129, 127), (144, 576), (200, 2000), (576, 64),
         (1000, 130), (256, 256), (300, 517), (101, 4096), (640, 700)]


def workspace(m, k, fill=0xFF):
    return torch.full((rt3d.rt3d_ortho_workspace(m, k),), fill, dtype=torch.uint8, device="cuda")       # NaNs to whoever reads before writing


def orthogonalize(g, **kw):
    out = torch.full((g.shape[0], g[0].numel() + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    m, k = g.shape[0], g[0].numel()
    rt3d.rt3d_orthogonalize(g, out[:, :k], workspace(m, k), **kw)
    torch.cuda.synchronize()
    assert rt3d.rt3d_last_device_status() == rt3d.OK
    assert bool((out[:, k:] == 7).all())
    return out[:, :k]


def off(got, want):
    return ((got.double().cpu() - want.cpu()).norm() / want.norm()).item()


@pytest.mark.parametrize("m,k", SIZES)
@pytest.mark.parametrize("kind", ["noise", "falling", "steep"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_directions(m, k, kind, dtype):
    g = (orthoref.matrix(kind, m, k, m + k) * 1e-3).to(dtype)
    want = orthoref.direction(g)
    got = orthogonalize(g.cuda())
    assert off(got, want) <= 2.0 ** -8 + 3e-3
    assert (got.double().cpu() - want).abs().max() <= 0.05 * max(1e-30, want.square().mean().sqrt().item()) + 2.0 ** -8 * want.abs().max()


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 10, 16])
def test_numbers_of_steps(steps):
    g = orthoref.matrix("noise", 96, 200, steps).float()
    assert off(orthogonalize(g.cuda(), steps=steps), orthoref.direction(g, steps)) <= 2.0 ** -8 + 3e-3


@pytest.mark.parametrize("coefs", [[(1.5, -0.5, 0.0)] * 8, [(2.0, -1.5, 0.5)] * 6, [(1.875, -1.25, 0.375)] * 3,
                                   [(7.5, -21.0, 14.5), (2.0, -1.0, 0.17), (2.2, -1.6, 0.4), (1.875, -1.25, 0.375), (1.875, -1.25, 0.375)],
                                   [(0.0, 0.0, 0.0)], [(-1.0, 0.0, 0.0)], [(1.0, 0.0, 0.0)] * 16])
def test_other_coefficients(coefs):
    g = orthoref.matrix("falling", 80, 130, 5).float()
    want = orthoref.direction(g, len(coefs), coefs=coefs)
    got = orthogonalize(g.cuda(), steps=len(coefs), coefs=coefs)
    assert (got.double().cpu() - want).norm() <= (2.0 ** -8 + 3e-3) * want.norm()


def test_scales_of_the_gradient():
    g = orthoref.matrix("noise", 70, 90, 1).float()
    for scale in (1e-30, 1e-12, 1.0, 1e15, 1e36):
        u = g * scale
        assert off(orthogonalize(u.cuda()), orthoref.direction(u)) <= 2.0 ** -8 + 3e-3, scale
    assert bool((orthogonalize(torch.zeros(33, 70, device="cuda")) == 0).all())


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_gradient_that_is_no_number(value):
    g = torch.randn(100, 150, device="cuda")
    g[3, 77] = value
    assert bool(orthogonalize(g).isnan().all())


def test_a_matrix_of_rank_one_and_a_repeated_row():
    a, b = torch.randn(60, 1, dtype=torch.float64), torch.randn(1, 400, dtype=torch.float64)
    for g in ((a @ b).float(), torch.cat([b, b, 2 * b, torch.randn(3, 400, dtype=torch.float64)]).float()):
        # directions that are zero up to the rounding of g itself are enlarged like any other: 2^-24 * 485 and less
        assert off(orthogonalize(g.cuda()), orthoref.direction(g)) <= 2.0 ** -8 + 3e-3


def test_rows_with_a_pitch_and_convolution_weights():
    wide = torch.randn(40, 300, device="cuda")
    a = orthogonalize(wide[:, 50:250])
    b = orthogonalize(wide[:, 50:250].contiguous().view(40, 8, 1, 5, 5))
    assert torch.equal(a, b)
    odd = torch.randn(40 * 301 + 1, device="cuda").to(torch.bfloat16)[1:].view(40, 301)
    assert torch.equal(orthogonalize(odd[:, 3:204]), orthogonalize(odd[:, 3:204].contiguous()))


UPDATE = dict(lr=0.02, nesterov=True, weight_decay=0.1, scale=3.0)


def state(m, k, masked, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    w = torch.randn(m, k, generator=gen) * 0.05
    momentum = (orthoref.matrix("falling", m, k, seed + 1) * 0.1).float()
    g = (orthoref.matrix("noise", m, k, seed + 2) * 0.01).to(dtype)
    mask = None
    if masked:
        keep = torch.rand(-(-m // 4), -(-k // 4), generator=gen) < 0.4
        mask = keep.repeat_interleave(4, 0)[:m].repeat_interleave(4, 1)[:, :k].to(torch.uint8).contiguous() * 255
    return w, momentum, g, mask


def check_update(w, momentum, g, mask, mu=0.95, **kw):
    m, k = w.shape
    args = {**UPDATE, **kw}
    want_w, want_m, o = orthoref.update(w, momentum, g, mask, args["lr"], mu, args["nesterov"], args["weight_decay"], args["scale"])
    wd, md = w.cuda(), momentum.cuda()
    rt3d.rt3d_ortho_update(wd, md, g.cuda(), None if mask is None else mask.cuda(), workspace(m, k), momentum_factor=mu, **args)
    torch.cuda.synchronize()
    assert rt3d.rt3d_last_device_status() == rt3d.OK
    # momentum: one fused multiply-add; w: the same, on values of at most |w| and lr scale |o|, and the direction's own error
    assert ((md.double().cpu() - want_m).abs() <= 2.0 ** -23 * (momentum.double().abs() + g.double().abs()).where(torch.isfinite(momentum), torch.zeros_like(want_m))).all()
    step = args["lr"] * args["scale"]
    allowed = step * 1e-4 * o.norm() + 2.0 ** -22 * (torch.nan_to_num(w).double().norm() + step * o.norm())
    assert (wd.double().cpu() - want_w).norm() <= allowed
    if mask is not None:
        assert bool((wd.cpu()[mask == 0] == 0).all()) and bool((md.cpu()[mask == 0] == 0).all())
    return wd, md


@pytest.mark.parametrize("m,k", SIZES)
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_updates(m, k, masked, dtype):
    check_update(*state(m, k, masked, dtype, m + k))


def test_update_variants():
    s = state(100, 220, True, torch.float32)
    check_update(*s, nesterov=False)
    check_update(*s, mu=0.0)
    check_update(*s, weight_decay=0.0, scale=1.0, lr=1e-4)
    check_update(*s, lr=0.0)
    w, momentum, g, mask = s
    check_update(w, momentum, g, torch.zeros_like(mask))
    check_update(w, momentum, torch.zeros_like(g), mask)


def test_infinities_and_nans_in_masked_places_do_no_harm():
    w, momentum, g, mask = state(64, 128, True, torch.float32)
    hole = mask == 0
    w[hole], momentum[hole], g[hole] = float("inf"), float("nan"), float("-inf")
    wd, md = w.cuda(), momentum.cuda()
    clean = [t.clone().masked_fill(hole, 0).cuda() for t in (w, momentum, g)]
    rt3d.rt3d_ortho_update(wd, md, g.cuda(), mask.cuda(), workspace(64, 128), **UPDATE)
    rt3d.rt3d_ortho_update(clean[0], clean[1], clean[2], mask.cuda(), workspace(64, 128), **UPDATE)
    assert torch.equal(wd, clean[0]) and torch.equal(md, clean[1]) and bool(wd.isfinite().all())


def test_a_row_and_a_matrix_whose_mask_leaves_nothing():
    w, momentum, g, mask = state(65, 300, True, torch.bfloat16)
    mask[7] = 0
    mask[:, 11] = 0
    check_update(w, momentum, g, mask)


def test_the_same_bits_again_on_a_side_stream_and_from_a_graph():
    w, momentum, g, mask = (t.cuda() for t in state(150, 700, True, torch.bfloat16))
    ws = workspace(150, 700)

    def once(stream=None):
        a, b, out = w.clone(), momentum.clone(), torch.empty(150, 700, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        ctx = torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream())
        with ctx:
            rt3d.rt3d_ortho_update(a, b, g, mask, ws, **UPDATE)
            rt3d.rt3d_orthogonalize(g, out, ws)
        torch.cuda.synchronize()
        return a, b, out

    first = once()
    for other in (once(), once(torch.cuda.Stream())):
        assert all(torch.equal(p, q) for p, q in zip(first, other))
    a, b, out = w.clone(), momentum.clone(), torch.empty(150, 700, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rt3d.rt3d_ortho_update(a, b, g, mask, ws, **UPDATE)
        rt3d.rt3d_orthogonalize(g, out, ws)
    for _ in range(2):
        a.copy_(w), b.copy_(momentum), out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, first[0]) and torch.equal(b, first[1]) and torch.equal(out, first[2])


def test_a_larger_matrix_of_both_orientations():
    for m, k in ((1500, 2300), (2300, 1500)):
        g = (orthoref.matrix("noise", m, k, 9, "cuda") * 1e-3).to(torch.bfloat16)
        assert off(orthogonalize(g), orthoref.direction(g)) <= 2.0 ** -8 + 3e-3


def test_steps_bring_singular_values_near_one():
    g = orthoref.matrix("noise", 128, 1024, 4, "cuda").float()
    s = torch.linalg.svdvals(orthogonalize(g).double())
    assert 0.6 < s.min() and s.max() < 1.3
    assert math.isclose(s.square().sum().item(), 128, rel_tol=0.3)


def test_nothing_is_launched_while_planning():
    g, out = torch.randn(40, 50, device="cuda"), torch.empty(40, 50, dtype=torch.bfloat16, device="cuda")
    ws, before, allocs = workspace(40, 50), rt3d.rt3d_launch_count(), rt3d.rt3d_alloc_count()
    with rt3d.planning():
        rt3d.rt3d_orthogonalize(g, out, ws)
    assert rt3d.rt3d_launch_count() == before
    rt3d.rt3d_orthogonalize(g, out, ws)
    assert rt3d.rt3d_launch_count() > before and rt3d.rt3d_alloc_count() == allocs


def test_arrays_on_odd_addresses():
    w, momentum, g, mask = state(97, 300, True, torch.float32)

    def shifted(t, by):
        flat = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
        out = flat[by:].view(t.shape)
        out.copy_(t)
        return out

    want_w, want_m, o = orthoref.update(w, momentum, g, mask, UPDATE["lr"], 0.95, True, UPDATE["weight_decay"], UPDATE["scale"])
    step = UPDATE["lr"] * UPDATE["scale"] * o.norm()
    for by in ((1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1), (3, 2, 1, 7)):
        wd, md, gd, kd = (shifted(t, b) for t, b in zip((w, momentum, g, mask), by))
        rt3d.rt3d_ortho_update(wd, md, gd, kd, workspace(97, 300), **UPDATE)
        assert (wd.double().cpu() - want_w).norm() <= 1e-4 * step + 2.0 ** -22 * (w.double().norm() + step)
        assert (md.double().cpu() - want_m).norm() <= 2.0 ** -23 * (momentum.double().norm() + g.double().norm())


@pytest.mark.parametrize("m,k", [(3, 50000), (50000, 3), (130, 20000), (900, 1100), (1024, 1500), (1030, 1040)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_and_middling_matrices(m, k, dtype):
    gen = torch.Generator(device="cuda").manual_seed(m)
    g = (torch.randn(m, k, generator=gen, device="cuda") * 1e-3).to(dtype)
    assert off(orthogonalize(g), orthoref.direction(g)) <= 2.0 ** -8 + 3e-3


def test_two_calls_at_once():
    """Two streams with a workspace each: steps that wait for one another inside a launch, a cluster's and a grid's."""
    for m, k in ((144, 576), (512, 2048), (700, 900)):
        states = [[t.cuda() for t in state(m, k, True, torch.float32, seed)] for seed in (1, 2)]
        alone = []
        for w, momentum, g, mask in states:
            a, b = w.clone(), momentum.clone()
            for _ in range(4):
                rt3d.rt3d_ortho_update(a, b, g, mask, workspace(m, k), **UPDATE)
            alone.append((a, b))
        torch.cuda.synchronize()
        streams, spaces = [torch.cuda.Stream() for _ in states], [workspace(m, k) for _ in states]
        together = [(w.clone(), momentum.clone()) for w, momentum, _, _ in states]
        torch.cuda.synchronize()
        for _ in range(4):
            for st, ws, (a, b), (_, _, g, mask) in zip(streams, spaces, together, states):
                with torch.cuda.stream(st):
                    rt3d.rt3d_ortho_update(a, b, g, mask, ws, **UPDATE)
        torch.cuda.synchronize()
        assert rt3d.rt3d_last_device_status() == rt3d.OK
        assert all(torch.equal(p, q) for x, y in zip(alone, together) for p, q in zip(x, y))


def test_rows_that_share_memory_are_refused():
    row = torch.randn(1, 64, device="cuda")
    with pytest.raises(rt3d.Rt3dError):
        rt3d.rt3d_orthogonalize(row.expand(32, 64), torch.empty(32, 64, dtype=torch.bfloat16, device="cuda"), workspace(32, 64))
    with pytest.raises(ValueError):
        rt3d.rt3d_orthogonalize(torch.randn(64, 32, device="cuda").t(), torch.empty(32, 64, dtype=torch.bfloat16, device="cuda"), workspace(32, 64))


def test_poisoned_shared_memory():
    for m, k in ((20, 100), (144, 576), (300, 3000)):
        g = (orthoref.matrix("falling", m, k, 3) * 1e-3).to(torch.bfloat16)
        rt3d.rt3d_debug_set(rt3d.DEBUG_POISON, 0x7FC07FC0)
        assert off(orthogonalize(g.cuda()), orthoref.direction(g)) <= 2.0 ** -8 + 3e-3
