"""4-bit weights on the GPU against numpy: codes and scales bit for bit, products in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2007_09835_b200 as rt3d
import w4ref

pytestmark = pytest.mark.gpu


def make_weights(m, k, seed, kind="normal"):
    rng = np.random.default_rng(seed)
    w = (rng.standard_normal((m, k)) * 0.05).astype(np.float32)
    if kind == "edges":                     # groups of zeros, of one sign, of tiny and of huge values, ties
        w[0] = 0
        w[1 % m] = np.abs(w[1 % m])
        w[2 % m] = -np.abs(w[2 % m])
        w[3 % m] *= np.float32(1e-38)
        w[4 % m] *= np.float32(1e38)
        w[5 % m] = np.float32(0.5) * rng.integers(-14, 15, k)
        w[6 % m] = np.float32(1e-44)
    return w


def quantized(w, group, zeros, dtype=torch.float32):
    wd = torch.from_numpy(w).cuda().to(dtype)
    q = rt3d.W4Weights(*w.shape, group, zeros=zeros)
    for t in (q.codes, q.scales, q.zeros):
        if t is not None:
            t.view(torch.uint8).fill_(0xA5)
    rt3d.rt3d_w4_quantize(wd, q)
    return wd, q


def reference(wd, group, zeros):
    w = wd.float().cpu().numpy()
    codes, scales, zero = w4ref.quantize(w, group, zeros)
    return w, codes, scales, zero


@pytest.mark.parametrize("m,k", [(1, 1), (1, 8273), (16, 64), (17, 65), (15, 31), (33, 100), (101, 4096), (64, 2048), (130, 129), (7, 96)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype,kind", [(torch.float32, "normal"), (torch.bfloat16, "normal"), (torch.float32, "edges")])
def test_codes_scales_and_zero_points(m, k, group, zeros, dtype, kind):
    wd, q = quantized(make_weights(m, k, m + k + group, kind), group, zeros, dtype)
    w, codes, scales, zero = reference(wd, group, zeros)
    np.testing.assert_array_equal(q.scales.float().cpu().numpy(), w4ref.tiled(scales))
    if zeros:
        np.testing.assert_array_equal(q.zeros.cpu().numpy(), w4ref.tiled(zero))
    spread = np.repeat(zero, group, 1)
    fill = np.repeat(zero[:, -1:], -(-k // 64) * 64, 1)
    fill[:, :min(fill.shape[1], spread.shape[1])] = spread[:, :fill.shape[1]]
    np.testing.assert_array_equal(q.codes.cpu().numpy(), w4ref.laid_out(codes, fill))
    for out_dtype in (torch.float32, torch.bfloat16):
        out = torch.full((m, k + 3), 7.0, dtype=out_dtype, device="cuda")
        rt3d.rt3d_w4_unpack(q, out[:, :k])
        want = torch.from_numpy(w4ref.values(codes, scales, zero, group).astype(np.float32)).to(out_dtype)
        assert torch.equal(out[:, :k].cpu(), want) and bool((out[:, k:] == 7).all())


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("zeros", [False, True])
def test_a_group_with_a_value_that_is_no_number(value, zeros):
    w = make_weights(20, 200, 3)
    w[18, 70] = value
    wd, q = quantized(w, 64, zeros)
    out = torch.empty_like(wd)
    rt3d.rt3d_w4_unpack(q, out)
    bad = torch.zeros_like(wd, dtype=torch.bool)
    bad[18, 64:128] = True
    assert torch.equal(out.isnan(), bad)
    x = torch.rand(3, 1, 1, 1, 200, device="cuda")
    y = torch.zeros(3, 1, 1, 1, 20, device="cuda")
    rt3d.rt3d_linear_w4(x, q, None, y)
    rows = y.view(3, 20).isnan()
    assert bool(rows[:, 18].all()) and not bool(rows[:, :18].any()) and not bool(rows[:, 19:].any())


def test_rows_with_a_pitch_and_convolution_weights():
    wide = torch.randn(40, 300, device="cuda")
    a, b = rt3d.W4Weights(40, 200, 32), rt3d.W4Weights(40, 200, 32)
    rt3d.rt3d_w4_quantize(wide[:, 50:250], a)
    rt3d.rt3d_w4_quantize(wide[:, 50:250].contiguous().view(40, 8, 1, 5, 5), b)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    odd = torch.empty(40 * 301 + 1, device="cuda", dtype=torch.bfloat16)[1:].view(40, 301)
    odd.copy_(torch.randn(40, 301, device="cuda"))
    c, d = rt3d.W4Weights(40, 201, 128, zeros=True), rt3d.W4Weights(40, 201, 128, zeros=True)
    rt3d.rt3d_w4_quantize(odd[:, 7:208], c)
    rt3d.rt3d_w4_quantize(odd[:, 7:208].contiguous(), d)
    assert torch.equal(c.codes, d.codes) and torch.equal(c.scales, d.scales) and torch.equal(c.zeros, d.zeros)


def run_linear(rows, m, k, group, zeros, dtype, relu, bias, seed=0, lead=(1, 1, 1), sign=False):
    rng = np.random.default_rng(seed + rows + m + k)
    w = make_weights(m, k, seed + 1)
    if sign:
        w = np.abs(w)
    wd, q = quantized(w, group, zeros)
    _, codes, scales, zero = reference(wd, group, zeros)
    unit = 8 if dtype == torch.bfloat16 else 4
    xp, yp = -(-k // unit) * unit + unit, -(-m // unit) * unit + unit
    x = torch.full((rows,) + lead + (xp,), float("nan"), dtype=dtype, device="cuda")      # behind the last channel: NaN
    xs = rng.uniform(0 if sign else -1, 1, (int(np.prod((rows,) + lead)), k)).astype(np.float32)
    x[..., :k] = torch.from_numpy(xs).view((rows,) + lead + (k,)).cuda()
    y = torch.full((rows,) + lead + (yp,), 7.0, dtype=dtype, device="cuda")
    b = torch.from_numpy((rng.standard_normal(m) * 0.1).astype(np.float32)).cuda() if bias else None
    rt3d.rt3d_linear_w4(rt3d.tensor_desc(x, k), q, b, rt3d.tensor_desc(y, m), relu=relu)
    xs = x[..., :k].float().cpu().numpy().reshape(-1, k)
    want, size = w4ref.linear(xs, w4ref.values(codes, scales, zero, group), None if b is None else b.cpu().numpy().astype(np.float64), relu)
    got = y[..., :m].float().cpu().numpy().reshape(-1, m).astype(np.float64)
    tol = w4ref.tolerance(size, k, group)
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    worst = (np.abs(got - want) / tol).max()
    assert worst <= 1, worst
    assert bool((y[..., m:] == 7).all())
    return x, q, b, y


ROWS = [1, 2, 3, 7, 8, 9, 16, 17, 31, 33, 64, 65, 130]


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_products_of_few_rows(rows, group, dtype):
    run_linear(rows, 101, 1000, group, rows % 2 == 0, dtype, rows % 3 == 0, True)


@pytest.mark.parametrize("m,k", [(1, 1), (1, 64), (5, 7), (16, 33), (487, 4096), (4096, 512), (33, 16384), (200, 63), (64, 8200), (1000, 129)])
@pytest.mark.parametrize("rows", [1, 5, 20, 150])
@pytest.mark.parametrize("dtype,zeros", [(torch.bfloat16, False), (torch.bfloat16, True), (torch.float32, True)])
def test_products_of_odd_extents(m, k, rows, dtype, zeros):
    run_linear(rows, m, k, 128 if k % 3 else 32, zeros, dtype, m % 2 == 1, m % 3 != 0, sign=k == 8200)


def test_every_voxel_is_a_row():
    run_linear(3, 40, 72, 32, True, torch.bfloat16, True, True, lead=(2, 3, 5))


def test_many_rows():
    run_linear(5000, 48, 160, 64, True, torch.bfloat16, False, True)


def test_more_rows_than_a_launch_takes():
    rows, m, k = (1 << 19) + 5, 8, 64
    wd, q = quantized(make_weights(m, k, 1), 32, True)
    _, codes, scales, zero = reference(wd, 32, True)
    values = torch.from_numpy(w4ref.values(codes, scales, zero, 32)).cuda()
    for dtype in (torch.bfloat16, torch.float32):
        x = (torch.rand(rows, 1, 1, 1, k, device="cuda") * 2 - 1).to(dtype)
        y = torch.zeros(rows, 1, 1, 1, m, dtype=dtype, device="cuda")
        rt3d.rt3d_linear_w4(x, q, None, y)
        want, size = x.view(rows, k).double() @ values.t(), x.view(rows, k).abs().double() @ values.abs().t()
        tol = w4ref.tolerance(size, k, 32)
        if dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * (want.abs() + tol)
        assert bool(((y.view(rows, m).double() - want).abs() <= tol).all())


def test_the_same_bits_again_on_a_side_stream_and_from_a_graph():
    x, q, b, y = run_linear(4, 300, 2048, 128, True, torch.bfloat16, True, True)
    first = y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y.fill_(1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rt3d.rt3d_linear_w4(rt3d.tensor_desc(x, q.k), q, b, rt3d.tensor_desc(y, q.m), relu=True)
    side.synchronize()
    assert torch.equal(y[..., :q.m], first[..., :q.m])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rt3d.rt3d_linear_w4(rt3d.tensor_desc(x, q.k), q, b, rt3d.tensor_desc(y, q.m), relu=True)
    for scale in (1.0, 2.0):
        x[..., :q.k] *= scale
        y.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        again = torch.empty_like(y)
        rt3d.rt3d_linear_w4(rt3d.tensor_desc(x, q.k), q, b, rt3d.tensor_desc(again, q.m), relu=True)
        assert torch.equal(y[..., :q.m], again[..., :q.m])


def test_infinities_and_nans_of_a_row_stay_in_it():
    x, q, b, y = run_linear(9, 70, 256, 64, True, torch.float32, False, True)
    x[4, ..., 100] = float("nan")
    x[6, ..., 3] = float("inf")
    rt3d.rt3d_linear_w4(rt3d.tensor_desc(x, q.k), q, b, rt3d.tensor_desc(y, q.m))
    fine = y[..., :q.m].isfinite().view(9, -1)
    assert not bool(fine[4].any())
    assert bool(fine[[0, 1, 2, 3, 5, 7, 8]].all())


def test_nothing_is_allocated_or_launched_while_planning():
    x, q, b, y = run_linear(2, 33, 64, 64, False, torch.bfloat16, False, True)
    before, allocs = rt3d.rt3d_launch_count(), rt3d.rt3d_alloc_count()
    with rt3d.planning():
        rt3d.rt3d_linear_w4(rt3d.tensor_desc(x, q.k), q, b, rt3d.tensor_desc(y, q.m))
    assert rt3d.rt3d_launch_count() == before
    rt3d.rt3d_linear_w4(rt3d.tensor_desc(x, q.k), q, b, rt3d.tensor_desc(y, q.m))
    assert rt3d.rt3d_launch_count() > before and rt3d.rt3d_alloc_count() == allocs


@pytest.mark.parametrize("rows", [2, 20])
def test_codes_past_32_bits(rows):
    """5.2 billion weights, 2.6 GB of codes: the last tile's filters against the same tile on its own, in 64 bits."""
    m, k, group = 40000, 131072, 64
    q = rt3d.W4Weights(m, k, group, zeros=True)
    q.codes.view(torch.int64).random_()
    q.scales.copy_(torch.rand(q.scales.shape, device="cuda") * 0.01)
    q.zeros.copy_(torch.randint(0, 16, q.zeros.shape, device="cuda"))
    x = (torch.rand(rows, 1, 1, 1, k, device="cuda") * 2 - 1).to(torch.bfloat16)
    y = torch.zeros(rows, 1, 1, 1, m, dtype=torch.bfloat16, device="cuda")
    rt3d.rt3d_linear_w4(x, q, None, y)
    last = rt3d.W4Weights(16, k, group, codes=q.codes[-16 * k // 2:].clone(), scales=q.scales[-1:].clone(), zeros=q.zeros[-1:].clone())
    values = torch.empty(16, k, device="cuda")
    rt3d.rt3d_w4_unpack(last, values)
    xs = x.view(rows, k).double()
    want, size = xs @ values.double().t(), xs.abs() @ values.double().abs().t()
    tol = w4ref.tolerance(size, k, group)
    tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert bool(((y.view(rows, m)[:, -16:].double() - want).abs() <= tol).all())


def test_two_streams_at_once():
    parts = [run_linear(rows, 300, 4096, 64, True, torch.bfloat16, True, True, seed=rows) for rows in (3, 70)]
    want = [p[3].clone() for p in parts]
    streams = [torch.cuda.Stream() for _ in parts]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, (x, q, b, y) in zip(streams, parts):
            with torch.cuda.stream(st):
                rt3d.rt3d_linear_w4(rt3d.tensor_desc(x, q.k), q, b, rt3d.tensor_desc(y, q.m), relu=True)
    torch.cuda.synchronize()
    assert rt3d.rt3d_last_device_status() == rt3d.OK
    assert all(torch.equal(p[3], w) for p, w in zip(parts, want))


def test_shared_and_poisoned_memory():
    """Products after every SM's shared and tensor memory has been filled with NaNs."""
    for rows, dtype in ((1, torch.bfloat16), (12, torch.float32), (40, torch.bfloat16), (100, torch.bfloat16), (40, torch.float32)):
        rt3d.rt3d_debug_set(rt3d.DEBUG_POISON, 0x7FC07FC0)
        run_linear(rows, 45, 200, 32, True, dtype, False, True)
        rt3d.rt3d_debug_set(rt3d.DEBUG_POISON, 0x7FC07FC0)
        run_linear(rows, 200, 130, 128, False, dtype, False, True)


def test_matrices_that_are_refused():
    q = rt3d.W4Weights(40, 200, 32)
    for w in (torch.zeros(40, 199, device="cuda"), torch.zeros(39, 200, device="cuda"), torch.zeros(200, 40, device="cuda").t(), torch.zeros(8000, device="cuda"),
              torch.zeros(40, 200, device="cuda", dtype=torch.float16), torch.zeros(40, 400, device="cuda")[:, ::2], torch.zeros(40, 8, 1, 5, 6, device="cuda")):
        for call in (lambda: rt3d.rt3d_w4_quantize(w, q), lambda: rt3d.rt3d_w4_unpack(q, w)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(rt3d.Rt3dError) as e:
        rt3d.rt3d_w4_quantize(torch.zeros(1, 200, device="cuda").expand(40, 200), q)         # rows that share memory
    assert e.value.status == rt3d.ERR_INVALID_ARG
    with pytest.raises((TypeError, AttributeError, ValueError)):
        rt3d.rt3d_w4_quantize(np.zeros((40, 200), np.float32), q)
