"""Measured cases of the weight operators: 4-bit weights and orthogonalised updates, each in its plain form and as the
library's calls.

A case is a dict of plain values.  Its "op" says which operator a pass runs:

  quantize  weights [M][K] to 4-bit codes with a scale (and, where "zeros", a zero point) for every `group` inputs of a
            filter, and back to the values the codes stand for: what a user runs to see what the quantisation costs
  linear    y = act(x W^T + b) on `rows` rows of activations with such 4-bit weights: the fully connected layers behind a
            network's convolutions
  ortho     a matrix's orthogonalised direction, by Newton-Schulz steps
  update    one optimiser step of a layer's weights: momentum, the orthogonalised direction, weight decay and the pruning
            mask

Layout of 4-bit weights (include/rt3d.h): tiles of 16 filters x 64 inputs, 32 units of 16 bytes; unit 4 g + t holds, for
the filters g and g + 8 and the two halves of 32 inputs, the inputs 8 t .. 8 t + 7 as a 32-bit word, input e of them at bits
4 ((e >> 1) + 4 (e & 1)).  Scales and zero points: [tile of 16 filters][group][16].
"""
import math

import torch

own = False

COEF = (3.4445, -4.7750, 2.0315)        # of the quintic step X <- a X + (b A + c A A) X, A = X X^T
EPS = 1e-7
LR, MU, DECAY = 1e-3, 0.95, 0.1         # learning rate, momentum and weight decay of the measured updates
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # the classifier of a C3D-shaped network on 487 classes (odd filter count), quantised on its own with zero points
        {"name": "quantize_fc8", "op": "quantize", "m": 487, "k": 4096, "group": 32, "zeros": True, "dtype": "fp32"},
        # the first fully connected layer of a C3D-shaped network, the largest of its weights
        {"name": "quantize_fc6", "op": "quantize", "m": 4096, "k": 8192, "group": 128, "zeros": False, "dtype": "fp32"},
        # one clip through the classifier: the smallest call, where latency counts
        {"name": "linear_fc8_1", "op": "linear", "rows": 1, "m": 487, "k": 4096, "group": 128, "zeros": False, "dtype": "bf16", "relu": False},
        # one clip through the first fully connected layer
        {"name": "linear_fc6_1", "op": "linear", "rows": 1, "m": 4096, "k": 8192, "group": 128, "zeros": False, "dtype": "bf16", "relu": True},
        # a few clips through a layer whose codes (134 MB) do not stay in the L2
        {"name": "linear_wide_4", "op": "linear", "rows": 4, "m": 16384, "k": 16384, "group": 64, "zeros": True, "dtype": "bf16", "relu": False},
        # fp32 activations, a small batch, the finest groups
        {"name": "linear_fc6_fp32_13", "op": "linear", "rows": 13, "m": 4096, "k": 8192, "group": 32, "zeros": True, "dtype": "fp32", "relu": True},
        # a large batch of clips
        {"name": "linear_fc6_256", "op": "linear", "rows": 256, "m": 4096, "k": 8192, "group": 128, "zeros": False, "dtype": "bf16", "relu": True},
        # the gradient of a thin 1x3x3 layer (64 filters, 64 channels)
        {"name": "ortho_thin", "op": "ortho", "m": 64, "k": 576, "dtype": "bf16"},
        # a late 3x3x3 layer of a C3D-shaped network (512 filters, 512 channels)
        {"name": "ortho_conv5", "op": "ortho", "m": 512, "k": 13824, "dtype": "bf16"},
        # the first fully connected layer of a C3D-shaped network
        {"name": "ortho_fc6", "op": "ortho", "m": 4096, "k": 8192, "dtype": "bf16"},
        # a spatial layer of the first stage of an R(2+1)D-shaped network, pruned
        {"name": "update_stage1", "op": "update", "m": 144, "k": 576, "dtype": "fp32", "mask": True},
        # the second 3x3x3 layer of a C3D-shaped network (256 filters, 256 channels), pruned, bf16 gradients
        {"name": "update_conv3b", "op": "update", "m": 256, "k": 6912, "dtype": "bf16", "mask": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "ortho", "update"])
    if op == "quantize":
        k = _log(rng, 16, 16384)
        return {"op": op, "m": _log(rng, 1, min(16384, (1 << 25) // k)), "k": k, "group": rng.choice([32, 64, 128]), "zeros": rng.random() < 0.5,
                "dtype": rng.choice(["fp32", "bf16"])}
    if op == "linear":
        rows = _log(rng, 1, 512)
        k = _log(rng, 64, 16384)
        m = _log(rng, 8, 16384)
        if rows * k * m > 1 << 33:
            m = max(8, (1 << 33) // (rows * k))
        return {"op": op, "rows": rows, "m": m, "k": k, "group": rng.choice([32, 64, 128]), "zeros": rng.random() < 0.5,
                "dtype": rng.choice(["bf16", "bf16", "fp32"]), "relu": rng.random() < 0.5}
    m = _log(rng, 16, 2048)
    k = _log(rng, 32, min(16384, (1 << 24) // m))
    if op == "ortho":
        return {"op": op, "m": m, "k": k, "dtype": rng.choice(["bf16", "bf16", "fp32"])}
    return {"op": op, "m": m, "k": k, "dtype": rng.choice(["fp32", "bf16"]), "mask": rng.random() < 0.7}


# ------------------------------------------------------------------------------------------------------------ inputs
def _gradient(gen, m, k):
    """A gradient of a layer's weights: a few strong directions that fall off, and noise."""
    rank = min(16, m, k)
    left = torch.randn(m, rank, generator=gen, device="cuda") / (1.0 + torch.arange(rank, device="cuda"))
    right = torch.randn(rank, k, generator=gen, device="cuda")
    return 1e-3 * (left @ right) + 2e-4 * torch.randn(m, k, generator=gen, device="cuda")


def _pitch(c, dtype):
    unit = 8 if dtype == torch.bfloat16 else 4
    return -(-c // unit) * unit


def _laid_out(codes, m, k):
    """[M][K] codes -> the tile layout, as bytes; places beyond the weights hold 8."""
    mt, kb = -(-m // 16), -(-k // 64)
    full = torch.full((mt * 16, kb * 64), 8, dtype=torch.int32, device=codes.device)
    full[:m, :k] = codes
    v = full.view(mt, 2, 8, kb, 2, 4, 4, 2)                                     # tile, h, g, block, half, t, e >> 1, e & 1
    shift = 4 * (torch.arange(4, device=codes.device)[:, None] + 4 * torch.arange(2, device=codes.device))
    words = (v.to(torch.int64) << shift).sum(dim=(-1, -2))                      # tile, h, g, block, half, t
    words = words.permute(0, 3, 2, 5, 4, 1).contiguous()                        # tile, block, g, t, half, h
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).view(torch.uint8).view(-1)


def _tiled(per_filter, m):
    """[M][groups] -> [tile][groups][16], zeros beyond the filters."""
    mt, g = -(-m // 16), per_filter.shape[1]
    full = torch.zeros(mt * 16, g, dtype=per_filter.dtype, device=per_filter.device)
    full[:m] = per_filter
    return full.view(mt, 16, g).transpose(1, 2).contiguous()


def _untiled(tiled, m):
    return tiled.transpose(1, 2).reshape(-1, tiled.shape[1])[:m]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    m, k, dtype = case["m"], case["k"], DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if case["op"] == "quantize":
        g, mt = -(-k // case["group"]), -(-m // 16)
        s["w"] = (0.05 * torch.randn(m, k, generator=gen, device="cuda")).to(dtype)
        s["codes"] = torch.empty(mt * -(-k // 64) * 512, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(mt, g, 16, dtype=torch.bfloat16, device="cuda")
        s["zeros"] = torch.empty(mt, g, 16, dtype=torch.uint8, device="cuda") if case["zeros"] else None
        s["values"] = torch.empty(m, k, device="cuda")
    elif case["op"] == "linear":
        rows, g = case["rows"], -(-k // case["group"])
        codes = torch.randint(0, 16, (m, k), generator=gen, device="cuda", dtype=torch.uint8)
        scales = (0.005 * (1.0 + torch.rand(m, g, generator=gen, device="cuda"))).to(torch.bfloat16)
        s["plain_codes"] = codes
        s["codes"] = _laid_out(codes, m, k)
        s["scales"] = _tiled(scales, m)
        s["zeros"] = _tiled(torch.randint(5, 11, (m, g), generator=gen, device="cuda", dtype=torch.uint8), m) if case["zeros"] else None
        s["bias"] = 0.01 * torch.randn(m, generator=gen, device="cuda")
        s["x"] = torch.zeros(rows, 1, 1, 1, _pitch(k, dtype), dtype=dtype, device="cuda")
        s["x"][..., :k] = torch.rand(rows, 1, 1, 1, k, generator=gen, device="cuda") * 2 - 1
        s["y"] = torch.zeros(rows, 1, 1, 1, _pitch(m, dtype), dtype=dtype, device="cuda")
    elif case["op"] == "ortho":
        s["g"] = _gradient(gen, m, k).to(dtype)
        s["out"] = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
    else:
        s["g"] = _gradient(gen, m, k).to(dtype)
        s["momentum"] = 10 * _gradient(gen, m, k)
        s["w"] = 0.05 * torch.randn(m, k, generator=gen, device="cuda")
        s["mask"] = None
        if case["mask"]:                                                        # 4 x 4 kernel groups, 40 % of the places kept
            keep = torch.rand(-(-m // 4), -(-k // 4), generator=gen, device="cuda") < 0.4
            s["mask"] = keep.repeat_interleave(4, 0)[:m].repeat_interleave(4, 1)[:, :k].to(torch.uint8).contiguous()
            s["momentum"] *= s["mask"]
            s["w"] *= s["mask"]
    return s


# ------------------------------------------------------------------------------------------------------ the plain form
def _spread(per_group, group, k):
    return per_group.repeat_interleave(group, 1)[:, :k]


def _quantize_plain(w, group, zeros):
    m, k = w.shape
    g = -(-k // group)
    full = torch.zeros(m, g * group, device=w.device)
    full[:, :k] = w.float()
    v = full.view(m, g, group)
    if zeros:
        low, high = v.amin(2).clamp(max=0), v.amax(2).clamp(min=0)
        scale = ((high - low) / torch.full_like(low, 15)).to(torch.bfloat16)
        s = scale.float()
        zero = torch.where(s > 0, torch.round(-low / s).clamp(0, 15), torch.full_like(s, 8))
    else:
        high = v.abs().amax(2)
        scale = (high / torch.full_like(high, 7)).to(torch.bfloat16)
        s = scale.float()
        zero = torch.full_like(s, 8)
    code = torch.where(s[..., None] > 0, (torch.round(v / s[..., None]) + zero[..., None]).clamp(0, 15), zero[..., None])
    return code.view(m, g * group)[:, :k], scale, zero


def _steps_plain(u, steps=5):
    a, b, c = COEF
    tall = u.shape[0] > u.shape[1]
    x = u.t() if tall else u
    x = x / (x.norm() + EPS)
    for _ in range(steps):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if tall else x


def _linear_plain(s):
    c = s["case"]
    m, k = c["m"], c["k"]
    zero = 8.0 if s["zeros"] is None else _spread(_untiled(s["zeros"], m).float(), c["group"], k)
    w = (s["plain_codes"].float() - zero) * _spread(_untiled(s["scales"], m).float(), c["group"], k)
    y = s["x"].view(c["rows"], -1)[:, :k].float() @ w.t() + s["bias"]
    return (y.clamp(min=0) if c["relu"] else y).to(s["x"].dtype)


def _update_plain(s):
    c = s["case"]
    g = s["g"].float()
    keep = None if s["mask"] is None else s["mask"] != 0
    momentum = MU * s["momentum"] + g
    if keep is not None:
        g, momentum = torch.where(keep, g, 0.0), torch.where(keep, momentum, 0.0)
    o = _steps_plain(g + MU * momentum)
    w = (1 - LR * DECAY) * s["w"] - LR * _scale(c) * o
    s["momentum"].copy_(momentum)
    s["w"].copy_(w if keep is None else torch.where(keep, w, 0.0))
    return {"w": s["w"], "momentum": s["momentum"]}


def _scale(c):
    return 0.2 * math.sqrt(max(c["m"], c["k"]))


def _run_plain(s):
    c = s["case"]
    if c["op"] == "quantize":
        code, scale, zero = _quantize_plain(s["w"], c["group"], c["zeros"])
        m, k = code.shape
        out = {"scales": _tiled(scale, m), "values": (code - _spread(zero, c["group"], k)) * _spread(scale.float(), c["group"], k)}
        if c["zeros"]:
            out["zeros"] = _tiled(zero.to(torch.uint8), m)
        return out
    if c["op"] == "linear":
        return _linear_plain(s)
    if c["op"] == "ortho":
        return _steps_plain(s["g"].float()).to(torch.bfloat16)
    return _update_plain(s)


# ---------------------------------------------------------------------------------------------------- the library's calls
def _weights(s):
    """The 4-bit weights as the library's calls take them, made once and kept with the state."""
    if "w4" not in s:
        import paper_2007_09835_b200 as rt3d
        c = s["case"]
        s["w4"] = rt3d.W4Weights(c["m"], c["k"], c["group"], s["codes"], s["scales"], s["zeros"])
    return s["w4"]


def _workspace(s):
    if "workspace" not in s:
        import paper_2007_09835_b200 as rt3d
        s["workspace"] = torch.empty(rt3d.rt3d_ortho_workspace(s["case"]["m"], s["case"]["k"]), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _run_own(s):
    import paper_2007_09835_b200 as rt3d
    c = s["case"]
    if c["op"] == "quantize":
        rt3d.rt3d_w4_quantize(s["w"], _weights(s))
        rt3d.rt3d_w4_unpack(_weights(s), s["values"])
        out = {"scales": s["scales"], "values": s["values"]}
        if c["zeros"]:
            out["zeros"] = s["zeros"]
        return out
    if c["op"] == "linear":
        rt3d.rt3d_linear_w4(s["x"], _weights(s), s["bias"], s["y"], relu=c["relu"])
        return s["y"].view(c["rows"], -1)[:, :c["m"]]
    if c["op"] == "ortho":
        rt3d.rt3d_orthogonalize(s["g"], s["out"], _workspace(s))
        return s["out"]
    rt3d.rt3d_ortho_update(s["w"], s["momentum"], s["g"], s["mask"], _workspace(s), lr=LR, momentum_factor=MU, nesterov=True,
                           weight_decay=DECAY, scale=_scale(c))
    return {"w": s["w"], "momentum": s["momentum"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# --------------------------------------------------------------------------------------------------- 64 bits, and floors
def exact(case, seed):
    s = prepare(case, seed)
    m, k = case["m"], case["k"]

    def direction(u):
        x = u.t() if m > k else u
        x = x / (torch.linalg.matrix_norm(x) + EPS)
        for _ in range(5):
            gram = torch.mm(x, x.t())
            x = COEF[0] * x + torch.mm(COEF[1] * gram + COEF[2] * torch.mm(gram, gram), x)
        return x.t() if m > k else x

    if case["op"] == "quantize":
        group = case["group"]
        scales = torch.zeros(m, -(-k // group), dtype=torch.float64, device="cuda")
        values = torch.zeros(m, k, dtype=torch.float64, device="cuda")
        for g in range(scales.shape[1]):
            v = s["w"][:, g * group:(g + 1) * group].double()
            if case["zeros"]:
                step = (v.max(1).values.clamp(min=0) - v.min(1).values.clamp(max=0)) / 15
                step = step.to(torch.bfloat16).double()
                zero = torch.round(-v.min(1).values.clamp(max=0) / step).clamp(0, 15)[:, None]
            else:
                step = (v.abs().max(1).values / 7).to(torch.bfloat16).double()
                zero = torch.full((m, 1), 8, dtype=torch.float64, device="cuda")
            scales[:, g] = step
            values[:, g * group:(g + 1) * group] = torch.nan_to_num(((torch.round(v / step[:, None]) + zero).clamp(0, 15) - zero) * step[:, None])
        out = {"scales": _tiled(scales, m), "values": values}
        if case["zeros"]:
            out["zeros"] = None
        return out
    if case["op"] == "linear":
        y = s["bias"].double().repeat(case["rows"], 1)
        x = s["x"].view(case["rows"], -1).double()
        scales = _untiled(s["scales"], m).double()
        zeros = None if s["zeros"] is None else _untiled(s["zeros"], m).double()
        for g in range(scales.shape[1]):
            at = slice(g * case["group"], min(k, (g + 1) * case["group"]))
            q = s["plain_codes"][:, at].double() - (8 if zeros is None else zeros[:, g:g + 1])
            y += torch.mm(x[:, at], q.t()) * scales[:, g]
        return torch.relu(y) if case["relu"] else y
    if case["op"] == "ortho":
        return direction(s["g"].double())
    keep = torch.ones(m, k, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"] > 0
    g = s["g"].double() * keep
    momentum = (MU * s["momentum"].double() + g) * keep
    w = s["w"].double() * (1 - LR * DECAY) - LR * _scale(case) * direction(g + MU * momentum)
    return {"w": w * keep, "momentum": momentum}


def work(case):
    """What a pass cannot do without.  Of the orthogonalisation: one product of the matrix with its transpose (of which the
    result is symmetric), one product that applies the polynomial, and two symmetric products of the small side for each
    step; of the rest: each input once, each output once."""
    m, k = case["m"], case["k"]
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] in ("quantize", "linear"):
        packed = m * k / 2 + m * -(-k // case["group"]) * (3 if case["zeros"] else 2)
        if case["op"] == "quantize":
            return {"bytes": m * k * (size + 4) + 2 * packed, "flops": 4 * m * k}
        return {"bytes": packed + 4 * m + size * case["rows"] * (m + k), "flops": 2 * case["rows"] * m * k}
    a, b = min(m, k), max(m, k)
    flops = 3 * a * a * b + 5 * 2 * a ** 3
    if case["op"] == "ortho":
        return {"bytes": m * k * (size + 2), "flops": flops}
    return {"bytes": m * k * (size + 16 + (1 if case["mask"] else 0)), "flops": flops}
