"""4-bit weights in numpy: the quantisation of include/rt3d.h in fp32 as it is defined, its layout, and products in 64 bits."""
import numpy as np


def bf16(a):
    """float32 -> float32 rounded to bfloat16, ties to even (finite values)."""
    u = np.asarray(a, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)


def quantize(w, group, zeros):
    """w float32 [m][k] -> codes uint8 [m][k], scales float32 [m][groups] (bfloat16 values), zero points uint8 [m][groups]."""
    m, k = w.shape
    g = -(-k // group)
    full = np.zeros((m, g * group), np.float32)
    full[:, :k] = w
    v = full.reshape(m, g, group)
    bad = ~np.isfinite(v).all(2)
    v = np.where(bad[..., None], np.float32(0), v)
    low, high = np.minimum(v.min(2), 0), np.maximum(v.max(2), 0)
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        raw = (high - low) / np.float32(15) if zeros else np.maximum(high, -low) / np.float32(7)
        bad |= ~np.isfinite(raw)
        scale = bf16(np.where(bad, 0, raw).astype(np.float32))
        bad |= ~np.isfinite(scale)
        scale = np.where(bad, np.float32(0), scale)
        zero = np.where(scale > 0, np.clip(np.rint(-low / scale), 0, 15), 8) if zeros else np.full((m, g), 8.0)
        code = np.clip(np.rint(v / scale[..., None]) + zero[..., None], 0, 15)
    code = np.where(scale[..., None] > 0, code, 8).reshape(m, g * group)[:, :k]
    return code.astype(np.uint8), np.where(bad, np.float32("nan"), scale).astype(np.float32), zero.astype(np.uint8)


def laid_out(codes, fill):
    """codes [m][k] -> the layout's bytes; `fill` [m][k up to 64] and 8 for filters beyond m: what places that do not exist hold."""
    m, k = codes.shape
    mt, kb = -(-m // 16), -(-k // 64)
    full = np.full((mt * 16, kb * 64), 8, np.uint32)
    full[:m] = fill
    full[:m, :k] = codes
    out = np.zeros((mt, kb, 8, 4, 2, 2), np.uint32)                     # tile, block, g, t, half, h
    for i in range(16):
        g, h = i % 8, i // 8
        for half in range(2):
            for t in range(4):
                for e in range(8):
                    out[:, :, g, t, half, h] |= full.reshape(mt, 16, kb, 64)[:, i, :, 32 * half + 8 * t + e] << (4 * ((e >> 1) + 4 * (e & 1)))
    return out.reshape(-1).view(np.uint8)


def tiled(per_filter, fill=0):
    """[m][groups] -> [tile][groups][16]."""
    m, g = per_filter.shape
    full = np.full((-(-m // 16) * 16, g), fill, per_filter.dtype)
    full[:m] = per_filter
    return full.reshape(-1, 16, g).transpose(0, 2, 1)


def values(codes, scales, zeros, group):
    k = codes.shape[1]
    spread = lambda a: np.repeat(a.astype(np.float64), group, 1)[:, :k]             # noqa: E731
    return (codes.astype(np.float64) - spread(zeros)) * spread(scales)


def linear(x, w, bias, relu):
    """In 64 bits, and the sum of the products' magnitudes."""
    y, size = x.astype(np.float64) @ w.T, np.abs(x).astype(np.float64) @ np.abs(w).T
    if bias is not None:
        y, size = y + bias, size + np.abs(bias)
    return np.maximum(y, 0) if relu else y, size


def tolerance(size, k, group):
    """Every rounding of an fp32 sum is off by at most a step (2^-23, should the adder cut off) of a partial sum, which is at
    most `size`; a path from a product to the result has at most a group's additions, one for each group, the multiplication by the
    scale and the additions that join lanes, warps, CTAs and the bias (fewer than 32)."""
    return (min(group, k) + -(-k // group) + 33) * 2.0 ** -23 * size
